"""A draft step and a body step in 8 bits (tabed_draft_step_q8, tabed_draft_body_step_q8), alone and as a serving loop runs them."""
import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2601_20357_amd import binding, synth

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def bits(a):
    return torch.from_numpy(a.view(np.int16).copy() if a.dtype == np.uint16 else a.copy()).to(DEV)


# ------------------------------------------------------------------ LM head and sampler
@pytest.mark.parametrize("n,B,V,d", [(4, 1, 5000, 768), (3, 8, 4099, 80), (4, 16, 32000, 768), (5, 12, 1023, 2064), (4, 16, 777, 16), (8, 16, 9000, 512),
                                     (2, 33, 6400, 144), (8, 64, 12288, 256), (4, 40, 50261, 1040), (16, 33, 2049, 768), (2, 16, 17000, 4112), (1, 3, 8200, 1008)])
def test_draft_step_q8_is_the_bf16_step_where_that_is_exact(n, B, V, d):
    """Small integers times powers of two are exact in bf16, and so are their products' sums in fp32: both steps then have the same logits
    bit for bit, and tokens that differ only where a decision is flagged."""
    g = torch.Generator().manual_seed(V + d)
    W8 = torch.randint(-9, 10, (V, d), generator=g, dtype=torch.int8).to(DEV)
    H8 = torch.randint(-9, 10, (B * n, d), generator=g, dtype=torch.int8).to(DEV)
    top = 2.0 ** -int(np.ceil(np.log2(d) / 2 + 3))
    ws, hs = (2.0 ** torch.randint(-2, 1, (k,), generator=g).float() for k in (V, B * n))
    ws, hs = (ws * top).to(DEV), hs.to(DEV)
    W, H = (W8.float() * ws[:, None]).bfloat16(), (H8.float() * hs[:, None]).bfloat16()
    temp = torch.tensor([0.0, 1.0, 0.7] * B, device=DEV)[:B].contiguous()
    cfg = binding.make_cfg(V=V, d=d, n=n, B=B, gamma=2, h=4, w_dtype=1, seed=5)
    plain, q8 = binding.RoundBuffers(cfg), binding.RoundBuffers(cfg)
    for b in (plain, q8):
        b.weights.copy_(torch.softmax(torch.randn(B, n, generator=torch.Generator().manual_seed(3)), 1).to(DEV))
        b.draft_logits.fill_(77)
    for pos in (0, 1):
        plain.draft_step(3, pos, W, H, temp)
        call = q8.prepare_draft_step_q8(0, pos, W8, ws, H8, hs, temp)
        call.set_round(3)
        call()
    torch.cuda.synchronize()
    assert torch.equal(plain.draft_logits, q8.draft_logits)
    # the same partial maxima; sums of at most 32 exponentials in another order, 2^-19 of them at the very most, mostly 2^-23
    assert ((plain.draft_lse - q8.draft_lse).abs() <= 2e-6).all()
    flagged = (plain.draft_flags | q8.draft_flags) != 0
    same = plain.draft_tokens == q8.draft_tokens
    assert (same | flagged).all() and flagged.float().mean() < 0.5
    assert ((plain.draft_q - q8.draft_q).abs() <= 1e-5 * plain.draft_q)[same].all()


def test_draft_step_q8_of_quantised_weights_is_near_the_unquantised():
    """What a user gets: W and H quantised row by row.  Every product is off by at most half a step of either factor."""
    wl = synth.scaled(synth.WORKLOADS["serving"], V=4096 + 40, B=3)
    g = torch.Generator().manual_seed(1)
    W, H = (torch.randn(wl.V, wl.d, generator=g) * 0.02).bfloat16().to(DEV), torch.randn(wl.B * wl.n, wl.d, generator=g).bfloat16().to(DEV)
    (W8, ws), (H8, hs) = binding.quantize_rows(W), binding.quantize_rows(H)
    cfg = binding.make_cfg(V=wl.V, d=wl.d, n=wl.n, B=wl.B, gamma=1, h=4, w_dtype=1, seed=5)
    b = binding.RoundBuffers(cfg)
    b.weights.fill_(1 / wl.n)
    b.prepare_draft_step_q8(0, 0, W8, ws, H8, hs, torch.ones(wl.B, device=DEV))()
    torch.cuda.synchronize()
    Wd, Hd = W.double(), H.double()
    want = Hd @ Wd.t()
    bound = 0.51 * (hs.double()[:, None] * Wd.abs().sum(1)[None, :] + ws.double()[None, :] * Hd.abs().sum(1)[:, None]
                    + wl.d * 0.51 * hs.double()[:, None] * ws.double()[None, :])
    got = b.draft_logits.view(wl.B * wl.n, wl.V).double()
    assert ((got - want).abs() <= bound).all()


# ------------------------------------------------------------------ body
class Pair:
    """The same weights, blocks and positions on the GPU and in the reference."""

    def __init__(self, bc, rows, seed, ctx):
        g = np.random.default_rng(seed)
        self.bc, self.rows, self.w = bc, rows, synth.make_body_weights(bc, seed)
        hd, width = bc.d // bc.heads, (bc.max_ctx + 63) // 64
        blocks = rows * width + 2
        self.table = g.permutation(blocks)[:rows * width].reshape(rows, width).astype(np.int32)
        shape = (bc.layers, blocks, bc.heads, 64 * hd)
        k, v = (g.integers(-127, 128, shape).astype(np.int8) for _ in range(2))
        ks, vs = (g.uniform(0.015, 0.03, shape[:3]).astype(np.float32) for _ in range(2))
        self.caches = [({"k": k[l].copy(), "v": v[l].copy()}, {"k": ks[l].copy(), "v": vs[l].copy()}) for l in range(bc.layers)]
        self.ctx = np.asarray(ctx, np.int32)
        self.cfg = binding.make_body_cfg(layers=bc.layers, d=bc.d, heads=bc.heads, d_ff=bc.d_ff, V=bc.V, max_ctx=bc.max_ctx,
                                         rope_theta=bc.rope_theta, rms_eps=bc.rms_eps)
        self.dev = {n: [bits(a) for a in x] if isinstance(x, list) else bits(x) for n, x in self.w.items()}
        self.weights = binding.make_body_weights(self.cfg, self.dev)
        self.set_gpu(k, v, ks, vs)
        self.ws = torch.empty(binding.tabed_body_q8_workspace_bytes(self.cfg, self.gpu, rows), dtype=torch.uint8, device=DEV)
        binding.tabed_body_q8_workspace_init(self.cfg, self.gpu, rows, self.ws)
        self.ctx_dev = bits(self.ctx)

    def set_gpu(self, k, v, ks, vs):
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        self.gpu = binding.CacheQ8(t(k), t(v), t(ks), t(vs), t(self.table), self.bc.d // self.bc.heads)

    def step(self, tokens, want_h=True, want_h8=True):
        d = self.bc.d
        H = torch.zeros((self.rows, d), dtype=torch.bfloat16, device=DEV) if want_h else None
        H8 = torch.zeros((self.rows, d), dtype=torch.int8, device=DEV) if want_h8 else None
        hs = torch.zeros(self.rows, device=DEV) if want_h8 else None
        binding.tabed_draft_body_step_q8(self.cfg, self.weights, self.ws, self.rows, bits(np.asarray(tokens, np.int32)), 1, 1, self.ctx_dev, self.gpu,
                                         H, H8, hs)
        torch.cuda.synchronize()
        return H, H8, hs


def values(cache, which, hd):
    """[..., blocks, heads, 64, hd] values of bytes and scales."""
    pool, scale = cache
    return pool[which][..., ref.layout(which, hd)].astype(np.float64) * scale[which][..., None, None]


@pytest.mark.parametrize("layers,d,heads,d_ff,rows", [(1, 64, 2, 96, 3), (2, 768, 12, 1024, 4), (2, 256, 2, 512, 20), (1, 512, 8, 768, 70), (1, 1280, 10, 320, 17),
                                                      (2, 128, 4, 256, 16), (1, 2048, 16, 512, 200)])
def test_body_step_q8(layers, d, heads, d_ff, rows):
    """The sides differ by fp32 against 64 bits inside projections and norms.  A value near a border of bf16, or then of int8, comes out a step apart
    and perturbs what follows, as in the bf16 body, to whose bars H is held (relative RMS 2^-7, no entry further than 2^-6 of its row's
    largest); an appended key or value may be a bf16 step (2^-7) of itself and of its block's largest, and an int8 step, apart; H8 half a
    step and what H may."""
    bc = synth.BodyConfig(layers=layers, d=d, heads=heads, d_ff=d_ff, V=500, max_ctx=200)
    g = np.random.default_rng(d + rows)
    ctx = g.integers(0, 198, rows)
    ctx[:3] = [0, 63, 64]
    p = Pair(bc, rows, d + layers, ctx)
    hd = d // heads
    for step in range(2):
        tokens = g.integers(0, 500, rows)
        H, H8, hs = p.step(tokens, want_h=step == 0)
        y = ref.body_step(bc, p.w, p.caches, p.table, p.ctx, tokens)
        top = np.abs(y).max(1, keepdims=True)
        got8 = H8.double().cpu().numpy() * hs.double().cpu().numpy()[:, None]
        assert (np.abs(got8 - y) <= 2.0 ** -6 * top + 0.5 * top / 127 * 1.02).all()
        assert (np.abs(H8.cpu().numpy()).max(1) == 127).all()
        if H is not None:
            diff = np.abs(H.double().cpu().numpy() - y)
            assert (diff <= 2.0 ** -6 * top).all() and np.sqrt((diff ** 2).mean() / (y ** 2).mean()) <= 2.0 ** -7
        p.ctx = p.ctx + 1
        assert np.array_equal(p.ctx_dev.cpu().numpy(), p.ctx)
        # the blocks: positions before the step's are the same values up to their re-rounding, everything else untouched
        for l in range(layers):
            gpu = ({n: getattr(p.gpu, n)[l].cpu().numpy() for n in ("k", "v")}, {n: getattr(p.gpu, n + "scale")[l].cpu().numpy() for n in ("k", "v")})
            for n in ("k", "v"):
                a, b = values(gpu, n, hd), values(p.caches[l], n, hd)
                size = np.maximum(gpu[1][n], p.caches[l][1][n])[..., None, None]
                assert (np.abs(a - b) <= size * (1.01 + 127 * 2.0 ** -7) + 2.0 ** -7 * np.abs(b)).all(), (l, n)
                begun = np.zeros(a.shape[0], bool)
                begun[[p.table[r, (p.ctx[r] - 1) // 64] for r in range(rows)]] = True
                assert np.array_equal(gpu[0][n][~begun], p.caches[l][0][n][~begun]) and np.array_equal(gpu[1][n][~begun], p.caches[l][1][n][~begun])
        # a common state for the next step
        p.set_gpu(*(np.stack([c[i][n] for c in p.caches]) for i, n in ((0, "k"), (0, "v"), (1, "k"), (1, "v"))))


def test_body_step_q8_outputs_agree_and_repeat():
    """H alone, H8 alone and both: the same rows, the same cache, positions moved on once each."""
    bc = synth.BodyConfig(layers=2, d=256, heads=4, d_ff=512, V=300, max_ctx=128)
    got = []
    for h, h8 in ((True, False), (False, True), (True, True), (True, True)):
        p = Pair(bc, 9, 3, np.arange(9) * 13)
        H, H8, hs = p.step(np.arange(9) * 7, h, h8)
        got.append((H, H8, hs, p.gpu.k.clone(), p.gpu.vscale.clone()))
        assert np.array_equal(p.ctx_dev.cpu().numpy(), np.arange(9) * 13 + 1)
    both = got[2]
    for other in got:
        assert all(o is None or torch.equal(o, b) for o, b in zip(other, both))
    q, s = binding.quantize_rows(both[0].float())
    assert (q.int() - both[1].int()).abs().max() <= 2             # (H was rounded to bf16 before it was quantised here)


# ------------------------------------------------------------------ together
def test_rounds_in_8_bits_eager_and_captured():
    """Body, LM head, sampling, verification and rollback of whole rounds with the drafts of a sequence sharing their first block: reproducible bit
    for bit, captured or not, and the shared blocks stay as they were."""
    n, B, gamma, V, d = 3, 2, 3, 900, 128
    bc = synth.BodyConfig(layers=2, d=d, heads=2, d_ff=256, V=V, max_ctx=192)
    rows = n * B

    def run(captured):
        p = Pair(bc, rows, 11, [70, 90, 64, 100, 66, 127])
        p.table[1:3, 0], p.table[4:6, 0] = p.table[0, 0], p.table[3, 0]           # one prompt's first block for the drafts of a sequence
        p.set_gpu(*(getattr(p.gpu, m).cpu().numpy() for m in ("k", "v", "kscale", "vscale")))
        before = p.gpu.k[:, p.table[[0, 3], 0].tolist()].clone()
        g = torch.Generator().manual_seed(2)
        W8, ws = binding.quantize_rows((torch.randn(V, d, generator=g) * 0.2).to(DEV))
        temp = torch.tensor([1.0, 0.0], device=DEV)
        cfg = binding.make_cfg(V=V, d=d, n=n, B=B, gamma=gamma, h=4, w_dtype=1, seed=9)
        b = binding.RoundBuffers(cfg)
        H8, hs = torch.zeros((rows, d), dtype=torch.int8, device=DEV), torch.zeros(rows, device=DEV)
        target = torch.randn(B, gamma + 1, V, generator=g).to(DEV)
        first, base = torch.tensor([5, 6], dtype=torch.int32, device=DEV), p.ctx_dev.clone()
        b.update_weights(True)
        torch.cuda.synchronize()

        def round_():
            for pos in range(gamma):
                src = (first, 0) if pos == 0 else (b.draft_tokens, pos - 1)
                binding.tabed_draft_body_step_q8(p.cfg, p.weights, p.ws, rows, src, 1 if pos == 0 else gamma, n, p.ctx_dev, p.gpu, None, H8, hs)
                b.prepare_draft_step_q8(1, pos, W8, ws, H8, hs, temp)()
            b.verify(1, target, temp, fused_update=True)
            binding.tabed_draft_body_rollback(rows, n, gamma, base, b.accept_len, p.ctx_dev)

        out = []
        graph = None
        if captured:
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.stream(side):
                graph.capture_begin()
                round_()
                graph.capture_end()
            torch.cuda.current_stream().wait_stream(side)
        for _ in range(4):
            if captured:
                graph.replay()
            else:
                round_()
            torch.cuda.synchronize()
            out.append([t.clone() for t in (b.out_tokens, b.accept_len, b.weights, b.draft_logits, H8, hs, p.ctx_dev, p.gpu.k, p.gpu.vscale)])
        assert torch.equal(before, p.gpu.k[:, p.table[[0, 3], 0].tolist()])
        assert torch.equal(p.ctx_dev, base + torch.clamp(b.accept_len + 1, max=gamma).repeat_interleave(n))
        assert (b.out_tokens[:, 0] >= 0).all() and torch.isfinite(b.draft_logits).all()
        return out

    eager, again, replayed = run(False), run(False), run(True)
    for a, b, c in zip(eager, again, replayed):
        for x, y, z in zip(a, b, c):
            assert torch.equal(x, y) and torch.equal(x, z)

"""The operators on trees together, as a round of tree drafting uses them; over the draft body's own caches; captured into graphs; on two streams."""
import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 10000.0


@pytest.fixture(scope="module")
def B():
    from paper_2601_20357_amd import binding
    binding.load()
    return binding


class Model:
    """Two layers of attention, no more, in torch around the operators: enough for a tree to be scored and for what is kept to matter."""

    def __init__(self, B, rows, N, f8, V=700, heads=4, kvh=2, hd=64, layers=2, ctx=192):
        g = torch.Generator().manual_seed(5)
        self.B, self.rows, self.heads, self.kvh, self.hd, self.V, self.layers = B, rows, heads, kvh, hd, V, layers
        d = heads * hd
        rand = lambda *s: (torch.randn(*s, generator=g) * d ** -0.5).to(torch.bfloat16).to(DEV)  # noqa: E731
        self.embed = torch.randn(V, d, generator=g).to(torch.bfloat16).to(DEV)
        self.qkv, self.o, self.head = [rand((heads + 2 * kvh) * hd, d) for _ in range(layers)], [rand(d, d) for _ in range(layers)], 4 * rand(V, d)
        self.cache = B.CachePaged.allocate(rows, ctx, kvh, hd, layers, torch.float8_e4m3fn if f8 else None)
        self.ws = B.new_attention_nodes_workspace(self.cache, rows, N, heads)

    def forward(self, tokens, ctx, parents, n_nodes=None):
        """Logits [rows, N, V] of the nodes; their keys and values go into the cache.  (Products in fp32: the same row gives the same bits in any batch.)"""
        rows, N = tokens.shape
        x = self.embed[tokens.long()].float()
        for i in range(self.layers):
            qkv = (x[:, :, None, :] * self.qkv[i].float()).sum(-1).to(torch.bfloat16).view(rows, N, -1, self.hd)
            q, k, v = qkv[:, :, :self.heads], qkv[:, :, self.heads:self.heads + self.kvh], qkv[:, :, self.heads + self.kvh:]
            turned, out = torch.empty(rows, N, self.heads, self.hd, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, N, self.heads, self.hd, dtype=torch.bfloat16, device=DEV)
            self.B.tabed_cache_append_nodes(self.cache, k, v, ctx, parents=parents, n_nodes=n_nodes, q=q, q_out=turned, rope_theta=THETA, layer=i)
            self.B.tabed_attention_nodes(self.cache, self.ws, turned, ctx, out, parents=parents, n_nodes=n_nodes, layer=i)
            x = x + (out.flatten(2).float()[:, :, None, :] * self.o[i].float()).sum(-1)
        return (x[:, :, None, :] * self.head.float()).sum(-1).contiguous()

    def held(self, length):
        """What the cache holds of every row's first `length` tokens, all layers, in bits."""
        at = torch.arange(length, device=DEV)
        page, slot = self.cache.table.long()[:, at // 64], at % 64
        bits = torch.int16 if self.cache.kscale is None else torch.uint8
        return [x.view(bits)[:, page, :, slot] for x in (self.cache.k, self.cache.v)] + ([] if self.cache.kscale is None else [self.cache.kscale[:, page, :, slot]])


@pytest.mark.parametrize("f8", [False, True])
def test_rounds_of_tree_drafting(B, f8):
    """Append, attention, verification, keep, over several rounds; then the emitted text alone, as chains, leaves the same bits in the cache: a node's position is
    its depth's, and what is kept is what a chain would have written."""
    rows, N, n, rounds = 3, 9, 2, 6
    model, again = Model(B, rows, N, f8), Model(B, rows, N, f8)
    g = torch.Generator().manual_seed(1)
    cfg = B.make_cfg(V=model.V, d=64, n=n, B=rows, gamma=8, h=4, w_dtype=1, seed=3)
    ws = B.new_verify_nodes_workspace(cfg, N)
    parents = torch.stack([ref.tree(N, "random", r) for r in range(rows)]).to(DEV)
    temp, weights = torch.tensor([1.0, 0.0, 0.7], device=DEV), torch.full((rows, n), 0.5, device=DEV)
    ctx = torch.zeros(rows, dtype=torch.int32, device=DEV)
    last = torch.tensor([5, 6, 7], dtype=torch.int32, device=DEV)
    texts = [[int(x)] for x in last]
    ring, head, count = torch.zeros(rows, 4, n, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV), torch.zeros(rows, dtype=torch.int32, device=DEV)
    accepted = 0
    for rnd in range(rounds):
        # Drafts: noise around what the target will say, node by node in order of depth (the target's own logits of a first pass over guesses).
        tokens = torch.randint(0, model.V, (rows, N), generator=g).to(torch.int32).to(DEV)
        tokens[:, 0] = last
        for _ in range(3):                                                # guesses settle level by level
            logits = model.forward(tokens, ctx, parents)
            best = logits.argmax(-1).to(torch.int32)
            for r in range(rows):
                for j in range(1, N):
                    if j % 4:
                        tokens[r, j] = best[r, ref.parent(parents.cpu(), r, j)]
        drafts = (logits[:, :, None] + 0.3 * torch.randn(rows, N, n, model.V, generator=g).to(DEV)).transpose(0, 1).contiguous()
        T = torch.where(temp > 0, temp, 1.0)[None, :, None]
        lse = torch.logsumexp(drafts.double() / T[..., None], -1)
        mix = (torch.exp(drafts.double() / T[..., None] - lse[..., None]) * weights[None, :, :, None]).sum(2)
        up = parents.clamp(min=0).long()
        q = torch.stack([mix[up[r], r].gather(1, tokens[r].long()[:, None])[:, 0] for r in range(rows)]).float().contiguous()
        target = model.forward(tokens, ctx, parents)
        o = {k: torch.empty(rows, N, dtype=t, device=DEV) for k, t in (("path", torch.int32), ("out", torch.int32), ("flags", torch.uint8))}
        n_path, valid, new_ctx = (torch.empty(rows, dtype=torch.int32, device=DEV) for _ in range(3))
        dev = torch.zeros(rows, 8, n, device=DEV)
        B.tabed_verify_nodes(cfg, ws, rnd, target, drafts, lse, tokens, q, weights, temp, o["path"], n_path, o["out"], o["flags"], parents=parents, dev=dev, n_valid=valid)
        B.tabed_update_weights(cfg, ws, rnd + 1, dev, valid, ring, head, count, weights)
        B.tabed_cache_keep_nodes(model.cache, ctx, o["path"], n_path, new_ctx)
        assert torch.equal(new_ctx, ctx + n_path) and torch.allclose(weights.sum(1), torch.ones(rows, device=DEV), atol=1e-6)
        for r in range(rows):
            said = o["out"][r, :n_path[r]].tolist()
            assert all(0 <= t < model.V for t in said) and (o["out"][r, n_path[r]:] == -1).all()
            texts[r] += said
            last[r] = said[-1]
            accepted += len(said) - 1
        ctx = new_ctx.clone()
    assert accepted > rounds
    # The text so far, but for the last token, which no cache holds yet, as chains of up to N tokens.
    have = torch.zeros(rows, dtype=torch.int32, device=DEV)
    assert ctx.tolist() == [len(t) - 1 for t in texts]
    while int((ctx - have).max()) > 0:
        part = (ctx - have).clamp(max=N)
        tokens = torch.zeros(rows, N, dtype=torch.int32, device=DEV)
        for r in range(rows):
            piece = texts[r][int(have[r]):int(have[r]) + int(part[r])]
            tokens[r, :len(piece)] = torch.tensor(piece, dtype=torch.int32)
        again.forward(tokens, have, None, part)
        have = have + part
    # (The first layer's keys and values depend on the token and its position alone: the same bits.  Later ones come through attention, whose sums are in another order.)
    for a, b in zip(model.held(int(ctx.min())), again.held(int(ctx.min()))):
        assert torch.equal(a[0], b[0])
    if not f8:
        k1, k2 = (m.cache.k[1][m.cache.table.long()[:, 0], :, :min(64, int(ctx.min()))].float() for m in (model, again))
        # one part in 2^5 of the largest: bf16's rounding (2^-8) through one layer's attention and two products
        assert (k1 - k2).abs().max() <= 2.0 ** -5 * k1.abs().max()


def test_over_the_draft_bodys_caches(B):
    """The caches that tabed_draft_body_step has filled, seen as paged ones: attention over them, and a tree's nodes behind what they hold."""
    layers, rows, heads, hd, max_ctx = 2, 3, 4, 64, 128
    d = heads * hd
    bcfg = B.make_body_cfg(layers=layers, d=d, heads=heads, d_ff=512, V=500, max_ctx=max_ctx)
    body = B.BodyBuffers(bcfg, rows, body_tensors(layers, d))
    tok = torch.randint(0, 500, (70,), generator=torch.Generator().manual_seed(1)).to(torch.int32).to(DEV)
    for i in range(70):
        body.prepare_step(tok, i, 0, 1)()
    torch.cuda.synchronize()
    cache = B.CachePaged.of_body(body.kcache.view(layers, rows, max_ctx, d), body.vcache.view(layers, rows, max_ctx, d), heads)
    N = 6
    g = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(rows, N, heads, hd, generator=g).to(torch.bfloat16) for _ in range(3))
    parents = torch.stack([ref.tree(N, "random", r) for r in range(rows)])
    ctx = body.ctx_len.clone()
    assert ctx.tolist() == [70] * rows
    ws = B.new_attention_nodes_workspace(cache, rows, N, heads)
    for layer in range(layers):
        before = body.kcache.view(layers, rows, max_ctx, d).clone()
        out, lse = torch.empty(rows, N, heads, hd, dtype=torch.bfloat16, device=DEV), torch.empty(rows, N, heads, device=DEV)
        B.tabed_cache_append_nodes(cache, k.to(DEV), v.to(DEV), ctx, parents=parents.to(DEV), layer=layer)
        B.tabed_attention_nodes(cache, ws, q.to(DEV), ctx, out, parents=parents.to(DEV), lse=lse, layer=layer)
        now = body.kcache.view(layers, rows, max_ctx, d)
        assert torch.equal(now[layer, :, 70:76].cpu(), k.flatten(2))
        now[layer, :, 70:76] = before[layer, :, 70:76]
        assert torch.equal(now, before)
        now[layer, :, 70:76] = k.flatten(2).to(DEV)
        kk, vv = (x.view(layers, rows * max_ctx // 64, 64, heads, hd)[layer].transpose(1, 2).cpu().double() for x in (body.kcache, body.vcache))
        want, wlse, mass = ref.attention(q.double(), kk, vv, cache.table.cpu(), rows * max_ctx // 64, [70] * rows, parents, [N] * rows, hd ** -0.5)
        tol = 2.0 ** -8 * want.abs() + mass * (2.0 ** -8 + 2.0 ** -12)
        assert ((out.cpu().double() - want).abs() <= tol).all() and ((lse.cpu().double() - wlse).abs() <= 2.0 ** -14).all()


def body_tensors(layers, d, d_ff=512, V=500):
    g = torch.Generator().manual_seed(3)
    m = lambda *s: (0.02 * torch.randn(*s, generator=g)).to(torch.bfloat16).to(DEV)  # noqa: E731
    gain = lambda: (1 + 0.1 * torch.randn(d, generator=g)).to(DEV)  # noqa: E731
    return {"embed": torch.randn(V, d, generator=g).to(torch.bfloat16).to(DEV), "g_final": gain(), "g_attn": [gain() for _ in range(layers)],
            "wqkv": [m(3 * d, d) for _ in range(layers)], "wo": [m(d, d) for _ in range(layers)], "g_mlp": [gain() for _ in range(layers)],
            "wgu": [m(2 * d_ff, d) for _ in range(layers)], "wdown": [m(d, d_ff) for _ in range(layers)]}


@pytest.mark.parametrize("f8", [False, True])
def test_captured_calls_share_a_workspace_with_eager_ones(B, f8):
    """Append and attention of two sizes captured into a graph each, on one workspace; replayed with other inputs in the same places, eager calls in between."""
    g = torch.Generator().manual_seed(4)
    sets, most = [], 0
    for rows, N, heads, kvh, hd, ctx in ((1, 5, 4, 2, 128, [5000]), (3, 40, 8, 2, 128, [2500, 10, 700])):
        cache = B.CachePaged.allocate(rows, max(ctx) + N, kvh, hd, dtype=torch.float8_e4m3fn if f8 else None)
        full = torch.randn(rows, 250, kvh, hd, generator=g).to(torch.bfloat16).to(DEV)
        for at in range(0, max(ctx), 250):
            B.tabed_cache_append_nodes(cache, full, full.flip(1).contiguous(), torch.full((rows,), at, dtype=torch.int32, device=DEV))
        x = {n: torch.zeros(rows, N, h, hd, dtype=torch.bfloat16, device=DEV) for n, h in (("q", heads), ("k", kvh), ("v", kvh), ("turned", heads), ("out", heads))}
        sets.append((cache, x, torch.tensor(ctx, dtype=torch.int32, device=DEV), torch.stack([ref.tree(N, "random", r) for r in range(rows)]).to(DEV), heads, N, rows))
        most = max(most, B.tabed_attention_nodes_workspace_bytes(cache, rows, N, heads))
    ws = torch.empty(most, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    graphs = []
    for cache, x, ctx, parents, heads, N, rows in sets:
        B.tabed_attention_nodes_workspace_init(cache, rows, N, heads, ws)
        calls = [B.prepare_cache_append_nodes(cache, x["k"], x["v"], ctx, parents=parents, q=x["q"], q_out=x["turned"], rope_theta=THETA, stream=side),
                 B.prepare_attention_nodes(cache, ws, x["turned"], ctx, x["out"], parents=parents, stream=side)]
        torch.cuda.synchronize()
        for call in calls:
            call()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            for call in calls:
                call()
        graphs.append(graph)
    for i in range(4):
        for graph, (cache, x, ctx, parents, heads, N, rows) in zip(graphs, sets):
            for n in ("q", "k", "v"):
                x[n].copy_(torch.randn(x[n].shape, generator=g))
            graph.replay()
            got = x["out"].clone()
            x["out"].zero_()
            turned, out = torch.empty_like(x["turned"]), torch.empty_like(x["out"])
            B.tabed_cache_append_nodes(cache, x["k"], x["v"], ctx, parents=parents, q=x["q"], q_out=turned, rope_theta=THETA)
            B.tabed_attention_nodes(cache, ws, turned, ctx, out, parents=parents)
            assert torch.equal(got, out) and torch.equal(turned, x["turned"]), i
            assert bool(torch.isfinite(out.float()).all()) and float(out.float().abs().max()) > 0


def test_two_streams_with_workspaces_of_their_own(B):
    cases = []
    for seed in (1, 2):
        g = torch.Generator().manual_seed(seed)
        cache = B.CachePaged.allocate(2, 4000, 4, 64)
        cache.k.copy_(torch.randn(cache.k.shape, generator=g))
        cache.v.copy_(torch.randn(cache.v.shape, generator=g))
        q = torch.randn(2, 12, 8, 64, generator=g).to(torch.bfloat16).to(DEV)
        ctx = torch.tensor([3900, 1000 * seed], dtype=torch.int32, device=DEV)
        want = torch.empty_like(q)
        B.tabed_attention_nodes(cache, B.new_attention_nodes_workspace(cache, 2, 12, 8), q, ctx, want)
        cases.append((cache, q, ctx, want, torch.cuda.Stream(), B.new_attention_nodes_workspace(cache, 2, 12, 8), torch.empty_like(q)))
    torch.cuda.synchronize()
    for _ in range(20):
        for cache, q, ctx, want, stream, ws, out in cases:
            B.tabed_attention_nodes(cache, ws, q, ctx, out, stream=stream)
    torch.cuda.synchronize()
    for case in cases:
        assert torch.equal(case[3], case[6])

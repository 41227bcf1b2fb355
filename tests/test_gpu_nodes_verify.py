"""Verification of trees of drafted tokens against its definition in 64 bits, against the chain's, and by what it is for: the target's distribution."""
import math

import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def binding():
    from paper_2601_20357_amd import binding
    binding.load()
    return binding


def make(B, N, n, V, kind="random", seed=0, temp=None, spread=2.0, noise=0.7, ragged=False):
    """Inputs on the CPU; a node's token is drawn from its parent's mixture."""
    g = torch.Generator().manual_seed(seed * 31 + V)
    c = {"parents": None if kind == "chain" else torch.stack([ref.tree(N, kind, seed + b) for b in range(B)])}
    c["nodes"] = torch.randint(0, N + 1, (B,), generator=g) if ragged else torch.full((B,), N)
    c["temp"] = torch.tensor([(temp or [1.0, 0.0, 0.6])[b % len(temp or [0] * 3)] for b in range(B)])
    base = spread * torch.randn(B, N, V, generator=g)
    c["target"] = base + noise * torch.randn(B, N, V, generator=g)
    c["drafts"] = (base.transpose(0, 1)[:, :, None] + torch.randn(N, B, n, V, generator=g)).contiguous()
    T = torch.where(c["temp"] > 0, c["temp"], 1.0).double()[:, None, None]
    c["lse"] = torch.logsumexp(c["drafts"].double() / T, -1)
    w = torch.rand(B, n, generator=g) + 0.1
    c["weights"] = w / w.sum(1, keepdim=True)
    mix = (torch.exp(c["drafts"].double() / T - c["lse"][..., None]) * c["weights"][..., None]).sum(2)            # [N, B, V]
    c["tokens"], c["q"] = torch.zeros(B, N, dtype=torch.int32), torch.ones(B, N)
    for b in range(B):
        for j in range(1, N):
            p = ref.parent(c["parents"], b, j)
            row = mix[max(p, 0), b]
            y = int(torch.multinomial(row.float(), 1, generator=g)) if c["temp"][b] > 0 or j % 2 else int(row.argmax())
            c["tokens"][b, j], c["q"][b, j] = y, float(row[y])
    c["u_acc"], c["u_res"] = torch.rand(B, N, generator=g), torch.rand(B, generator=g)
    return c


def run(binding, c, gamma=None, ws=None, cfg=None, stream=None, rnd=0, uniforms=True, **cfg_more):
    B, N, V = c["target"].shape
    n = c["drafts"].shape[2]
    gamma = gamma or min(32, N)
    cfg = cfg or binding.make_cfg(V=V, d=64, n=n, B=B, gamma=gamma, h=8, w_dtype=1, seed=77, **cfg_more)
    ws = binding.new_verify_nodes_workspace(cfg, N) if ws is None else ws
    dev = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    o = {"path": torch.full((B, N), 99, dtype=torch.int32, device=DEV), "n_path": torch.full((B,), 99, dtype=torch.int32, device=DEV),
         "out": torch.full((B, N), 99, dtype=torch.int32, device=DEV), "flags": torch.full((B, N), 99, dtype=torch.uint8, device=DEV),
         "dev": torch.full((B, gamma, n), 7.0, device=DEV), "n_valid": torch.full((B,), 99, dtype=torch.int32, device=DEV)}
    i32 = lambda t: None if t is None else t.to(torch.int32).to(DEV)  # noqa: E731
    call = binding.prepare_verify_nodes(cfg, ws, rnd, dev(c["target"]), dev(c["drafts"]), dev(c["lse"]), i32(c["tokens"]), dev(c["q"]), dev(c["weights"]), dev(c["temp"]),
                                        o["path"], o["n_path"], o["out"], o["flags"], parents=i32(c["parents"]), n_nodes=i32(c["nodes"]),
                                        u_acc=dev(c["u_acc"]) if uniforms else None, u_res=dev(c["u_res"]) if uniforms else None, dev=o["dev"], n_valid=o["n_valid"],
                                        stream=stream)
    call()
    return o, call, ws


def check(binding, c, gamma=None, tvd=False, ws=None):
    B, N, V = c["target"].shape
    gamma = gamma or min(32, N)
    o, _, _ = run(binding, c, gamma, ws, distance=int(tvd))
    rows = ref.verify(c["target"], c["drafts"], c["lse"], c["tokens"], c["q"], c["parents"], c["nodes"], c["weights"], c["temp"], c["u_acc"], c["u_res"], gamma, tvd)
    o = {k: v.cpu() for k, v in o.items()}
    for b, (path, out, flags, last, dist, close) in enumerate(rows):
        assert close > 1e-10, "inputs too close to a decision's border"
        pad = [-1] * (N - len(path))
        assert o["n_path"][b] == len(path) and o["path"][b].tolist() == path + pad, b
        assert o["out"][b].tolist() == out + pad, b
        want = [flags.get(j, 0) for j in range(N)]
        want[0] = last if c["temp"][b] > 0 else 0
        assert o["flags"][b].tolist() == want, b
        assert o["n_valid"][b] == len(dist)
        # Sums in fp64 over V terms, then one rounding to fp32 (2^-24); differences of sums of up to about 10^2.
        got = o["dev"][b].double()
        for i, d in enumerate(dist):
            d = torch.tensor(d, dtype=torch.float64)
            fin = torch.isfinite(d)
            assert torch.equal(got[i][~fin], d[~fin])
            assert ((got[i] - d).abs()[fin] <= 2.0 ** -24 * d.abs()[fin] + 1e-11).all(), (b, i)
        assert (got[len(dist):] == 7).all()
    return o


@pytest.mark.parametrize("V", [1, 2, 3, 4, 5, 63, 257, 1000, 2047, 2048, 2049, 4097, 9001])
def test_vocabularies(binding, V):
    check(binding, make(5, 9, 2, V, seed=V))


@pytest.mark.parametrize("B,V", [(1, 65536), (1, 65537), (4, 65533), (5, 65536), (85, 2999), (86, 2999), (3, 32001)])
@pytest.mark.parametrize("tvd", [False, True])
def test_sizes_of_pieces(binding, B, V, tvd):
    check(binding, make(B, 5, 3 if B < 50 else 1, V, seed=B), tvd=tvd)


@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 8, 15, 16])
def test_drafts(binding, n):
    check(binding, make(4, 7, n, 3000, seed=n))
    check(binding, make(4, 7, n, 777, seed=n), tvd=True)


@pytest.mark.parametrize("kind", ["chain", "star", "deep", "random", "forest"])
@pytest.mark.parametrize("N", [1, 2, 30, 65, 256])
def test_trees(binding, N, kind):
    check(binding, make(4, N, 2, 300, kind=kind, seed=N, ragged=N > 2, noise=0.2))


@pytest.mark.parametrize("spread,noise", [(0.1, 0.05), (1.0, 3.0), (6.0, 0.5)])
def test_distributions(binding, spread, noise):
    check(binding, make(12, 16, 3, 5000, spread=spread, noise=noise, seed=3, temp=[1.0, 0.25, 3.0, 0.0]))


def test_large_vocabulary_and_batch(binding):
    check(binding, make(2, 6, 2, 262144, seed=1))
    check(binding, make(70, 12, 2, 2500, seed=2, ragged=True), gamma=3)


def test_tokens_outside_and_repeated(binding):
    c = make(8, 12, 2, 500, kind="star", seed=5, temp=[1.0, 0.0], noise=3.0)
    c["tokens"][:, 3], c["tokens"][:, 5], c["tokens"][:, 7] = -1, 500, 2 ** 31 - 1
    c["tokens"][:, 8] = c["tokens"][:, 1]
    c["u_acc"][:, :9] = 1.0 - 2.0 ** -24
    o = check(binding, c)
    assert (o["flags"][:, [3, 5, 7]] == 4).any()                                     # (in the rows where none before them was accepted)


def test_masked_logits_and_ties(binding):
    c = make(6, 8, 2, 600, seed=6)
    c["target"][:, :, 100:400] = -math.inf
    c["target"][:, :, 500] = c["target"][:, :, 37] = c["target"].amax() + 1.0            # greedy: the lower index
    check(binding, c)
    c["drafts"][..., 50:60] = -math.inf
    c["lse"] = torch.logsumexp(c["drafts"].double() / torch.where(c["temp"] > 0, c["temp"], 1.0).double()[:, None, None], -1)
    o = check(binding, c)                                                             # the target has mass where a draft has none: an infinite distance
    assert torch.isinf(o["dev"]).any()


def test_no_mass_left(binding):
    """Target and draft alike: behind a rejection nothing is left, and the draw is from p, flagged."""
    c = make(3, 3, 1, 64, kind="star", seed=7, temp=[1.0])
    c["target"][:] = -math.inf
    c["target"][:, :, 5] = 3.0
    c["drafts"][:] = -math.inf
    c["drafts"][..., 5] = 3.0
    c["lse"][:] = 3.0
    c["tokens"][:, 1:], c["q"][:] = 6, 1.0
    c["u_acc"][:] = 0.999
    o, _, _ = run(binding, c)
    assert o["out"][:, 0].tolist() == [5] * 3 and o["flags"][:, 0].tolist() == [4] * 3 and o["n_path"].tolist() == [1] * 3


def test_nan_logits_end_flagged(binding):
    c = make(3, 4, 2, 3000, seed=8, temp=[1.0])
    c["target"][1, 0, 17] = math.nan
    o, _, _ = run(binding, c)
    assert o["n_path"][1] == 1 and o["path"][1].tolist() == [0, -1, -1, -1] and o["flags"][1, 0] == 4 and 0 <= int(o["out"][1, 0]) < 3000


def test_as_the_chain_is_verified(binding):
    """A chain of gamma + 1 nodes, and tabed_verify with the same round: the same tokens, lengths and distances, with Philox's uniforms and with explicit ones."""
    gamma, Bn, n, V = 5, 24, 3, 2000
    c = make(Bn, gamma + 1, n, V, kind="chain", seed=11, temp=[1.0, 0.7])
    for uniforms in (False, True):
        o, _, _ = run(binding, c, gamma=gamma, rnd=9, uniforms=uniforms)
        cfg = binding.make_cfg(V=V, d=64, n=n, B=Bn, gamma=gamma, h=8, w_dtype=1, seed=77)
        ws = binding.new_workspace(cfg)
        k, out = torch.empty(Bn, dtype=torch.int32, device=DEV), torch.empty(Bn, gamma + 1, dtype=torch.int32, device=DEV)
        dev, valid = torch.empty(Bn, gamma, n, device=DEV), torch.empty(Bn, dtype=torch.int32, device=DEV)
        flags = torch.empty(Bn, gamma + 1, dtype=torch.uint8, device=DEV)
        u = dict(u_acc=c["u_acc"][:, 1:].contiguous().to(DEV), u_res=c["u_res"].to(DEV)) if uniforms else {}
        binding.tabed_verify(cfg, ws, 9, c["target"].to(DEV), c["drafts"][:gamma].contiguous().to(DEV), c["lse"][:gamma].contiguous().to(DEV),
                             c["tokens"][:, 1:].contiguous().to(DEV), c["q"][:, 1:].contiguous().to(DEV), c["weights"].to(DEV), c["temp"].to(DEV), k, out, dev, valid, flags, **u)
        sure = (flags == 0).all(1)
        assert sure.sum() > Bn // 2
        assert torch.equal(o["n_path"][sure], k[sure] + 1) and torch.equal(o["out"][sure], out[sure]) and torch.equal(o["n_valid"][sure], valid[sure])
        for b in range(Bn):
            if sure[b]:
                m = int(valid[b])
                # (there in fp32 with sums in fp64: 2^-20 of terms of some tens)
                assert ((o["dev"][b, :m] - dev[b, :m]).abs() <= 1e-5 * dev[b, :m].abs() + 2e-5).all()


def test_chain_without_the_last_slot(binding):
    c = make(4, 6, 2, 900, kind="chain", seed=12)
    a, _, _ = run(binding, c)
    c["drafts"], c["lse"] = c["drafts"][:5].contiguous(), c["lse"][:5].contiguous()
    b, _, _ = run(binding, c)
    for k in a:
        assert torch.equal(a[k], b[k])


@pytest.mark.parametrize("kind", ["star", "random"])
def test_first_token_follows_the_target(binding, kind):
    """Lossless: over many rows with Philox's uniforms, siblings drawn from q, the first token emitted is distributed as p (chi-square, 1 in 10^6)."""
    Bn, N, V, n = 40_000, 4, 6, 2
    g = torch.Generator().manual_seed(3)
    c = make(1, N, n, V, kind=kind, seed=4, temp=[1.0], noise=1.0, spread=1.0)
    p = torch.softmax(c["target"][0, 0].double(), 0)
    mix = (torch.exp(c["drafts"][:, 0].double() - c["lse"][:, 0][..., None]) * c["weights"][0][:, None]).sum(1)          # [N, V]
    big = {"parents": None if c["parents"] is None else c["parents"].expand(Bn, N).contiguous(), "nodes": torch.full((Bn,), N), "temp": torch.ones(Bn),
           "target": c["target"].expand(Bn, N, V).contiguous(), "drafts": c["drafts"].expand(N, Bn, n, V).contiguous(), "lse": c["lse"].expand(N, Bn, n).contiguous(),
           "weights": c["weights"].expand(Bn, n).contiguous(), "u_acc": None, "u_res": None}
    tokens, q = torch.zeros(Bn, N, dtype=torch.int32), torch.ones(Bn, N)
    for j in range(1, N):
        row = mix[ref.parent(c["parents"], 0, j)].float()
        y = torch.multinomial(row, Bn, replacement=True, generator=g)
        tokens[:, j], q[:, j] = y.to(torch.int32), row[y]
    big["tokens"], big["q"] = tokens, q
    o, _, _ = run(binding, big, uniforms=False, rnd=5)
    seen = torch.bincount(o["out"][:, 0].cpu().long(), minlength=V).double()
    chi = float(((seen - Bn * p) ** 2 / (Bn * p)).sum())
    assert chi < 36.2, (seen / Bn, p)                                                  # 5 degrees of freedom: 10^-6 above 36.2
    assert int((o["n_path"] > 1).sum()) > Bn // 4


# ------------------------------------------------------------------ workspaces, streams, graphs
def test_one_workspace_for_all_sizes(binding):
    cases = [make(3, 9, 2, 5000, seed=1), make(1, 40, 1, 9000, seed=2), make(40, 3, 4, 300, seed=3), make(3, 9, 2, 5000, seed=4)]
    sizes = []
    for c in cases:
        Bn, N, V = c["target"].shape
        cfg = binding.make_cfg(V=V, d=64, n=c["drafts"].shape[2], B=Bn, gamma=min(32, N), h=8, w_dtype=1)
        sizes.append((binding.tabed_verify_nodes_workspace_bytes(cfg, N), cfg, N))
    ws = torch.full((max(s[0] for s in sizes),), 255, dtype=torch.uint8, device=DEV)
    _, cfg, N = max(sizes, key=lambda s: s[0])
    binding.tabed_verify_nodes_workspace_init(cfg, N, ws)
    for _ in range(2):
        for c in cases:
            check(binding, c, ws=ws)


def test_unprepared_workspace_ends_flagged(binding):
    c = make(3, 5, 2, 5000, seed=1)
    for fill in (0, 255):
        cfg = binding.make_cfg(V=5000, d=64, n=2, B=3, gamma=5, h=8, w_dtype=1)
        ws = torch.full((binding.tabed_verify_nodes_workspace_bytes(cfg, 5),), fill, dtype=torch.uint8, device=DEV)
        o, _, _ = run(binding, c, ws=ws)
        assert o["n_path"].tolist() == [0] * 3 and (o["path"] == -1).all() and (o["out"] == -1).all() and (o["flags"][:, 0] == 4).all() and (o["n_valid"] == 0).all()


def test_two_streams_at_once(binding):
    """Two verifications and a stream of products side by side, each with a workspace of its own."""
    cs = [make(16, 12, 2, 20_000, seed=s) for s in (1, 2)]
    alone = [run(binding, c)[0] for c in cs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    calls = []
    for c, s in zip(cs, streams):
        with torch.cuda.stream(s):
            calls.append(run(binding, c, stream=s))
    x = torch.randn(4096, 4096, device=DEV)
    with torch.cuda.stream(streams[2]):
        for _ in range(20):
            x = torch.mm(x, x).clamp(-1, 1)
    for _ in range(30):
        for _, call, _ in calls:
            call()
    torch.cuda.synchronize()
    for (o, _, _), want in zip(calls, alone):
        for k in o:
            assert torch.equal(o[k], want[k]), k


def test_captured_and_eager_calls_share_a_workspace(binding):
    """Two graphs and eager calls of other sizes on one workspace, one after the other; several replays each."""
    big, small = make(8, 10, 3, 7000, seed=1), make(2, 4, 2, 3000, seed=2)
    want_big, _, ws = run(binding, big)
    want_small = run(binding, small)[0]
    graphs = []
    for c in (big, small):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        o, call, _ = run(binding, c, ws=ws, stream=side)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            call()
        graphs.append((g, o, call))
    for i in range(5):
        for (g, o, _), want in zip(graphs, (want_big, want_small)):
            for t in o.values():
                t.fill_(3)
            g.replay()
            torch.cuda.synchronize()
            for k in ("path", "n_path", "out", "flags", "n_valid"):
                assert torch.equal(o[k], want[k]), (i, k)
        again = run(binding, big, ws=ws)[0]
        assert torch.equal(again["out"], want_big["out"])


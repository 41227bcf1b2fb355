"""The operators on trees of drafted tokens against their definitions in 64 bits."""
import math

import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
THETA = 10000.0
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    from paper_2601_20357_amd import binding
    binding.load()
    return binding


def gen(seed):
    return torch.Generator().manual_seed(seed)


def trees(rows, N, kind):
    if kind == "chain":
        return None
    return torch.stack([ref.tree(N, kind, r) for r in range(rows)])


def make_cache(B, rows, tokens, kvh, hd, f8=False, layers=1, by_token=False, seed=0, fill="values", spare=3):
    """A cache whose blocks lie in no order; fill: 'values', or 'nan' (every byte 0xff)."""
    g = gen(seed)
    width = max(1, (tokens + 63) // 64)
    blocks = rows * width + spare
    shape = (layers, blocks, 64, kvh, hd) if by_token else (layers, blocks, kvh, 64, hd)
    table = torch.randperm(blocks, generator=g)[:rows * width].view(rows, width).to(torch.int32)
    pool = []
    for _ in range(2):
        if fill == "nan":
            x = torch.full((*shape, 1 if f8 else 2), 255, dtype=torch.uint8).view(F8 if f8 else torch.bfloat16).squeeze(-1)
        else:
            x = torch.randn(shape, generator=g).to(torch.bfloat16)
            x = x.float().clamp(-400, 400).to(F8) if f8 else x
        x = x.to(DEV)
        pool.append(x.transpose(2, 3) if by_token else x)
    scales = [None, None]
    if f8:
        scales = [(torch.rand(layers, blocks, kvh, 64, generator=g) * 0.5 + 0.5).to(DEV) if fill != "nan" else torch.full((layers, blocks, kvh, 64), math.nan, device=DEV)
                  for _ in range(2)]
    return B.CachePaged(*pool, table.to(DEV), *scales)


def values(cache, name, layer=0):
    """The cache's keys or values, [blocks, kv_heads, 64, hd] in 64 bits on the CPU."""
    x = getattr(cache, name)
    x = (x if x.dim() == 5 else x[None])[layer].cpu().double()
    s = getattr(cache, name + "scale")
    return x if s is None else x * s.view(cache.layers, -1, cache.kv_heads, 64)[layer].cpu().double()[..., None]


# ------------------------------------------------------------------ append
def check_append(B, rows, N, qh, kvh, hd, f8=False, kind="random", src=torch.bfloat16, theta=THETA, ragged=True, by_token=False, ctx_hi=130, seed=0, layers=1, layer=0,
                 inplace=False, tokens=None):
    g = gen(seed + 1)
    tokens = ctx_hi + N if tokens is None else tokens
    cache = make_cache(B, rows, tokens, kvh, hd, f8, layers, by_token, seed)
    before = [x.clone() for x in (cache.k, cache.v)]
    parents = trees(rows, N, kind)
    ctx = torch.randint(0, ctx_hi + 1, (rows,), generator=g)
    ctx[0] = 0
    nodes = torch.randint(0, N + 1, (rows,), generator=g) if ragged else torch.full((rows,), N)
    nodes[-1] = N
    qkv = (1.3 * torch.randn(rows, N, (qh + 2 * kvh) * hd, generator=g)).to(src)
    dev = qkv.to(DEV)
    q, k, v = (dev[..., a * hd:(a + h) * hd].unflatten(-1, (h, hd)) for a, h in ((0, qh), (qh, kvh), (qh + kvh, kvh)))
    q_out = q if inplace else torch.full((rows, N, qh, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    i32 = lambda t: None if t is None else t.to(torch.int32).to(DEV)  # noqa: E731
    B.tabed_cache_append_nodes(cache, k, v, i32(ctx), parents=i32(parents), n_nodes=i32(nodes), q=q, q_out=q_out, rope_theta=theta, layer=layer)
    got_q = q_out.cpu().double()
    want = {}
    hq, hk, hv = (qkv[..., a * hd:(a + h) * hd].unflatten(-1, (h, hd)).double() for a, h in ((0, qh), (qh, kvh), (qh + kvh, kvh)))
    for r in range(rows):
        for j in range(N):
            if j >= nodes[r]:
                assert torch.equal(got_q[r, j], hq[r, j] if inplace else torch.full((qh, hd), 7.0, dtype=torch.float64))
                continue
            pos = int(ctx[r]) + len(ref.above(parents, r, j)) - 1
            x = ref.rotated(hq[r, j], pos, theta)
            # One rounding to bf16, and fp32's in the two products and the angle's sine and cosine.
            size = hq[r, j][:, :hd // 2].abs() + hq[r, j][:, hd // 2:].abs()
            assert ((got_q[r, j] - x).abs() <= 2.0 ** -8 * x.abs() + 2.0 ** -21 * size.repeat(1, 2)).all(), (r, j)
            at = ref.place(cache.table.cpu(), cache.struct.blocks, r, int(ctx[r]) + j)
            if at is not None:
                want[at] = (ref.rotated(hk[r, j], pos, theta), hv[r, j], hk[r, j])
    for name, i in (("k", 0), ("v", 1)):
        pool = getattr(cache, name)
        new, old = ((x if x.dim() == 5 else x[None]).cpu() for x in (pool, before[i]))
        same = (new.view(torch.uint8) == old.view(torch.uint8)).all(-1) if f8 else (new.view(torch.int16) == old.view(torch.int16)).all(-1)
        held = values(cache, name, layer)
        scale = getattr(cache, name + "scale")
        for (block, slot), w in want.items():
            same[layer, block, :, slot] = True
            x, got = w[i], held[block, :, slot]
            size = (w[2][:, :hd // 2].abs() + w[2][:, hd // 2:].abs()).repeat(1, 2) if i == 0 and theta else torch.zeros_like(x)
            slack = 2.0 ** -21 * size
            if not f8:
                assert ((got - x).abs() <= 2.0 ** -8 * x.abs() + slack).all()
                continue
            s = scale.view(cache.layers, -1, kvh, 64)[layer, block, :, slot].cpu().double()
            most = x.abs().amax(1)
            assert ((s - most / 448).abs() <= 2.0 ** -23 * most / 448 + slack.amax(1) / 448).all()
            # Half a step of e4m3: 2^-4 of the value, 2^-10 of the scale among the smallest; the clamp at 448 takes what the scale's rounding adds.
            assert ((got - x).abs() <= 2.0 ** -4 * x.abs() * (1 + 2.0 ** -20) + 2.0 ** -10 * s[:, None] * (1 + 2.0 ** -20) + slack).all()
        assert same.all(), "an entry that no node has was written"


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
def test_append_sizes(B, hd, f8):
    check_append(B, 3, 9, 6, 2, hd, f8, seed=hd)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("rows,N,qh,kvh,kind,src,theta,by_token", [
    (1, 1, 1, 1, "chain", torch.bfloat16, THETA, False), (2, 65, 3, 3, "chain", torch.float32, THETA, True), (2, 64, 7, 1, "random", torch.float32, 500000.0, False),
    (1, 256, 4, 2, "deep", torch.bfloat16, THETA, False), (4, 33, 5, 5, "star", torch.float32, 0.0, True), (3, 30, 8, 4, "forest", torch.bfloat16, THETA, True)])
def test_append_trees(B, rows, N, qh, kvh, kind, src, theta, by_token, f8):
    check_append(B, rows, N, qh, kvh, 64, f8, kind, src, theta, by_token=by_token, seed=N)


def test_append_in_place_layer_and_short_table(B):
    check_append(B, 2, 5, 4, 4, 64, inplace=True, layers=3, layer=2, seed=3)
    check_append(B, 3, 40, 2, 2, 64, tokens=64, ctx_hi=70, seed=4)                    # some positions are past the table


def test_append_far_positions(B):
    """The angle at positions up to 2^31 (keys past the table are dropped, queries turn all the same)."""
    cache = make_cache(B, 3, 64, 1, 64)
    ctx = torch.tensor([2 ** 31 - 1, 2 ** 24 + 1, 1_234_567_891], dtype=torch.int32)
    x = torch.randn(3, 4, 1, 64, generator=gen(5)).to(torch.bfloat16)
    out, kept = torch.empty(3, 4, 1, 64, dtype=torch.bfloat16, device=DEV), cache.k.clone()
    B.tabed_cache_append_nodes(cache, x.to(DEV), x.to(DEV), ctx.to(DEV), q=x.to(DEV), q_out=out, rope_theta=THETA)
    for r in range(3):
        for j in range(4):
            want = ref.rotated(x[r, j].double(), int(ctx[r]) + j, THETA)
            size = (x[r, j][:, :32].abs() + x[r, j][:, 32:].abs()).double().repeat(1, 2)
            # (the product of position and frequency is off by 2^-52 of 2^31 turns' radians, twice)
            assert ((out[r, j].cpu().double() - want).abs() <= 2.0 ** -8 * want.abs() + size * 2.0 ** -18).all()
    assert torch.equal(cache.k, kept)


def test_append_holes_negative_context_and_counts(B):
    cache = make_cache(B, 4, 128, 2, 64)
    cache.table[1, 0] = -1
    cache.table[2, 0] = cache.struct.blocks
    before = cache.k.clone()
    x = torch.randn(4, 3, 2, 64, generator=gen(6)).to(torch.bfloat16).to(DEV)
    ctx = torch.tensor([-5, 3, 4, 62], dtype=torch.int32, device=DEV)
    nodes = torch.tensor([99, 3, 3, -1], dtype=torch.int32, device=DEV)
    B.tabed_cache_append_nodes(cache, x, x, ctx, n_nodes=nodes)
    first = int(cache.table[0, 0])
    assert torch.equal(cache.k[0, first, :, :3], x[0].transpose(0, 1))
    cache.k[0, first, :, :3] = before[0, first, :, :3]
    assert torch.equal(cache.k, before)


def test_append_e4m3_marks_and_repeats(B):
    cache = make_cache(B, 1, 64, 4, 64, f8=True)
    x = torch.randn(1, 1, 4, 64, generator=gen(7))
    x[0, 0, 0, 5], x[0, 0, 1, 40], x[0, 0, 2], x[0, 0, 3, 0] = math.nan, -math.inf, 2.0 ** -101, 3e38
    ctx = torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tabed_cache_append_nodes(cache, x.to(DEV), x.to(DEV), ctx)
    b = int(cache.table[0, 0])
    s, k = cache.kscale[0, b, :, 0].cpu(), cache.k[0, b, :, 0].float().cpu()
    assert s[0].isnan() and s[1].isnan() and s[2] == 0 and (k[:3] == 0).all()
    assert k[3, 0] == 448 and abs(float(s[3]) * 448 / 3e38 - 1) < 2.0 ** -22 and (k[3, 1:] == 0).all()
    again = [t.clone() for t in (cache.k.view(torch.uint8), cache.kscale, cache.v.view(torch.uint8))]
    B.tabed_cache_append_nodes(cache, x.to(DEV), x.to(DEV), ctx)
    for a, t in zip(again, (cache.k.view(torch.uint8), cache.kscale, cache.v.view(torch.uint8))):
        assert torch.equal(a.nan_to_num(-1), t.nan_to_num(-1)) if t.is_floating_point() else torch.equal(a, t)


def test_append_e4m3_steps_are_the_nearest(B):
    """Every value of e4m3 in [-448, 448] and the points half way between neighbours (to even), with a scale of 1."""
    grid = torch.arange(127, dtype=torch.uint8).view(F8).float()
    mid = (grid[1:] + grid[:-1]) / 2
    x = torch.cat([grid, mid, -grid, -mid, torch.zeros(4)])
    n = (len(x) + 62) // 63
    x = torch.cat([x, torch.zeros(n * 63 - len(x))]).view(1, n, 1, 63)
    x = torch.cat([torch.full((1, n, 1, 1), 448.0), x], -1)                            # the largest magnitude: a scale of 1
    cache = make_cache(B, 1, n, 1, 64, f8=True)
    B.tabed_cache_append_nodes(cache, x.to(DEV), x.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV))
    got, y = cache.v[0, int(cache.table[0, 0]), 0, :n].float().cpu(), x[0, :, 0]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    assert torch.equal(got, torch.round(y / step) * step)


# ------------------------------------------------------------------ attention
def check_attention(B, rows, N, qh, kvh, hd, ctx, f8=False, kind="random", by_token=False, ragged=True, holes=(), seed=0, layers=1, layer=0, spoil=True, ws=None,
                    loud=1.5, strided=False):
    """ctx: one length a row.  spoil: everything that no node sees holds NaN."""
    g = gen(seed + 2)
    tokens = max(ctx) + N
    cache = make_cache(B, rows, tokens, kvh, hd, f8, layers, by_token, seed)
    for r, e in holes:
        cache.table[r, e] = -1 if r % 2 else 2 ** 31 - 1
    parents = trees(rows, N, kind)
    nodes = torch.randint(1, N + 1, (rows,), generator=g) if ragged else torch.full((rows,), N)
    nodes[0] = N
    table = cache.table.cpu()
    if spoil:
        nan = make_cache(B, rows, tokens, kvh, hd, f8, layers, by_token, seed, fill="nan")
        keep = torch.zeros(cache.struct.blocks, 64, dtype=torch.bool)
        for r in range(rows):
            for p in range(ctx[r] + int(nodes[r])):
                at = ref.place(table, cache.struct.blocks, r, p)
                if at:
                    keep[at] = True
        keep = keep.to(DEV)
        for name in ("k", "v"):
            x, y = getattr(cache, name), getattr(nan, name)
            bits = torch.uint8 if f8 else torch.int16
            x.view(bits).copy_(torch.where(keep[None, :, None, :, None], x.view(bits), y.view(bits)))
            if f8:
                s = getattr(cache, name + "scale")
                s.copy_(torch.where(keep[None, :, None], s, math.nan))
    q = (loud * torch.randn(rows, N, qh, hd, generator=g)).to(torch.bfloat16)
    dq = q.to(DEV)
    out = torch.full((rows, N, qh, hd), 7.0, dtype=torch.bfloat16, device=DEV)
    if strided:                                                                        # views into larger rows, off by one element
        big = torch.zeros(rows, N, qh * hd + 9, dtype=torch.bfloat16, device=DEV)
        big[..., 1:1 + qh * hd] = dq.flatten(2)
        dq = big[..., 1:1 + qh * hd].unflatten(-1, (qh, hd))
        out = torch.full((N, rows, qh * hd + 3), 7.0, dtype=torch.bfloat16, device=DEV)[..., 3:].unflatten(-1, (qh, hd)).transpose(0, 1)
    lse = torch.full((rows, N, qh), 7.0, device=DEV)
    if ws is None:
        ws = B.new_attention_nodes_workspace(cache, rows, N, qh)
    i32 = lambda t: None if t is None else torch.as_tensor(t).to(torch.int32).to(DEV)  # noqa: E731
    args = dict(parents=i32(parents), n_nodes=i32(nodes), lse=lse, layer=layer)
    B.tabed_attention_nodes(cache, ws, dq, i32(ctx), out, **args)
    scale = hd ** -0.5
    k, v = values(cache, "k", layer), values(cache, "v", layer)
    want, wlse, mass = ref.attention(q.double(), k, v, table, cache.struct.blocks, ctx, parents, nodes.tolist(), scale)
    got, glse = out.cpu().double(), lse.cpu().double()
    live = torch.arange(N)[None] < nodes[:, None]
    assert (got[~live] == 7).all() and (glse[~live] == 7).all()
    # Scores: hd exact products summed in fp32, each addition off by 2^-24 of at most the sum of magnitudes; one product with the scale, one
    # with a key's scale; exp2 of a difference: 2^-22 of it at most 2^7 and 2^-23 in itself.  What that is relative in a probability:
    big = float((q.double().abs().sum(-1).amax() * k.nan_to_num(0).abs().amax() * scale).clamp(max=2.0 ** 12))
    rel = (hd + 4) * 2.0 ** -24 * big + 2.0 ** -14
    # The result: its own rounding, a probability's rounding (2^-8), its error twice (itself, the sum), and the sums in fp32.
    tol = 2.0 ** -8 * want.abs() + mass * (2.0 ** -8 + 2 * rel + 2.0 ** -14)
    bad = (got - want).abs() > tol
    assert not bad[live].any(), f"{int(bad[live].sum())} off, at most {float(((got - want).abs() / tol)[live].nan_to_num(9e9).max()):.2f} times the tolerance"
    assert torch.equal(torch.isinf(glse[live]), torch.isinf(wlse[live]))
    fine = live[..., None] & torch.isfinite(wlse)
    assert ((glse - wlse).abs()[fine] <= rel + 2.0 ** -22 * wlse.abs()[fine]).all()
    first = out.clone()
    for _ in range(2):                                                                 # the same bits every time
        B.tabed_attention_nodes(cache, ws, dq, i32(ctx), out, **args)
        assert torch.equal(first, out)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("N,qh,kvh", [(1, 2, 2), (7, 6, 2), (20, 8, 2), (40, 12, 3)])
def test_attention_sizes(B, N, qh, kvh, hd, f8):
    check_attention(B, 3, N, qh, kvh, hd, [0, 100, 333], f8, seed=N + hd, by_token=hd % 64 == 0)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("kind", ["chain", "star", "deep", "forest"])
@pytest.mark.parametrize("N", [2, 33, 64, 65, 130, 256])
def test_attention_trees(B, N, kind, f8):
    check_attention(B, 2, N, 2, 1, 64, [61, 130], f8, kind=kind, seed=N)


@pytest.mark.parametrize("ctx", [0, 1, 15, 16, 31, 32, 33, 63, 64, 65, 127, 128, 129, 511, 512, 513, 2000, 2047])
@pytest.mark.parametrize("N", [1, 17])
def test_attention_lengths(B, ctx, N):
    check_attention(B, 2, N, 4, 2, 128, [ctx, max(0, ctx - 5)], seed=ctx, ragged=False)
    check_attention(B, 1, N, 3, 3, 64, [ctx], f8=True, seed=ctx)


@pytest.mark.parametrize("N,qh,kvh,hd,ctx", [(1, 4, 4, 64, 20_011), (16, 8, 2, 128, 9001), (3, 8, 1, 256, 5003), (100, 4, 1, 128, 4100), (256, 2, 2, 64, 3000)])
def test_attention_long(B, N, qh, kvh, hd, ctx):
    check_attention(B, 1, N, qh, kvh, hd, [ctx], seed=ctx, spoil=False)
    check_attention(B, 1, N, qh, kvh, hd, [ctx], f8=True, seed=ctx, spoil=False)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("rows,N,qh,kvh,hd", [(1, 6, 12, 12, 64), (10, 9, 12, 12, 64), (11, 9, 12, 12, 64), (3, 20, 4, 4, 32), (2, 31, 4, 4, 64), (15, 4, 32, 8, 128), (16, 4, 32, 8, 128)])
def test_attention_few_and_many_rows(B, rows, N, qh, kvh, hd, f8):
    check_attention(B, rows, N, qh, kvh, hd, [(1500, 0, 31, 257, 1, 700, 1024, 255, 512)[i % 9] for i in range(rows)], f8, seed=rows)


@pytest.mark.parametrize("f8", [False, True])
def test_attention_holes(B, f8):
    check_attention(B, 4, 9, 4, 2, 64, [300, 200, 64, 0], f8, holes=[(0, 0), (0, 3), (1, 3), (2, 0), (2, 1), (3, 0)], seed=1)
    check_attention(B, 1, 5, 2, 2, 128, [3000], f8, holes=[(0, e) for e in range(0, 47, 2)], seed=2)
    check_attention(B, 2, 5, 2, 2, 128, [3000, 10], f8, holes=[(0, e) for e in range(47)] + [(1, 0)], seed=3)


def test_attention_strides_layers_and_large_scores(B):
    check_attention(B, 3, 6, 4, 2, 64, [70, 5, 128], strided=True, seed=1)
    check_attention(B, 2, 6, 4, 2, 64, [70, 5], layers=3, layer=1, f8=True, seed=2)
    check_attention(B, 2, 6, 4, 2, 64, [70, 5], layers=2, layer=1, by_token=True, seed=2)
    check_attention(B, 2, 21, 4, 2, 64, [170, 5], loud=60.0, seed=4)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("N,qh", [(6, 2), (40, 8)])
def test_attention_what_is_not_finite_stays_with_those_who_see_it(B, N, qh, f8):
    """A node with NaN, another with an infinite value, and a block's scale: NaN (or the infinity) for the nodes below, nothing for the others."""
    rows, kvh, hd, ctx = 1, 2, 64, [150]
    cache = make_cache(B, rows, 150 + N, kvh, hd, f8, seed=9)
    parents = trees(rows, N, "random")
    bad = 2
    b, s = ref.place(cache.table.cpu(), cache.struct.blocks, 0, 150 + bad)
    q = torch.randn(rows, N, qh, hd, generator=gen(3)).to(torch.bfloat16).to(DEV)
    i32 = lambda t: torch.as_tensor(t).to(torch.int32).to(DEV)  # noqa: E731
    ws = B.new_attention_nodes_workspace(cache, rows, N, qh)

    def call():
        out = torch.zeros_like(q)
        B.tabed_attention_nodes(cache, ws, q, i32(ctx), out, parents=i32(parents))
        return out[0].float().cpu()
    clean = call()
    below = torch.tensor([bad in ref.above(parents, 0, j) for j in range(N)])
    assert 0 < below.sum() < N
    spoils = [("kscale", math.nan), ("vscale", math.nan), ("vscale", math.inf)] if f8 else [("k", math.nan), ("v", math.nan), ("v", math.inf), ("v", -math.inf)]
    for name, what in spoils:
        t = getattr(cache, name)
        kept = t.clone()
        if f8:
            t[0, b, :, s] = what
        else:
            t[0, b, :, s, 7] = what
        got = call()
        assert torch.equal(got[~below], clean[~below]), (name, what)
        seen = got[below]
        if f8 or name == "k":
            assert (~torch.isfinite(seen)).flatten(1).any(1).all()
        else:
            assert (seen[..., 7].isnan().all() if math.isnan(what) else (seen[..., 7] == what).all())
            seen[..., 7] = clean[below][..., 7]
            assert torch.equal(seen, clean[below])
        t.copy_(kept)
    assert torch.equal(call(), clean)


def test_attention_one_workspace_for_all_sizes(B):
    cache = make_cache(B, 1, 20_100, 4, 128)
    ws = torch.full((max(B.tabed_attention_nodes_workspace_bytes(cache, *s) for s in ((1, 1, 32), (64, 16, 32), (3, 256, 32), (2, 40, 12))) * 3,), 255, dtype=torch.uint8, device=DEV)
    B.tabed_attention_nodes_workspace_init(cache, 1, 1, 4, ws)
    for rows, N, qh, kvh, hd, ctx in ((1, 1, 4, 4, 128, [9000]), (2, 40, 12, 3, 64, [500, 20]), (3, 7, 4, 1, 256, [3000, 5, 100]), (1, 16, 8, 8, 32, [6000]), (1, 1, 4, 4, 128, [9000])):
        check_attention(B, rows, N, qh, kvh, hd, ctx, ws=ws, seed=N, spoil=False)


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("rows,N,ctx", [(2, 5, 300), (1, 24, 5000), (3, 70, 2500), (2, 256, 40)])
def test_attention_in_place_of_its_queries(B, rows, N, ctx, f8):
    cache = make_cache(B, rows, ctx + N, 2, 64, f8)
    q = torch.randn(rows, N, 8, 64, generator=gen(N)).to(torch.bfloat16).to(DEV)
    out, lens = torch.zeros_like(q), torch.full((rows,), ctx, dtype=torch.int32, device=DEV)
    ws, parents = B.new_attention_nodes_workspace(cache, rows, N, 8), trees(rows, N, "random").to(DEV)
    B.tabed_attention_nodes(cache, ws, q, lens, out, parents=parents)
    B.tabed_attention_nodes(cache, ws, q, lens, q, parents=parents)
    assert torch.equal(q, out)


def test_attention_workspace_of_the_largest_call_serves_smaller_ones(B):
    need = B.tabed_attention_nodes_workspace_bytes(make_cache(B, 70, 3200, 2, 64), 70, 64, 8)
    ws = torch.full((need + (32 << 20),), 0x5a, dtype=torch.uint8, device=DEV)
    for rows, N in ((70, 64), (70, 1), (20, 64), (3, 33), (3, 8), (1, 3), (1, 1)):
        check_attention(B, rows, N, 8, 2, 64, [3000 - 31 * i % 2999 for i in range(rows)], seed=rows + N, ws=ws, spoil=False)
        assert bool((ws[need:] == 0x5a).all()), (rows, N)


def test_attention_past_2_32_bytes(B):
    """Blocks at the far end of a pool of more than 2^32 bytes, in elements too."""
    blocks, kvh, hd = 33_000, 8, 128
    k, v = (torch.zeros((blocks, kvh, 64, hd), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    assert k.numel() > 2 ** 31 and k.numel() * 2 > 2 ** 32
    table = torch.tensor([[blocks - 1, blocks - 3], [blocks - 2, 5]], dtype=torch.int32, device=DEV)
    cache = B.CachePaged(k, v, table)
    small = B.CachePaged(torch.zeros((4, kvh, 64, hd), dtype=torch.bfloat16, device=DEV), torch.zeros((4, kvh, 64, hd), dtype=torch.bfloat16, device=DEV),
                         torch.tensor([[3, 1], [2, 0]], dtype=torch.int32, device=DEV))
    x = [torch.randn(2, 100, h, hd, generator=gen(i)).to(torch.bfloat16).to(DEV) for i, h in ((1, kvh), (2, kvh), (3, 16))]
    ctx = torch.zeros(2, dtype=torch.int32, device=DEV)
    outs = []
    for c in (cache, small):
        q_out, out = torch.empty_like(x[2]), torch.empty_like(x[2])
        B.tabed_cache_append_nodes(c, x[0], x[1], ctx, q=x[2], q_out=q_out, rope_theta=THETA)
        B.tabed_attention_nodes(c, B.new_attention_nodes_workspace(c, 2, 100, 16), q_out, ctx, out)
        path = torch.tensor([list(range(0, 100, 2)) + [-1] * 50] * 2, dtype=torch.int32, device=DEV)
        B.tabed_cache_keep_nodes(c, ctx, path, torch.tensor([50, 7], dtype=torch.int32, device=DEV), torch.empty_like(ctx))
        again = torch.empty_like(out)
        B.tabed_attention_nodes(c, B.new_attention_nodes_workspace(c, 2, 100, 16), q_out, ctx, again)
        outs.append((q_out, out, again))
    for a, b in zip(*outs):
        assert torch.equal(a, b)
    assert not torch.equal(outs[0][1], outs[0][2])


# ------------------------------------------------------------------ keep
@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("hd,N,by_token", [(32, 40, False), (64, 6, True), (96, 17, False), (128, 256, False), (256, 70, True)])
def test_keep(B, hd, N, by_token, f8):
    rows, kvh, layers = 4, 3, 2
    g = gen(hd)
    cache = make_cache(B, rows, 130 + N, kvh, hd, f8, layers, by_token, seed=hd)
    ctx = [0, 63, 64, 130]
    paths, counts = [], []
    for r in range(rows):
        some = 1 + int(torch.randint(0, N, (1,), generator=g))
        p = [0] + sorted((torch.randperm(N - 1, generator=g)[:some - 1] + 1).tolist())
        if r == 1:
            p = list(range(1, N))                                                     # every entry moves down by one
        paths.append(p + [-1] * (N - len(p)))
        counts.append(len(p))
    names = ["k", "v"] + (["kscale", "vscale"] if f8 else [])
    bits = {"k": torch.uint8 if f8 else torch.int16, "v": torch.uint8 if f8 else torch.int16, "kscale": torch.int32, "vscale": torch.int32}
    want = {n: getattr(cache, n).view(bits[n]).cpu().clone() for n in names}
    table = cache.table.cpu()
    for r in range(rows):
        for i in range(counts[r]):
            (fb, fs), (tb, ts) = (ref.place(table, cache.struct.blocks, r, ctx[r] + x) for x in (paths[r][i], i))
            for n in names:
                want[n][:, tb, :, ts] = want[n][:, fb, :, fs]
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)  # noqa: E731
    out = i32([-1] * rows)
    B.tabed_cache_keep_nodes(cache, i32(ctx), i32(paths), i32(counts), out)
    assert out.tolist() == [c + n for c, n in zip(ctx, counts)]
    for n in names:
        assert torch.equal(getattr(cache, n).view(bits[n]).cpu(), want[n]), n


def test_keep_paths_that_end_and_holes(B):
    cache = make_cache(B, 6, 128, 2, 64, seed=2)
    cache.table[4, 1] = -1
    i32 = lambda t: torch.tensor(t, dtype=torch.int32, device=DEV)  # noqa: E731
    paths = [[0, 2, 2, 5], [0, 3, 1, 5], [0, 4, 5, 8], [-1, 1, 2, 3], [0, 3, 5, 7], [1, 2, 3, 4]]
    paths = [p + [9, 10, 11, 12] for p in paths]
    before = cache.k.cpu().clone()
    ctx, out = i32([0, 10, -3, 4, 60, 2]), i32([0] * 6)
    B.tabed_cache_keep_nodes(cache, ctx, i32(paths), i32([4, 4, 3, 4, 4, 99]), out)
    # (8 nodes: an 8 ends the path of row 2 behind 0, 4, 5; row 5's ends at 9)
    kept = [2, 2, 3, 0, 4, 4]
    assert out.tolist() == [0 + 2, 10 + 2, 0 + 3, 4, 64, 6]
    table = cache.table.cpu()
    want = before.clone()
    for r in range(6):
        base = max(ctx.tolist()[r], 0)
        for i in range(kept[r]):
            a, b = (ref.place(table, cache.struct.blocks, r, base + x) for x in (paths[r][i], i))
            if a and b:
                want[:, b[0], :, b[1]] = want[:, a[0], :, a[1]]
    assert torch.equal(cache.k.cpu(), want)

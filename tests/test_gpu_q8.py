"""The 8-bit operators (tabed_norm_q8, tabed_linear_q8, tabed_cache_append_q8, tabed_attention_q8) against plain definitions, at the sizes,
types, strides and masks where they can go wrong."""
import math

import numpy as np
import pytest
import torch

import q8_reference as ref
from paper_2601_20357_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(shape, generator=g).to(dtype)


# ------------------------------------------------------------------ norm
def norm_case(x, delta, gain, eps, in_place=False, pad=0):
    """Runs the kernel on views whose rows stand `pad` values apart; returns CPU tensors (q, scale, sum) and checks the padding."""
    rows, d = x.shape

    def wide(t, fill):
        buf = torch.full((rows, d + pad), fill, dtype=t.dtype, device=DEV)
        buf[:, :d] = t.to(DEV)
        return buf

    xb = wide(x, 7)
    db = None if delta is None else wide(delta, 7)
    qb = torch.full((rows, d + pad), 99, dtype=torch.int8, device=DEV)
    sb = xb if in_place else (None if delta is None else torch.full((rows, d + pad), 5, dtype=x.dtype, device=DEV))
    scale = torch.empty(rows, device=DEV)
    view = lambda t: None if t is None else t[:, :d]
    binding.tabed_norm_q8(view(xb), view(qb), scale, delta=view(db), sum_out=view(sb), gain=None if gain is None else gain.to(DEV), eps=eps)
    torch.cuda.synchronize()
    if pad:
        assert (qb[:, d:] == 99).all() and (sb is None or (sb[:, d:] == (7 if in_place else 5)).all())
    return qb[:, :d].cpu(), scale.cpu(), None if sb is None else sb[:, :d].cpu()


# Roundings of y: at most 32 fp32 additions a lane, 6 + 16 between lanes and waves, half of which reaches the root; then the mean, the root,
# the reciprocal and two products: 32 half steps of fp32 and less.
Y_HALF_STEPS = 64


@pytest.mark.parametrize("rows,d,xt,dt,pad", [
    (1, 1, F32, None, 0), (3, 7, BF16, BF16, 1), (4, 768, F32, None, 0), (5, 64, BF16, F32, 3), (1027, 100, F32, BF16, 0), (2, 2048, BF16, None, 8),
    (3, 2049, F32, F32, 0), (2, 2051, BF16, BF16, 5), (1, 8192, F32, BF16, 0), (2, 8193, BF16, F32, 0), (1, 32768, F32, F32, 0), (1024, 16, BF16, BF16, 0)])
@pytest.mark.parametrize("with_gain", [True, False])
def test_norm_q8(rows, d, xt, dt, pad, with_gain):
    g = gen(rows * 7919 + d)
    x = randn(g, rows, d, dtype=xt) * 3
    delta = None if dt is None else randn(g, rows, d, dtype=dt)
    gain = 1 + 0.2 * randn(g, d) if with_gain else None
    q, scale, total = norm_case(x, delta, gain, 1e-5, pad=pad)
    r, y, s = ref.norm(x, delta, gain, 1e-5)
    if total is not None:      # one fp32 addition, one rounding to the type
        assert ((total.double() - r).abs() <= r.abs() * (ref.half_step(xt) * (xt != F32) + 2 * 2.0 ** -24)).all()
    tol = Y_HALF_STEPS * 2.0 ** -24
    assert ((scale.double() - s).abs() <= s * tol).all()
    # y / scale is at most 127 and off by 2 tol of it; rounding adds half a step
    assert ((q.double() - y / s[:, None]).abs() <= 0.5 + 127 * 2 * tol).all()
    assert (q.abs().amax(1) == 127).all()


def test_norm_q8_in_place_and_rounding_of_the_sum():
    g = gen(5)
    x, delta, gain = randn(g, 9, 300, dtype=BF16), randn(g, 9, 300, dtype=BF16), 1 + 0.1 * randn(g, 300)
    q, scale, total = norm_case(x, delta, gain, 1e-5, in_place=True)
    q2, scale2, total2 = norm_case(x, delta, gain, 1e-5)
    assert torch.equal(q, q2) and torch.equal(scale, scale2) and torch.equal(total, total2)
    assert torch.equal(total, (x.float() + delta.float()).to(BF16))


def test_norm_q8_rows_of_zeros_tiny_and_not_finite():
    x = torch.randn(7, 130, generator=gen(1))
    x[1] = 0
    x[2] = x[2] * 2.0 ** -110                 # nothing reaches 2^-100
    x[3, 129] = math.inf
    x[4, 0] = math.nan
    x[5, 64] = -math.inf
    for gain in (None, torch.ones(130)):
        q, scale, _ = norm_case(x, None, gain, 1e-5)
        bad = torch.tensor([3, 4, 5])
        assert torch.isnan(scale[bad]).all() and (q[bad] == 0).all()
        assert scale[1] == 0 and (q[1] == 0).all()
        good = torch.tensor([0, 6])
        assert torch.isfinite(scale[good]).all() and (q[good].abs().amax(1) == 127).all()
        assert scale[2] == 0 and (q[2] == 0).all()
    huge = torch.full((1, 64), 1e25)          # squares past fp32
    _, scale, _ = norm_case(huge, None, torch.ones(64), 1e-5)
    assert torch.isnan(scale).all()
    _, scale, _ = norm_case(huge, None, None, 1e-5)
    assert scale[0] == np.float32(1e25) / np.float32(127)


# ------------------------------------------------------------------ linear
def linear_case(x, sx, w, sw, yt, ldx=None, ldy=None):
    M, K = x.shape
    N = w.shape[0]
    xb = torch.zeros((M, ldx or K), dtype=torch.int8, device=DEV)
    xb[:, :K] = x.to(DEV)
    y = torch.full((M + 1, ldy or N), 77.0, dtype=yt, device=DEV)
    binding.tabed_linear_q8(xb[:, :K], sx.to(DEV), w.to(DEV), sw.to(DEV), y[:M, :N])
    torch.cuda.synchronize()
    assert (y[M] == 77).all() and (y[:M, N:] == 77).all()          # nothing behind the last row or column
    return y[:M, :N].cpu()


def check_linear(y, x, sx, w, sw, yt):
    whole = x.double() @ w.double().t()                            # exact: below 2^53
    want = whole * sx.double()[:, None] * sw.double()[None, :]
    # the integer to fp32, a product for each scale, the rounding for storage
    tol = want.abs() * (3.01 * 2.0 ** -24 + (0 if yt == F32 else 1.01 * ref.half_step(yt)))
    assert ((y.double() - want).abs() <= tol).all()


@pytest.mark.parametrize("M", [1, 3, 16, 17, 33, 64, 65, 130, 300])
@pytest.mark.parametrize("N,K", [(1, 16), (31, 64), (32, 48), (100, 80), (257, 768), (515, 2064), (4100, 528)])
def test_linear_q8(M, N, K):
    g = gen(M * 31 + N * 7 + K)
    yt = BF16 if (M + N) % 2 else F32
    x, w = (torch.randint(-128, 128, s, generator=g, dtype=torch.int8) for s in ((M, K), (N, K)))
    sx, sw = torch.rand(M, generator=g) + 0.1, torch.rand(N, generator=g) * 0.01
    y = linear_case(x, sx, w, sw, yt, ldx=K + 32 if M % 3 == 0 else None, ldy=N + 5 if N % 2 else None)
    check_linear(y, x, sx, w, sw, yt)


@pytest.mark.parametrize("M,N,K", [(2, 40, 131056), (70, 130, 131056), (257, 300, 4096), (512, 1024, 1024), (200, 2049, 4112), (1030, 70, 256)])
def test_linear_q8_longest_sums_and_larger_sizes(M, N, K):
    g = gen(K)
    x, w = (torch.randint(-128, 128, s, generator=g, dtype=torch.int8) for s in ((M, K), (N, K)))
    x[0], w[0], w[N - 1] = -128, -128, 127                         # K 128^2: the largest sum there is, and nearly the smallest
    sx, sw = torch.rand(M, generator=g) + 0.1, torch.rand(N, generator=g) * 0.01
    check_linear(linear_case(x, sx, w, sw, F32), x, sx, w, sw, F32)


@pytest.mark.parametrize("M,N,K", [(3, 70001, 4112), (40, 40001, 1040), (17, 66000, 2064), (64, 33000, 2048)])
def test_linear_q8_workgroups_that_go_on(M, N, K):
    """More tiles than run at once."""
    g = torch.Generator(device=DEV).manual_seed(N)
    x, w = (torch.randint(-127, 128, s, generator=g, dtype=torch.int8, device=DEV) for s in ((M, K), (N, K)))
    sx, sw = torch.ones(M, device=DEV), torch.ones(N, device=DEV)
    y = torch.empty((M, N), device=DEV)
    binding.tabed_linear_q8(x, sx, w, sw, y)
    want = x.double() @ w.double().t()
    assert torch.equal(y, want.float())                            # one rounding of an exact integer


@pytest.mark.parametrize("M,N,K", [(5, 90, 1008), (40, 100, 1040), (33, 65, 3088), (70, 129, 2032), (1, 8200, 16), (16, 8200, 528), (30, 8200, 1008),
                                   (40, 9000, 16), (50, 9000, 240), (64, 8200, 528), (33, 17000, 16), (64, 17000, 784), (7, 17000, 4112),
                                   (130, 8000, 16), (129, 8010, 400), (190, 6000, 128)])
def test_linear_q8_ends_of_k_in_small_tiles(M, N, K):
    """K that ends in each part of a block that several waves share, for every number of them."""
    g = torch.Generator(device=DEV).manual_seed(K)
    x, w = (torch.randint(-128, 128, s, generator=g, dtype=torch.int8, device=DEV) for s in ((M, K), (N, K)))
    wide = torch.full((M, K + 16), 99, dtype=torch.int8, device=DEV)                     # what lies behind a row is not taken
    wide[:, :K] = x
    y = torch.full((M + 1, N + 3), 7.0, device=DEV)
    binding.tabed_linear_q8(wide[:, :K], torch.ones(M, device=DEV), w, torch.ones(N, device=DEV), y[:M, :N])
    want = x.double() @ w.double().t()
    assert torch.equal(y[:M, :N], want.float()) and (y[M] == 7).all() and (y[:, N:] == 7).all()


def test_linear_q8_outputs_past_four_gigabytes():
    M, N, K = 70, 2 ** 24, 16
    w = torch.ones((N, K), dtype=torch.int8, device=DEV)
    w[-3:] = torch.tensor([[2], [-3], [4]], dtype=torch.int8, device=DEV)
    x = torch.ones((M, K), dtype=torch.int8, device=DEV)
    x[-1] = 5
    y = torch.zeros((M, N), device=DEV)
    binding.tabed_linear_q8(x, torch.ones(M, device=DEV), w, torch.ones(N, device=DEV), y)
    assert (y[:-1, :-3] == 16).all() and (y[-1, :-3] == 80).all()
    assert y[0, -3:].tolist() == [32, -48, 64] and y[-1, -3:].tolist() == [160, -240, 320]


def test_linear_q8_bad_rows_stay_their_own():
    g = gen(3)
    x, w = (torch.randint(-127, 128, s, generator=g, dtype=torch.int8) for s in ((9, 64), (70, 64)))
    sx, sw = torch.ones(9), torch.ones(70)
    sx[4], sw[11], sw[69] = math.nan, math.inf, 0.0
    y = linear_case(x, sx, w, sw, F32)
    whole = (x.double() @ w.double().t()).float()
    assert torch.isnan(y[4]).all() and (y[[0, 8]][:, 69] == 0).all()
    keep = [i for i in range(69) if i != 11]
    assert torch.equal(y[:4][:, keep], whole[:4][:, keep]) and torch.equal(y[5:][:, keep], whole[5:][:, keep])


# ------------------------------------------------------------------ cache
class Cache:
    """A cache on the GPU and its copy on the CPU."""

    def __init__(self, rows, width, kvh, hd, seed, spare=3):
        g = np.random.default_rng(seed)
        self.rows, self.width, self.kvh, self.hd = rows, width, kvh, hd
        blocks = rows * width + spare
        self.table = g.permutation(blocks)[:rows * width].reshape(rows, width).astype(np.int32)
        self.pool = {n: g.integers(-127, 128, (blocks, kvh, 64 * hd)).astype(np.int8) for n in ("k", "v")}
        self.scale = {n: g.uniform(0.5, 1.5, (blocks, kvh)).astype(np.float32) / 40 for n in ("k", "v")}
        self.push()

    def push(self):
        t = lambda a: torch.from_numpy(a.copy()).to(DEV)
        self.gpu = binding.CacheQ8(t(self.pool["k"]), t(self.pool["v"]), t(self.scale["k"]), t(self.scale["v"]), t(self.table), self.hd)

    def append(self, k, v, ctx, n_new=None, type=F32, stream=None):
        dev = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device=DEV)
        kt, vt = k.to(type), v.to(type)
        binding.tabed_cache_append_q8(self.gpu, kt.to(DEV), vt.to(DEV), dev(ctx), dev(n_new), stream=stream)
        torch.cuda.synchronize()
        for n, x in (("k", kt), ("v", vt)):
            ref.append(self.pool[n], self.scale[n], self.table, n, x.float().numpy(), ctx, n_new, self.hd)

    def same(self):
        """Every block and scale as the definition, byte by byte: those that nothing was appended to too."""
        for n in ("k", "v"):
            got, want = getattr(self.gpu, n + "scale").cpu().numpy(), self.scale[n]
            assert np.array_equal(got, want, equal_nan=True), n
            assert np.array_equal(getattr(self.gpu, n).cpu().numpy(), self.pool[n]), n




@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("T,type", [(1, F32), (1, BF16), (5, F32), (64, BF16), (131, F32)])
def test_cache_append(hd, T, type):
    c = Cache(6, 5, 3, hd, seed=hd + T)
    g = gen(hd * T)
    ctx = [0, 1, 63, 64, 100, 188]
    for size in (0.05, 1.0, 30.0):             # under the old scale, about it, and far over it: kept tokens are rounded again
        k, v = randn(g, 6, T, 3, hd) * size, randn(g, 6, T, 3, hd) * size
        c.append(k, v, ctx, type=type)
        c.same()
        ctx = [min(x + T, 320 - T) for x in ctx]


def test_cache_append_of_ragged_rows_and_missing_blocks():
    c = Cache(7, 4, 2, 64, seed=1)
    c.table[1, 1], c.table[2, 0], c.table[3, 2] = -1, 10 ** 6, c.pool["k"].shape[0]        # no blocks
    c.push()
    g = gen(2)
    T = 90
    k, v = randn(g, 7, T, 2, 64), randn(g, 7, T, 2, 64)
    c.append(k, v, [10, 20, 30, 100, 200, -5, 2 ** 31 - 1], [90, 90, 90, 90, 90, 33, 90])   # row 4 runs past the table, row 6 lies behind it
    c.same()
    c.append(k, v, [0, 1, 2, 3, 4, 5, 6], [0, -3, 1, 1000, 64, 7, 2])
    c.same()
    c.append(k, v, [0, 1, 2, 3, 4, 5, 6], [0, -3, 1, 1000, 64, 7, 2])                       # again: nothing changes
    c.same()


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("T,type", [(4, BF16), (8, BF16), (8, F32), (9, BF16)])
def test_cache_append_of_a_few_ragged_tokens(hd, T, type):
    """Rows that end inside a block, on its last token and behind it, at sizes that grow and do not grow a scale."""
    c = Cache(8, 3, 2, hd, seed=T)
    c.table[7, 0] = -1
    c.push()
    g = gen(T + hd)
    for size, ctx in ((0.02, [0, 56, 60, 63, 64, 127, 190, 58]), (20.0, [3, 58, 62, 64, 71, 120, 191, 61]), (1.0, [1, 57, 61, 60, 68, 126, 185, 59])):
        n_new = [T, T - 1, T, 2, 0, T, T, T]
        c.append(randn(g, 8, T, 2, hd) * size, randn(g, 8, T, 2, hd) * size, ctx, n_new, type=type)
        c.same()


def test_cache_append_of_zeros_tiny_and_not_finite():
    c = Cache(4, 2, 2, 32, seed=4)
    k = torch.zeros(4, 1, 2, 32)
    v = torch.full((4, 1, 2, 32), 2.0 ** -120)
    k[1, 0, 1, 5], k[2, 0, 0, 31], v[3, 0, 1, 0] = math.nan, math.inf, -math.inf
    c.append(k, v, [64, 64, 64, 64])
    c.same()
    assert (c.scale["k"][c.table[0, 1]] == 0).all() and np.isnan(c.scale["k"][c.table[1, 1], 1]) and not np.isnan(c.scale["k"][c.table[1, 1], 0])
    c.append(torch.ones(4, 1, 2, 32), torch.ones(4, 1, 2, 32), [65, 65, 65, 65])            # a bad block stays bad until it begins anew
    c.same()
    assert np.isnan(c.scale["k"][c.table[1, 1], 1])
    c.append(torch.ones(4, 1, 2, 32), torch.ones(4, 1, 2, 32), [64, 64, 64, 64])
    c.same()
    assert not np.isnan(c.scale["k"][c.table[1, 1], 1])


def test_cache_append_reads_strided_views_on_another_stream():
    c = Cache(3, 3, 4, 64, seed=6)
    g = gen(9)
    qkv = randn(g, 3, 10, 3 * 4 * 64 + 1, dtype=BF16).to(DEV)                # rows of odd length: tokens at any alignment of their own
    k, v = qkv[:, 2:9, 256:512], qkv[:, 2:9, 512:768]
    stream = torch.cuda.Stream()
    ctx = torch.tensor([5, 60, 64], dtype=torch.int32, device=DEV)
    torch.cuda.synchronize()
    binding.tabed_cache_append_q8(c.gpu, k, v, ctx, stream=stream)
    stream.synchronize()
    for n, x in (("k", k), ("v", v)):
        ref.append(c.pool[n], c.scale[n], c.table, n, x.float().cpu().reshape(3, 7, 4, 64).numpy(), [5, 60, 64], None, 64)
    c.same()


# ------------------------------------------------------------------ attention
def attend(c, q, ctx, n_new=None, out_type=F32, scale=None, with_lse=True, ws=None, into=None):
    rows, T, qh, hd = q.shape
    out = torch.full((rows, T, qh, hd), 55.0, dtype=out_type, device=DEV) if into is None else into
    lse = torch.full((rows, T, qh), 66.0, device=DEV) if with_lse else None
    dev = lambda a: None if a is None else torch.tensor(a, dtype=torch.int32, device=DEV)
    ws = binding.new_attention_workspace(c.gpu, rows, T, qh) if ws is None else ws
    binding.tabed_attention_q8(c.gpu, ws, q.to(DEV), dev(ctx), out, n_new=dev(n_new), scale=scale, lse=lse)
    torch.cuda.synchronize()
    return out.cpu(), None if lse is None else lse.cpu()


def check_attention(c, q, ctx, n_new, out, lse, scale=None):
    hd = q.shape[-1]
    want, wlse, bound = ref.attention(c.pool, c.scale, c.table, q.float().numpy(), ctx, n_new, scale or hd ** -0.5, hd)
    left = np.isnan(wlse)                                           # tokens from n_new on
    o = out.double().numpy()
    assert (o[left] == 55).all() and (lse is None or (lse.numpy()[left] == 66).all())
    tol = bound[..., None] + (0 if out.dtype == F32 else ref.half_step(out.dtype) * (np.abs(want) + bound[..., None]))
    assert (np.abs(o - want)[~left] <= tol[~left]).all()
    if lse is not None:
        empty = ~left & np.isneginf(wlse)
        assert np.isneginf(lse.numpy()[empty]).all() and (o[empty] == 0).all()
        full = ~left & ~empty
        # bound / max|v| would be the error of log of the sum; the values here are below 4, and m + log l is rounded twice at its size
        assert (np.abs(lse.double().numpy()[full] - wlse[full]) <= bound[full] * 8 + 4 * 2.0 ** -24 * (np.abs(wlse[full]) + 8)).all()


@pytest.mark.parametrize("hd", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("kvh,group,T,qt,ot", [(3, 1, 1, F32, F32), (2, 4, 1, BF16, F32), (1, 7, 2, F32, BF16), (2, 2, 3, BF16, BF16), (1, 8, 6, F32, F32)])
def test_attention(hd, kvh, group, T, qt, ot):
    c = Cache(6, 9, kvh, hd, seed=hd + T)
    q = randn(gen(hd + group), 6, T, kvh * group, hd, dtype=qt)
    ctx = [0, 1, 62, 64, 300, 570]
    out, lse = attend(c, q, ctx, out_type=ot)
    check_attention(c, q, ctx, None, out, lse)


@pytest.mark.parametrize("T,n_new", [(1, None), (1, [1, 0, 1]), (33, [33, 0, 20]), (70, [1, 69, 64])])
def test_attention_over_many_ranges(T, n_new):
    c = Cache(3, 130, 1, 64, seed=T)
    q = randn(gen(T), 3, T, 2, 64)
    ctx = [8200, 700, 129]
    out, lse = attend(c, q, ctx, n_new)
    check_attention(c, q, ctx, n_new, out, lse)


def test_attention_where_nothing_or_little_is_there():
    c = Cache(6, 6, 2, 64, seed=5)
    c.table[0, :] = -1                                              # nothing at all
    c.table[1, 1:4] = -1                                            # a gap
    c.table[2, 0] = 10 ** 6
    c.table[3, 5] = c.pool["k"].shape[0]
    c.push()
    q = randn(gen(8), 6, 4, 4, 64)
    ctx = [300, 300, 10, 380, 100000, -7]                           # row 2: its only block is none; rows 3, 4: past the table
    out, lse = attend(c, q, ctx)
    check_attention(c, q, ctx, None, out, lse)
    assert (out[0] == 0).all() and (out[2] == 0).all()


def test_attention_ignores_what_lies_behind_and_shows_what_is_bad():
    c = Cache(3, 4, 1, 64, seed=7)
    for r in range(3):
        for n in ("k", "v"):
            c.scale[n][c.table[r, 2:]] = np.nan                     # blocks behind the rows' tokens
    c.scale["v"][c.table[1, 0]] = np.nan                            # a bad block that row 1 sees
    c.push()
    q = randn(gen(9), 3, 2, 3, 64)
    q[2, 0, 1, 3] = math.nan
    q[2, 1, 0, 3] = math.inf
    q[0, 0, 0] = 0                                                  # no direction: the plain mean
    ctx = [100, 70, 126]
    out, lse = attend(c, q, ctx)
    assert torch.isnan(out[1]).all() and torch.isfinite(lse[1]).all()
    assert torch.isnan(out[2, 0, 1]).all() and torch.isnan(out[2, 1, 0]).all() and torch.isnan(lse[2, 0, 1]) and torch.isnan(lse[2, 1, 0])
    q[2, 0, 1], q[2, 1, 0] = 0, 0
    c.scale["v"][c.table[1, 0]] = 0.01
    c.push()
    again, lse2 = attend(c, q, ctx)
    check_attention(c, q, ctx, None, again, lse2)
    assert torch.equal(again[0], out[0]) and torch.equal(again[2, 0, [0, 2]], out[2, 0, [0, 2]])


def test_attention_with_scores_far_apart():
    """Scores of some hundreds: one token has all of the weight, others underflow, and a masked one would be the largest."""
    c = Cache(4, 3, 1, 128, seed=8)
    for n in ("k", "v"):
        c.scale[n][:] = 1.0
    c.push()
    q = randn(gen(10), 4, 3, 2, 128) * torch.tensor([1e-3, 0.1, 1.0, 40.0])[:, None, None, None]
    ctx = [150, 64, 63, 10]
    out, lse = attend(c, q, ctx)
    check_attention(c, q, ctx, None, out, lse)


def test_attention_is_the_same_every_time_and_in_place_of_strided_views():
    c = Cache(5, 40, 2, 64, seed=11)
    q = randn(gen(12), 5, 2, 4, 64)
    ctx = [2500, 17, 900, 64, 2000]
    ws = binding.new_attention_workspace(c.gpu, 5, 2, 4)
    first, lse = attend(c, q, ctx, ws=ws)
    for _ in range(20):
        out, l2 = attend(c, q, ctx, ws=ws)
        assert torch.equal(out, first) and torch.equal(l2, lse)
    wide = torch.full((5, 2, 7 * 64 + 3), 55.0, device=DEV)           # queries and outputs inside wider rows
    wide[:, :, 1:257] = q.reshape(5, 2, 256).to(DEV)
    res = torch.full((5, 2, 300), 55.0, device=DEV)
    binding.tabed_attention_q8(c.gpu, ws, wide[:, :, 1:257], torch.tensor(ctx, dtype=torch.int32, device=DEV), res[:, :, 9:265])
    torch.cuda.synchronize()
    assert torch.equal(res[:, :, 9:265].cpu().reshape(5, 2, 4, 64), first)
    assert (res[:, :, :9] == 55).all() and (res[:, :, 265:] == 55).all()


@pytest.mark.parametrize("T", [1, 5])
def test_attention_at_any_alignment_of_the_values(T):
    """bf16 queries and outputs that begin at odd addresses of two bytes, tokens 2 bytes past a multiple of 16 apart."""
    c = Cache(4, 6, 2, 96, seed=20)
    q = randn(gen(21), 4, T, 6, 96, dtype=BF16)
    ctx = [300, 5, 64, 200]
    wide_q, wide_o = (torch.full((4, T, 6 * 96 + 9), 55.0, dtype=BF16, device=DEV) for _ in range(2))
    wide_q[:, :, 3:3 + 576] = q.reshape(4, T, 576).to(DEV)
    ws = binding.new_attention_workspace(c.gpu, 4, T, 6)
    binding.tabed_attention_q8(c.gpu, ws, wide_q[:, :, 3:579], torch.tensor(ctx, dtype=torch.int32, device=DEV), wide_o[:, :, 1:577])
    torch.cuda.synchronize()
    assert (wide_o[:, :, 0] == 55).all() and (wide_o[:, :, 577:] == 55).all()
    out, _ = attend(c, q, ctx, out_type=BF16, ws=ws)
    assert torch.equal(wide_o[:, :, 1:577].cpu().reshape(4, T, 6, 96), out)
    check_attention(c, q, ctx, None, out, None)


def test_cache_past_four_gigabytes():
    """Blocks behind the first 2^32 bytes of the pool: appended to and read."""
    kvh, hd, blocks = 8, 128, 66000
    k, v = (torch.empty((blocks, kvh, 64 * hd), dtype=torch.int8, device=DEV) for _ in range(2))
    ks, vs = (torch.empty((blocks, kvh), device=DEV) for _ in range(2))
    table = torch.tensor([[blocks - 1, 3], [65999 - 40, 65600]], dtype=torch.int32, device=DEV)
    big = binding.CacheQ8(k, v, ks, vs, table, hd)
    small = binding.CacheQ8.allocate(2, 128, kvh, hd)
    g = gen(22)
    x, y, q = (randn(g, 2, 100, kvh, hd, dtype=BF16).to(DEV) for _ in range(3))
    outs = []
    for cache in (big, small):
        ctx = torch.zeros(2, dtype=torch.int32, device=DEV)
        binding.tabed_cache_append_q8(cache, x, y, ctx)
        out = torch.zeros((2, 100, kvh, hd), device=DEV)
        binding.tabed_attention_q8(cache, binding.new_attention_workspace(cache, 2, 100, kvh), q, ctx, out)
        outs.append(out)
    assert torch.equal(*outs) and (outs[0][:, 0] != 0).any()
    for name, pool in (("k", k), ("v", v)):                         # the tokens' bytes (what lies behind the 100th is nobody's)
        where = torch.from_numpy(ref.layout(name, hd)).to(DEV)
        at = [p[:, :, where].transpose(1, 2).reshape(2, 128, kvh, hd)[:, :100] for p in (pool[table.flatten().tolist()], getattr(small, name))]
        assert torch.equal(*at)


def test_two_streams_at_once():
    """Calls with workspaces of their own on two streams, running side by side."""
    c = Cache(4, 60, 2, 64, seed=23)
    q = [randn(gen(24 + i), 4, 1, 4, 64).to(DEV) for i in range(2)]
    ctx = torch.tensor([3000, 64, 3500, 1000], dtype=torch.int32, device=DEV)
    ws = [binding.new_attention_workspace(c.gpu, 4, 1, 4) for _ in range(2)]
    alone = []
    for i in range(2):
        out = torch.zeros((4, 1, 4, 64), device=DEV)
        binding.tabed_attention_q8(c.gpu, ws[i], q[i], ctx, out)
        alone.append(out)
    torch.cuda.synchronize()
    streams, outs = [torch.cuda.Stream() for _ in range(2)], [torch.zeros((4, 1, 4, 64), device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            binding.tabed_attention_q8(c.gpu, ws[i], q[i], ctx, outs[i], stream=streams[i])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], alone[0]) and torch.equal(outs[1], alone[1])


def test_attention_reads_shared_blocks():
    c = Cache(4, 5, 2, 64, seed=13)
    c.table[1:, :3] = c.table[0, :3]                                # one beginning for all rows
    c.push()
    q = randn(gen(14), 4, 1, 6, 64)
    ctx = [200, 250, 192, 319]
    out, lse = attend(c, q, ctx)
    check_attention(c, q, ctx, None, out, lse)


# ------------------------------------------------------------------ together
def test_captured_decode_steps_replay_as_eager():
    """append, attention, quantisation and product of a decode step, captured once and replayed over growing rows."""
    rows, kvh, hd, steps = 3, 2, 64, 6
    d = kvh * hd
    c, e = (Cache(rows, 3, kvh, hd, seed=15) for _ in range(2))
    g = gen(16)
    w = torch.randint(-127, 128, (96, d), generator=g, dtype=torch.int8).to(DEV)
    sw, gain = (torch.rand(96, generator=g) * 0.01).to(DEV), torch.ones(d, device=DEV)
    inputs = [tuple(randn(g, rows, d).to(DEV) for _ in range(3)) for _ in range(steps)]

    def program(c, st):
        binding.tabed_cache_append_q8(c.gpu, st["k"], st["v"], st["ctx"])
        binding.tabed_attention_q8(c.gpu, st["ws"], st["q"], st["ctx"], st["att"])
        binding.tabed_norm_q8(st["att"], st["a8"], st["s"], gain=gain)
        binding.tabed_linear_q8(st["a8"], st["s"], w, sw, st["y"])

    def state(c):
        z = lambda *s, dt=F32: torch.zeros(s, dtype=dt, device=DEV)
        return dict(q=z(rows, d), k=z(rows, d), v=z(rows, d), ctx=torch.tensor([60, 0, 127], dtype=torch.int32, device=DEV),
                    ws=binding.new_attention_workspace(c.gpu, rows, 1, kvh), att=z(rows, d), a8=z(rows, d, dt=torch.int8), s=z(rows), y=z(rows, 96))

    a, b = state(c), state(e)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph.capture_begin()
        program(c, a)
        graph.capture_end()
    torch.cuda.current_stream().wait_stream(side)
    for x in inputs:
        for st in (a, b):
            for n, t in zip(("q", "k", "v"), x):
                st[n].copy_(t)
        graph.replay()
        program(e, b)
        torch.cuda.synchronize()
        for n in ("att", "a8", "s", "y"):
            assert torch.equal(a[n], b[n]), n
        assert torch.isfinite(a["y"]).all() and (a["a8"] != 0).any()
        a["ctx"] += 1
        b["ctx"] += 1
    for n in ("k", "v", "kscale", "vscale"):
        assert torch.equal(getattr(c.gpu, n), getattr(e.gpu, n))

"""Attention over trees in an e4m3 cache whose scales differ by many powers of two, and what one node's entry means for the others."""
import math

import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn
# Nodes, query and key / value heads: waves with tiles of their own (one, two groups of queries), waves that share tiles (one, two, four with queries of their own).
SHAPES = [(6, 4, 2), (12, 4, 2), (20, 4, 2), (40, 4, 2), (40, 8, 2)]


@pytest.fixture(scope="module")
def B():
    from paper_2601_20357_amd import binding
    binding.load()
    return binding


def i32(t):
    return None if t is None else torch.as_tensor(t).to(torch.int32).to(DEV)


def make(B, tokens, kvh, hd, seed, vscale=None, bf16=False):
    """One row's cache, blocks in order; vscale(token) [tokens rounded up]: its scales of values."""
    g = torch.Generator().manual_seed(seed)
    blocks = (tokens + 63) // 64
    k, v = (torch.randn(1, blocks, kvh, 64, hd, generator=g).to(torch.bfloat16) for _ in range(2))
    table = torch.arange(blocks, dtype=torch.int32, device=DEV)[None]
    if bf16:
        return B.CachePaged(k.to(DEV), v.to(DEV), table)
    ks, vs = (torch.rand(1, blocks, kvh, 64, generator=g) * 0.5 + 0.5 for _ in range(2))
    if vscale is not None:
        vs *= vscale(torch.arange(blocks * 64)).view(blocks, 1, 64)[None]
    return B.CachePaged(k.float().to(F8).to(DEV), v.float().to(F8).to(DEV), table, ks.to(DEV), vs.to(DEV))


def held(cache, name):
    x, s = getattr(cache, name), getattr(cache, name + "scale")
    x = x[0].cpu().double()
    return x if s is None else x * s[0].cpu().double()[..., None]


def call(B, cache, q, ctx, parents):
    N, qh = q.shape[1:3]
    ws = B.new_attention_nodes_workspace(cache, 1, N, qh)
    out, lse = torch.zeros_like(q), torch.zeros(1, N, qh, device=DEV)
    B.tabed_attention_nodes(cache, ws, q, i32([ctx]), out, parents=i32(parents), lse=lse)
    return out, lse


def check(B, cache, q, ctx, parents, prob=2.0 ** -8):
    """prob: what a probability is rounded to, relative.  Two 16-bit types hold them: 2^-11 next to the largest product with a scale, 2^-8 far below it."""
    N, qh, hd = q.shape[1:]
    out, lse = call(B, cache, q.to(DEV), ctx, parents)
    k, v = held(cache, "k"), held(cache, "v")
    want, wlse, mass = ref.attention(q.double(), k, v, cache.table.cpu(), k.shape[0], [ctx], parents, [N], hd ** -0.5)
    # As in the tests of sizes: scores' sums in fp32, the product with the scale, the exponential of a difference of up to 2^7; then the result's own rounding, the
    # probability's, its error twice, the sums in fp32 (whose terms are up to 2^17 here: 2^-24 for every doubling of a sum's length, 2^-14 covers them).
    rel = (hd + 4) * 2.0 ** -24 * float((q.double().abs().sum(-1).amax() * k.abs().amax() * hd ** -0.5).clamp(max=2.0 ** 12)) + 2.0 ** -14
    # Results below the smallest normal number of bf16 and fp32, 2^-126, may be rounded to 0 or to any of the few numbers there.  So may probabilities, and products of
    # them and scales: they are taken relative to the largest product, which becomes 2^7 at least, with scales counted as 2^-40 to 2^38.  No probability is above 1, so lost are
    # probabilities, or products, below 2^-133 of the largest scale so counted: of each token that, once as it is and once times its scale, times a value of at most 448.
    lost = 0.0
    if cache.vscale is not None:
        most = float(cache.vscale.max())
        lost = (ctx + N) * 448 * 2.0 ** -133 * min(max(most, 2.0 ** -40), 2.0 ** 38) * max(1.0, most)
    tol = 2.0 ** -8 * want.abs() + mass * (prob + 2 * rel + 2.0 ** -14) + 2.0 ** -126 + lost
    got = out.cpu().double()
    bad = (got - want).abs() > tol
    assert not bad.any(), f"{int(bad.sum())} of {bad.numel()} off, at most {float(((got - want).abs() / tol).nan_to_num(9e9).max()):.2f} times the tolerance"
    assert ((lse.cpu().double() - wlse).abs() <= rel + 2.0 ** -22 * wlse.abs()).all()


def queries(N, qh, hd, seed):
    return (1.5 * torch.randn(1, N, qh, hd, generator=torch.Generator().manual_seed(seed))).to(torch.bfloat16)


def tree(N):
    return ref.tree(N, "random", 3)[None]


SCALES = {"up": lambda t: torch.exp2(8.0 * (t // 32)), "down": lambda t: torch.exp2(-8.0 * (t // 32)), "steps": lambda t: torch.exp2(7.0 * (t % 11)),
          "tiny": lambda t: torch.exp2(-100.0 - (t % 5)), "large": lambda t: torch.exp2(90.0 + t % 5), "zeros": lambda t: (t % 3 != 0).float(),
          "some": lambda t: torch.where(t % 50 == 7, 2.0 ** 40, 1.0), "both": lambda t: torch.exp2(100.0 * (t % 3 - 1))}


@pytest.mark.parametrize("kind", list(SCALES))
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_scales_of_values(B, N, qh, kvh, hd, kind):
    ctx = 350
    check(B, make(B, ctx + N, kvh, hd, hd + N, SCALES[kind]), queries(N, qh, hd, 1), ctx, tree(N))


@pytest.mark.parametrize("kind", ["both", "large", "up", "some"])
@pytest.mark.parametrize("N,qh,kvh,hd,ctx", [(130, 12, 3, 256, 100), (40, 8, 2, 128, 350), (5, 4, 2, 64, 200), (17, 2, 1, 64, 900)])
def test_scales_and_scores_far_apart(B, N, qh, kvh, hd, ctx, kind):
    """Scores of 30 and more either side of the mean: products of any size, some of them of tokens whose value is 0 in a dim."""
    check(B, make(B, ctx + N, kvh, hd, hd + N, SCALES[kind]), (20 * queries(N, qh, hd, 8).float()).to(torch.bfloat16), ctx, tree(N))


@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_probabilities_keep_eleven_bits(B, N, qh, kvh, hd):
    """Scales and scores within 2^14 of each other: all are rounded to 2^-11."""
    for ctx in (40, 2500):
        check(B, make(B, ctx + N, kvh, hd, hd + N), queries(N, qh, hd, 2), ctx, tree(N), prob=2.0 ** -11)


@pytest.mark.parametrize("scale", [2.0 ** 17, 2.0 ** 30, 2.0 ** 60, 2.0 ** 118])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_a_large_sibling_is_nothing_to_those_beside_it(B, N, qh, kvh, hd, scale):
    ctx, bad = 75, 2
    cache, parents, q = make(B, ctx + N, kvh, hd, 5), tree(N), queries(N, qh, hd, 3).to(DEV)
    below = torch.tensor([bad in ref.above(parents, 0, j) for j in range(N)])
    assert 0 < below.sum() < N
    clean = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
    cache.vscale[0, (ctx + bad) // 64, :, (ctx + bad) % 64] = scale
    got = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
    for a, c in zip(got, clean):                                         # (lse of those below: sums relative to another power of two, checked next)
        assert torch.equal(a[~below], c[~below])
    check(B, cache, q.cpu(), ctx, parents)


@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_a_large_sibling_beside_tokens_without_values(B, N, qh, kvh):
    """As above, where the others see tokens whose scale is 0 next to it: what they add to the sums of probabilities, they add in the same order."""
    hd = 64
    for ctx, bad in ((75, 2), (60, 1), (0, 2)):
        cache, parents, q = make(B, ctx + N, kvh, hd, 15), tree(N), queries(N, qh, hd, 13).to(DEV)
        cache.vscale[0, :, :, ::3] = 0.0
        below = torch.tensor([bad in ref.above(parents, 0, j) for j in range(N)])
        clean = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
        cache.vscale[0, (ctx + bad) // 64, :, (ctx + bad) % 64] = 2.0 ** 60
        got = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
        for a, c in zip(got, clean):
            assert torch.equal(a[~below], c[~below])
        check(B, cache, q.cpu(), ctx, parents)


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("hd", [64, 128, 256])
@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_a_loud_sibling_is_nothing_to_those_beside_it(B, N, qh, kvh, hd, bf16):
    """Scores of 100 and more for those who see it: the others' results are the same bits."""
    ctx, bad = 75, 2
    cache, parents, q = make(B, ctx + N, kvh, hd, 6, bf16=bf16), tree(N), queries(N, qh, hd, 4).to(DEV)
    below = torch.tensor([bad in ref.above(parents, 0, j) for j in range(N)])
    clean = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
    (cache.k if bf16 else cache.kscale)[0, (ctx + bad) // 64, :, (ctx + bad) % 64] *= 100
    got = [x[0].cpu() for x in call(B, cache, q, ctx, parents)]
    for a, c in zip(got, clean):
        assert torch.equal(a[~below], c[~below])
        assert not torch.equal(a[below], c[below])
    check(B, cache, q.cpu(), ctx, parents)


@pytest.mark.parametrize("scale", [2.0 ** 17, 2.0 ** 30, 2.0 ** 60])
@pytest.mark.parametrize("N,qh,kvh", SHAPES)
def test_a_large_token_that_counts_for_nothing(B, N, qh, kvh, scale):
    """Its score is 150 below the others': its values times 2^60 are still nothing."""
    ctx, hd, at = 600, 64, 130
    cache, q = make(B, ctx + N, kvh, hd, 7), queries(N, qh, hd, 5).abs()
    cache.k[0, at // 64, :, at % 64] = -8.0
    cache.kscale[0, at // 64, :, at % 64] = 150.0 / (8.0 * float(q.float().sum(-1).min()) * hd ** -0.5)
    cache.vscale[0, at // 64, :, at % 64] = scale
    check(B, cache, q, ctx, tree(N))


@pytest.mark.parametrize("share,tokens", [(4e-3, 30_000), (1e-3, 30_000), (1e-4, 30_000), (1e-5, 30_000), (1e-6, 9_000)])
@pytest.mark.parametrize("zeros", ["values", "scale"])
@pytest.mark.parametrize("N,qh,kvh", [(3, 2, 1), (20, 2, 1), (40, 4, 1)])
def test_a_first_token_that_takes_nearly_all_and_holds_nothing(B, N, qh, kvh, zeros, share, tokens):
    """All others together have `share` of the probability, and make the result."""
    hd = 64
    cache = make(B, tokens + N, kvh, hd, 8)
    q = queries(1, 1, hd, 6).expand(1, N, qh, hd).contiguous()
    k, scale = held(cache, "k"), hd ** -0.5
    rest = float(torch.logsumexp((k @ q[0, 0, 0].double()).flatten()[1:tokens] * scale, 0))
    cache.k[0, 0, 0, 0] = q[0, 0, 0].float().to(F8).to(DEV)
    dot = float((cache.k[0, 0, 0, 0].cpu().double() * q[0, 0, 0].double()).sum()) * scale
    cache.kscale[0, 0, 0, 0] = (rest - math.log(share)) / dot
    if zeros == "values":
        cache.v[0, 0, 0, 0] = torch.full((hd,), 2.0 ** -9).to(F8).to(DEV)
        cache.v[0, 0, 0, 0, :8] = 0.0
    else:
        cache.vscale[0, 0, 0, 0] = 0.0
    check(B, cache, q, tokens, tree(N))


@pytest.mark.parametrize("N,qh,kvh", [(6, 4, 2), (40, 8, 2)])
def test_ranges_with_scales_of_their_own(B, N, qh, kvh):
    """A long row, cut into ranges whose scales and scores lie far apart: their sums are joined as one."""
    ctx, hd = 5000, 128
    for step, loud in ((7, 0.0), (-7, 0.0), (7, -5.0), (-7, 5.0)):
        cache = make(B, ctx + N, kvh, hd, 9, lambda t: torch.exp2(float(step) * (t // 512)))
        at = torch.arange(cache.k.shape[1] * 64).view(-1, 1, 64)
        cache.kscale[0] *= torch.exp2(loud * (at // 512) / 10).to(DEV)
        check(B, cache, queries(N, qh, hd, 7), ctx, tree(N))

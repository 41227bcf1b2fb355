"""tabed_attention_q8 where tokens of one call see different blocks, where its workspace serves several sizes, at scores of any size, and in each of
the forms that sizes choose between."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20357_amd import binding, synth
from q8_reference import layout
from test_gpu_q8 import BF16, DEV, F32, Cache, attend, check_attention, gen, randn
from test_gpu_q8_step import Pair

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which,value", [("v", math.nan), ("v", math.inf), ("k", math.nan)])
@pytest.mark.parametrize("hd,group,T", [(64, 1, 2), (64, 2, 2), (96, 1, 4), (256, 1, 3), (64, 4, 6), (128, 8, 2), (96, 7, 40), (256, 3, 5), (32, 1, 70)])
def test_a_bad_block_stays_with_the_tokens_that_see_it(hd, group, T, which, value):
    """The tokens of a call straddle the border of a block that is bad, as appending leaves it where a later token is not finite: those before it
    have the results, bit for bit, of a call where it is good.  Rows in one range and in several."""
    c = Cache(4, 40, 2, hd, seed=hd + T)
    q = randn(gen(T), 4, T, 2 * group, hd)
    ctx = [63, 64 * 39 - 1, 64 * 3 - 2, 100]                          # rows 0 to 2: token 0 (and 1) end a block; row 3: 28 tokens do
    good, glse = attend(c, q, ctx)
    check_attention(c, q, ctx, None, good, glse)
    first = [(x // 64 + 1) * 64 - x for x in ctx]                      # the first token in the next block
    for r in range(4):
        c.scale[which][c.table[r, ctx[r] // 64 + 1]] = value
    c.push()
    out, lse = attend(c, q, ctx)
    for r in range(4):
        n = first[r]
        assert torch.equal(out[r, :n], good[r, :n]) and torch.equal(lse[r, :n], glse[r, :n]), r
        assert (not torch.isfinite(out[r, n:]).any()), r
        if which == "v":
            assert torch.equal(lse[r, n:], glse[r, n:]), r


def test_a_bad_token_leaves_earlier_tokens_of_its_call_alone():
    """Appending and attending to tokens of which a later one, alone in its block, is not finite."""
    rows, kvh, hd = 2, 1, 64
    outs = []
    for bad in (1.0, math.nan, math.inf):
        cache = binding.CacheQ8.allocate(rows, 128, kvh, hd)
        g = gen(3)
        zero = torch.zeros(rows, dtype=torch.int32, device=DEV)
        binding.tabed_cache_append_q8(cache, randn(g, rows, 63, kvh, hd).to(DEV), randn(g, rows, 63, kvh, hd).to(DEV), zero)
        k, v, q = (randn(g, rows, 2, kvh, hd) for _ in range(3))
        v[0, 1, 0, 7] = bad
        ctx = zero + 63
        binding.tabed_cache_append_q8(cache, k.to(DEV), v.to(DEV), ctx)
        out = torch.zeros((rows, 2, kvh, hd), device=DEV)
        binding.tabed_attention_q8(cache, binding.new_attention_workspace(cache, rows, 2, kvh), q.to(DEV), ctx, out)
        outs.append(out.cpu())
    for out in outs[1:]:
        assert torch.isnan(out[0, 1]).all()
        assert torch.equal(out[0, 0], outs[0][0, 0]) and torch.equal(out[1], outs[0][1])


def test_one_workspace_serves_calls_of_different_sizes():
    """A loop that verifies blocks of six tokens and decodes single ones in between, over two caches: the largest call's workspace serves them all."""
    caches = [Cache(2, 130, 2, 64, seed=31), Cache(5, 40, 1, 96, seed=32)]
    ctx = [[8200, 3000], [2500, 17, 900, 64, 2000]]
    calls = [(i, randn(gen(10 * T + i), caches[i].rows, T, 4, caches[i].hd)) for i in (0, 1) for T in (1, 2, 6, 40)]
    need = [binding.tabed_attention_q8_workspace_bytes(caches[i].gpu, caches[i].rows, q.shape[1], 4) for i, q in calls]
    assert len(set(need)) > 4
    want = [attend(caches[i], q, ctx[i]) for i, q in calls]
    check_attention(caches[0], calls[2][1], ctx[0], None, *want[2])
    ws = torch.empty(max(need), dtype=torch.uint8, device=DEV)
    ws.fill_(0xa5)
    binding.tabed_attention_q8_workspace_init(caches[0].gpu, 2, 1, 4, ws)            # (prepared by the sizes of a small call)
    for at in (0, 7, 3, 2, 0, 5, 6, 1, 4, 2, 3, 7, 0, 2, 0):
        i, q = calls[at]
        out, lse = attend(caches[i], q, ctx[i], ws=ws)
        assert torch.equal(out, want[at][0]) and torch.equal(lse, want[at][1]), at


def test_one_workspace_serves_body_steps_of_different_sizes():
    bcs = [synth.BodyConfig(layers=2, d=256, heads=4, d_ff=512, V=300, max_ctx=1000), synth.BodyConfig(layers=1, d=128, heads=1, d_ff=256, V=300, max_ctx=640)]
    sizes = [(0, 3), (0, 20), (1, 2), (1, 9)]
    ctx = lambda i, rows: [(bcs[i].max_ctx - 10) // (1 + r) for r in range(rows)]
    pairs = lambda: [Pair(bcs[i], rows, 40 + rows, ctx(i, rows)) for i, rows in sizes]
    want = [p.step(np.arange(p.rows) * 7) for p in pairs()]
    ps = pairs()
    ws = max((p.ws for p in ps), key=lambda w: w.numel()).clone()
    ws.fill_(0xa5)
    binding.tabed_body_q8_workspace_init(ps[0].cfg, ps[0].gpu, 3, ws)
    for at in (1, 0, 3, 2):
        ps[at].ws = ws
        for got, w in zip(ps[at].step(np.arange(ps[at].rows) * 7), want[at]):
            assert torch.equal(got, w), at
    for at in (2, 1, 3, 0):                                                         # again, from the first step's state
        fresh = Pair(bcs[sizes[at][0]], sizes[at][1], 40 + sizes[at][1], ctx(*sizes[at]))
        fresh.ws = ws
        for got, w in zip(fresh.step(np.arange(fresh.rows) * 7), want[at]):
            assert torch.equal(got, w), at


@pytest.mark.parametrize("size", [300.0, 3e6, 7e6, 4.1e8, -1e10, 1e20, -1e30])
@pytest.mark.parametrize("hd,group,T", [(64, 8, 1), (128, 5, 2), (256, 6, 1), (96, 1, 40), (64, 2, 1)])
def test_attention_with_scores_of_any_size(hd, group, T, size):
    """Queries of one direction: a score is a key's step times the same number, so tokens of the extreme step share the weight equally, and n others,
    a step or more away, have at most n exp(-|size| / sqrt(hd)) of it, which moves outputs by at most the difference of two values, 254, times that
    (a trace at the first size, nothing at the others).  Counted in half steps of fp32 (2^-24): probabilities are equal and exact; the sums over
    blocks as in the reference (2 (blocks + 220)), scales, division and places 12.  At the first size, where scores are below 2^20, many queries
    have them scaled in the addition that takes the maximum off, except in a block that is seen in part: the probabilities of equal scores are then off by
    e = (a rounding each of score, maximum and difference, of the score's size, + 14 and exp2's 2) ln 2 or less, twice in their quotient.  The logarithm: a score is a product of six roundings
    (query's step twice, scale, key's scale, score, base 2 to e), each of its own size, log2 and the sum two more, of the sum of at most 60 ties (below 6)."""
    c = Cache(5, 70, 2, hd, seed=hd + T)
    for n in ("k", "v"):
        c.scale[n][:] = 1.0
    c.push()
    q = torch.zeros(5, T, 2 * group, hd)
    for i in range(2 * group):
        q[..., i, (7 * i + 3) % hd] = size
    ctx = [0, 64 * 4 - 1, 64 * 69 - 1, 1000, 30]
    out, lse = attend(c, q, ctx)
    for r in range(5):
        for t in range(T):
            n = ctx[r] + t + 1
            blocks = (n + 63) // 64
            for i in range(2 * group):
                h, dim = i // group, (7 * i + 3) % hd
                k, v = (np.concatenate([c.pool[w][c.table[r, b], h][layout(w, hd)] for b in range(blocks)])[:n].astype(np.float64) for w in ("k", "v"))
                score = k[:, dim] * float(np.float32(size)) * hd ** -0.5
                best = score == score.max()
                want, wlse = v[best].mean(0), score.max() + math.log(best.sum())
                assert best.sum() <= 60
                others = n * math.exp(-abs(size) * hd ** -0.5)
                e = 3 * abs(wlse) + 20 if abs(size) < 1000 else 0
                tol = (2 * (blocks + 220) + 12 + 2 * e) * 2.0 ** -24 * np.abs(v[best]).max(0) + 254 * others
                assert (np.abs(out[r, t, i].double().numpy() - want) <= tol).all(), (r, t, i)
                assert abs(float(lse[r, t, i]) - wlse) <= (8 * abs(wlse) + 8 * 6 + e) * 2.0 ** -24 + others, (r, t, i)

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


@pytest.mark.parametrize("hd", [32, 64, 96, 128])
@pytest.mark.parametrize("group,T,n_new", [(1, 1, None), (4, 1, [1, 0] * 17), (3, 6, [6, 0, 3, 5, 1, 2, 6, 4, 6, 6] * 3 + [6, 6, 0, 6]), (8, 1, None), (2, 33, None)])
def test_rows_and_heads_that_fill_the_chip(hd, group, T, n_new):
    """More than 256 rows x heads x tiles of queries: workgroups of four waves, one range a row."""
    rows, kvh = 34, 8
    c = Cache(rows, 7, kvh, hd, seed=hd + T)
    c.table[3, 1], c.table[4, :], c.table[5, 0] = -1, -1, 10 ** 7
    c.push()
    assert rows * kvh * 1 > 256
    q = randn(gen(hd + T), rows, T, kvh * group, hd, dtype=BF16 if group == 4 else F32)
    ctx = [int(x) for x in np.random.default_rng(T).integers(0, 380, rows)]
    ctx[:3] = [0, 63, 64]
    out, lse = attend(c, q, ctx, n_new)
    check_attention(c, q, ctx, n_new, out, lse)


@pytest.mark.parametrize("hd,kvh,group,T,rows,blocks", [(64, 4, 1, 1, 65, 530), (64, 4, 2, 3, 65, 530), (32, 2, 8, 1, 129, 300), (256, 1, 1, 1, 257, 270), (256, 1, 6, 1, 257, 259)])
def test_waves_that_open_more_than_64_blocks(hd, kvh, group, T, rows, blocks):
    """Rows in one range with more blocks than a wave of four opens at a time, from a small pool, missing ones around the border of the 64th of a wave and
    of a whole opening among them."""
    assert blocks > 4 * 64 and rows * kvh > 256
    c = Cache(4, 3, kvh, hd, seed=hd + blocks)
    g = np.random.default_rng(blocks)
    pool = c.pool["k"].shape[0]
    c.rows, c.width = rows, blocks
    c.table = g.integers(0, pool, (rows, blocks)).astype(np.int32)
    c.table[1, 250:262] = -1
    c.table[2, :256] = -1                                              # a whole opening is missing
    c.table[3, 256:] = -1
    c.table[5, 253::4] = pool                                          # one wave's
    c.push()
    q = randn(gen(T), rows, T, kvh * group, hd)
    ctx = [int(x) for x in g.integers(255 * 64, blocks * 64 - T, rows)]
    ctx[:8] = [256 * 64 - 1, blocks * 64 - T, blocks * 64 - T, blocks * 64 - T, 256 * 64, blocks * 64 - T, 70, 0]
    out, lse = attend(c, q, ctx)
    few = [0, 1, 2, 3, 4, 5, 6, 7, rows - 1]                           # (the definition takes its time: these rows, and that equal rows are equal)
    c.rows, c.table = len(few), c.table[few]
    check_attention(c, q[few], [ctx[r] for r in few], None, out[few], lse[few])
    assert torch.isfinite(out).all()


@pytest.mark.parametrize("rows", [200, 256])
def test_eight_waves_that_open_more_than_64_blocks(rows):
    """Workgroups of eight waves with more than 512 blocks: one long row among short ones, in two ranges (200 rows) and in one (256)."""
    hd, blocks = 64, 1100
    c = Cache(4, 3, 1, hd, seed=3)
    g = np.random.default_rng(5)
    c.rows, c.width = rows, blocks
    c.table = g.integers(0, c.pool["k"].shape[0], (rows, blocks)).astype(np.int32)
    c.table[0, 500:530], c.table[0, 1060:1066] = -1, -1
    c.push()
    q = randn(gen(3), rows, 1, 2, hd)
    ctx = [blocks * 64 - 1] + [int(x) for x in g.integers(0, 300, rows - 1)]
    out, lse = attend(c, q, ctx)
    few = [0, 1, 2, rows - 1]
    c.rows, c.table = len(few), c.table[few]
    check_attention(c, q[few], [ctx[r] for r in few], None, out[few], lse[few])


@pytest.mark.parametrize("hd,kvh,group,T,qt", [(64, 1, 4, 700, F32), (128, 2, 2, 333, BF16), (256, 1, 3, 130, F32), (32, 1, 1, 1500, BF16)])
def test_a_prompt(hd, kvh, group, T, qt):
    """Hundreds of new tokens a row: many tiles of queries over the same blocks, each with an end of its own."""
    width = (T + 200) // 64 + 1
    c = Cache(2, width, kvh, hd, seed=T)
    q = randn(gen(T), 2, T, kvh * group, hd, dtype=qt)
    ctx, n_new = [0, 137], [T, T - 61]
    out, lse = attend(c, q, ctx, n_new)
    check_attention(c, q, ctx, n_new, out, lse)

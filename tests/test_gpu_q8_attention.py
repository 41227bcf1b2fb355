"""tabed_attention_q8 where tokens of one call see different blocks, where its workspace serves several sizes, at scores of any size, and in each of
the forms that sizes choose between."""
import math

import numpy as np
import pytest
import torch

from paper_2601_20357_amd import binding
from test_gpu_q8 import BF16, DEV, F32, Cache, attend, check_attention, gen, randn

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

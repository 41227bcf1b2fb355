"""Attention over trees where the block table is much wider than the rows are long, as a table for the longest context that is allowed."""
import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def B():
    from paper_2601_20357_amd import binding
    binding.load()
    return binding


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("N,qh,kvh", [(1, 4, 2), (7, 4, 2), (24, 4, 4), (40, 8, 2)])
@pytest.mark.parametrize("ctx", [[600], [0, 1, 63, 64, 200, 700], [300] * 80])
def test_a_table_wider_than_the_rows_changes_nothing_but_the_order_of_sums(B, ctx, N, qh, kvh, f8):
    hd, rows, wide = 64, len(ctx), 600
    g = torch.Generator().manual_seed(5)
    tokens = [c + N for c in ctx]
    each = [(t + 63) // 64 for t in tokens]
    shape = (1, sum(each), kvh, 64, hd)
    k, v = (torch.randn(shape, generator=g).to(torch.bfloat16) for _ in range(2))
    scales = [None, None]
    if f8:
        k, v = k.float().to(F8), v.float().to(F8)
        scales = [torch.rand(1, sum(each), kvh, 64, generator=g) * 0.5 + 0.5 for _ in range(2)]
    order, tight = torch.randperm(sum(each), generator=g).to(torch.int32), torch.full((rows, max(each)), -1, dtype=torch.int32)
    for r, n in enumerate(each):
        tight[r, :n] = order[sum(each[:r]):sum(each[:r]) + n]
    loose = torch.full((rows, wide), -1, dtype=torch.int32)              # (a missing block is none of the row's)
    loose[:, :max(each)] = tight
    parents = torch.stack([ref.tree(N, "random", r) for r in range(rows)])
    q = torch.randn(rows, N, qh, hd, generator=g).to(torch.bfloat16)
    dev = lambda x: None if x is None else x.to(DEV)  # noqa: E731

    def call(table):
        cache = B.CachePaged(dev(k), dev(v), dev(table), *map(dev, scales))
        ws = B.new_attention_nodes_workspace(cache, rows, N, qh)
        out, lse = torch.zeros(rows, N, qh, hd, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, N, qh, device=DEV)
        for _ in range(2):                                               # (what the first call leaves in the workspace means nothing to the second)
            B.tabed_attention_nodes(cache, ws, dev(q), torch.tensor(ctx, dtype=torch.int32, device=DEV), out, parents=parents.to(torch.int32).to(DEV), lse=lse)
        return out.cpu().double(), lse.cpu().double()

    full = [x[0].double() * (1.0 if s is None else s[0].double()[..., None]) for x, s in zip((k, v), scales)]
    want, wlse, mass = ref.attention(q.double(), *full, tight, shape[1], ctx, parents, [N] * rows, hd ** -0.5)
    # Scores' sums of hd terms in fp32, which the exponential takes over, and the sums' over up to 2^10 tokens, 2^-14 with room; a probability's rounding, 2^-8, once as it is
    # and once in the sum that results are divided by; the result's own rounding, 2^-8.
    rel = (hd + 4) * 2.0 ** -24 * float(q.double().abs().sum(-1).amax() * full[0].abs().amax() * hd ** -0.5) + 2.0 ** -14
    for out, lse in (call(tight), call(loose)):
        assert ((out - want).abs() <= 2.0 ** -8 * want.abs() + (2 * 2.0 ** -8 + 2 * rel) * 1.01 * mass).all()
        assert ((lse - wlse).abs() <= 2.0 ** -23 * wlse.abs() + rel).all()

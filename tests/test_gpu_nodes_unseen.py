"""Attention over trees: what nobody sees costs nothing either, whatever it holds."""
import math

import pytest
import torch

import nodes_reference as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F8 = torch.float8_e4m3fn


@pytest.mark.parametrize("f8", [False, True])
@pytest.mark.parametrize("N,qh,kvh", [(6, 4, 2), (40, 8, 2)])
def test_time_does_not_go_by_what_nobody_sees(N, qh, kvh, f8):
    """A row whose first block is not there, so that all its tiles go by what is seen; the pool's first block, read in its place, and the slots behind the row's end are zeros, or NaN."""
    from paper_2601_20357_amd import binding as B
    ctx, hd = 6000, 64
    g = torch.Generator().manual_seed(N)
    width = (ctx + N + 63) // 64
    table = torch.arange(1, width + 1, dtype=torch.int32, device=DEV)[None].clone()
    table[0, 0] = -1
    k, v = (torch.randn(width + 1, kvh, 64, hd, generator=g).to(F8 if f8 else torch.bfloat16).to(DEV) for _ in range(2))
    scales = [torch.rand(width + 1, kvh, 64, generator=g).to(DEV) + 0.5 for _ in range(2)] if f8 else [None, None]
    cache = B.CachePaged(k, v, table, *scales)
    q = torch.randn(1, N, qh, hd, generator=g).to(torch.bfloat16).to(DEV)
    parents, lens = ref.tree(N, "random")[None].to(DEV), torch.tensor([ctx], dtype=torch.int32, device=DEV)
    ws, out = B.new_attention_nodes_workspace(cache, 1, N, qh), torch.zeros_like(q)
    end = (ctx + N) % 64

    def fill(what):
        for t in (k, v, *scales):
            if t is not None:
                bits = t.view(torch.uint8 if t.dtype == F8 else t.dtype)
                value = (0xff if math.isnan(what) else 0) if t.dtype == F8 else what
                bits[0] = value
                bits[-1, :, end:] = value

    def least():
        times = []
        for _ in range(15):
            B.tabed_prof_reset()
            B.tabed_prof_enable(True)
            B.tabed_attention_nodes(cache, ws, q, lens, out, parents=parents)
            torch.cuda.synchronize()
            B.tabed_prof_enable(False)
            ms, count = B.tabed_prof_read(B.K_BODY)
            assert count == 1
            times.append(ms)
        return min(times), out.clone()
    fill(0.0)
    time, want = least()
    fill(math.nan)
    spoilt, got = least()
    print(f"{time * 1e3:.1f} us, {spoilt * 1e3:.1f}")
    assert torch.equal(got, want)
    assert spoilt < 1.5 * time, (spoilt, time)

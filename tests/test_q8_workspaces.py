"""Workspaces of the 8-bit attention and body step: what a call expects to find in one is at the same place, and as much, for all sizes."""
import ctypes as C

import pytest

from paper_2601_20357_amd import binding


def cache(**kw):
    f = dict(kv_heads=2, head_dim=64, blocks=10, max_blocks=500)
    f.update(kw)
    return C.byref(binding.TabedCacheQ8(f["kv_heads"], f["head_dim"], f["blocks"], f["max_blocks"]))


@pytest.mark.parametrize("kv_heads,rows,T,q_heads", [(2, 128, 1, 4), (1, 300, 1, 1), (8, 4096, 1, 32), (2, 16, 70, 16), (1024, 65, 2, 1024)])
def test_calls_in_one_range_need_the_counters_alone(kv_heads, rows, T, q_heads):
    """Sizes that fill the chip are not cut into ranges: nothing is joined, whatever the number of their workgroups."""
    need = binding.load().tabed_attention_q8_workspace_bytes
    counters = need(cache(kv_heads=1, max_blocks=1), 1, 1, 1)
    assert 0 < counters <= 1024
    assert need(cache(kv_heads=kv_heads), rows, T, q_heads) == counters


def test_calls_in_several_ranges_need_more():
    need = binding.load().tabed_attention_q8_workspace_bytes
    counters = need(cache(kv_heads=1, max_blocks=1), 1, 1, 1)
    for rows in (1, 3, 127):
        assert need(cache(), rows, 1, 4) > counters

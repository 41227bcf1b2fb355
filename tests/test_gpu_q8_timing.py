"""Kernel timing of the 8-bit operators: which id their launches count under."""
import pytest
import torch

from paper_2601_20357_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_products_do_not_count_as_lm_heads():
    z = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype, device=DEV)
    cfg = binding.make_cfg(V=1000, d=64, n=2, B=3, gamma=2, h=4, w_dtype=1)
    b = binding.RoundBuffers(cfg)
    b.weights.fill_(0.5)
    W8, H8 = z(1000, 64, dtype=torch.int8), z(6, 64, dtype=torch.int8)
    head = b.prepare_draft_step_q8(0, 0, W8, z(1000), H8, z(6), torch.ones(3, device=DEV))
    y = z(6, 1000)
    torch.cuda.synchronize()
    binding.tabed_prof_reset()
    binding.tabed_prof_enable(True)
    try:
        head()
        for _ in range(3):
            binding.tabed_linear_q8(H8, z(6), W8, z(1000), y)
        binding.tabed_norm_q8(y, z(6, 1000, dtype=torch.int8), z(6))
    finally:
        binding.tabed_prof_enable(False)
    counts = [binding.tabed_prof_read(i)[1] for i in range(binding.K_COUNT)]
    binding.tabed_prof_reset()
    assert counts[binding.K_LMHEAD] == 1 and counts[binding.K_SAMPLE] == 1 and counts[binding.K_BODY] == 4 and sum(counts) == 6

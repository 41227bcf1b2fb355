"""tabed_norm_q8 without a gain against its definition to the letter: the values, and so their roundings, are known exactly."""
import numpy as np
import pytest
import torch

from paper_2601_20357_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,d,with_delta", [(700, 400, False), (200, 1000, True), (100, 2001, False), (60, 4001, True), (20, 8001, False), (10, 16001, True),
                                              (6, 32768, False)])
def test_steps_are_the_division_rounded_to_even(rows, d, with_delta):
    """Values in the middle between two steps, and the fp32 numbers next to it, at scales of all sizes: q = rint(x / scale), both operations as
    fp32 has them, scale = max / 127."""
    g = np.random.default_rng(d)
    top = np.ldexp(1 + g.random((rows, 1)), g.integers(-60, 60, (rows, 1))).astype(np.float32)
    scale = top / np.float32(127)
    middle = ((g.integers(-126, 126, (rows, d)) + np.float32(0.5)) * scale).astype(np.float32)
    x = (middle.view(np.int32) + g.integers(-1, 2, (rows, d), dtype=np.int32)).view(np.float32)
    x[np.arange(rows), g.integers(0, d, rows)] = top[:, 0]
    delta = None
    if with_delta:                                     # parts whose sum is x exactly
        delta = np.where(g.random((rows, d)) < 0.5, x, np.float32(0))
        x = x - delta
    gpu = lambda a: None if a is None else torch.from_numpy(a).to("cuda:0")
    q, s = torch.empty((rows, d), dtype=torch.int8, device="cuda:0"), torch.empty(rows, device="cuda:0")
    binding.tabed_norm_q8(gpu(x), q, s, delta=gpu(delta))
    whole = x if delta is None else x + delta
    want = np.rint(whole / scale)
    assert np.abs(want).max() == 127 and np.array_equal(s.cpu().numpy(), scale[:, 0])
    assert np.array_equal(q.cpu().numpy(), want.astype(np.int8))

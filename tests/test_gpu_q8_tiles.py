"""tabed_linear_q8 and the 8-bit LM head in every tile that sizes choose between (rows, columns, waves that share K, stages of W and of X): odd numbers of
rows and columns, K of one k-block to more than there are stages, both ways tiles are dealt out, both output types."""
import ctypes as C

import pytest
import torch

import test_gpu_q8_step as step
from paper_2601_20357_amd import binding

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tile(M, N, K, head=False):
    t = (C.c_int32 * 5)()
    assert binding.load().tabed_testing_linear_tile(M, N, K, int(head), t) == 0
    return tuple(t)


T32, T32x64, T64, T64_deep, T64x128 = (32, 32, 8, 2, 2), (32, 64, 4, 3, 3), (64, 64, 2, 2, 2), (64, 64, 2, 3, 3), (64, 128, 1, 3, 3)
T128, T128x256, T256 = (128, 128, 1, 4, 4), (128, 256, 1, 3, 3), (256, 256, 1, 3, 2)
SHORT = [16, 112, 144, 256, 400, 512, 656, 1008]         # of 128 bytes: one to eight k-blocks, whole and ragged
# (tile, rows, columns, lengths of K)
SIZES = [(T32, 61, 333, [16, 1008, 1040, 2064, 4112]), (T32, 250, 61, [1024, 3088]), (T32x64, 41, 8011, [16, 496, 528, 1040, 1552, 2576]),
         (T32x64, 31, 17001, [4112, 5648]), (T64, 63, 16999, SHORT), (T64, 7, 33333, [1040, 2064]), (T64_deep, 191, 4999, SHORT + [2064]), (T64_deep, 37, 8300, [256, 784]),
         (T64x128, 29, 20021, SHORT), (T64x128, 127, 12011, SHORT), (T128, 999, 4001, SHORT + [2064]), (T128, 65, 20001, [16, 656, 2064]),
         (T128x256, 1499, 4099, SHORT), (T256, 385, 20002, SHORT + [2064]), (T128x256, 71, 50003, [400, 528]), (T256, 1500, 8201, SHORT + [2064]), (T128x256, 257, 33007, SHORT + [2064]),
         (T256, 1000, 9001, [4112])]
CASES = [(t, M, N, K) for t, M, N, Ks in SIZES for K in Ks]


@pytest.mark.parametrize("want,M,N,K", CASES)
def test_products_in_every_tile(want, M, N, K):
    """Scales are powers of two: one rounding of an exact integer, and that of the type."""
    assert tile(M, N, K) == want
    g = torch.Generator(device=DEV).manual_seed(M * N + K)
    x, w = (torch.randint(-128, 128, s, generator=g, dtype=torch.int8, device=DEV) for s in ((M, K), (N, K)))
    sx, sw = (2.0 ** torch.randint(-9, 10, (n,), generator=g, device=DEV) for n in (M, N))
    wide = torch.full((M, K + 48), 99, dtype=torch.int8, device=DEV)
    wide[:, :K] = x
    exact = (x.double() @ w.double().t()).float() * sx[:, None] * sw[None, :]
    for dtype in (torch.float32, torch.bfloat16):
        for pad in (0, 32 - N % 32):                                   # rows that begin anywhere, or on 64 bytes
            y = torch.full((M + 1, N + pad), 7.0, dtype=dtype, device=DEV)
            binding.tabed_linear_q8(wide[:, :K] if pad else x, sx, w, sw, y[:M, :N])
            assert torch.equal(y[:M, :N], exact.to(dtype)), (dtype, pad)
            assert (y[M] == 7).all() and (y[:, N:] == 7).all(), (dtype, pad)


# n B rows, V entries; rows of V with V % 16 = 0 and few logits go past L2, others through it
HEADS = [(T32, 4, 5, 1001, 256), (T32x64, 5, 7, 8011, 656), (T32x64, 3, 9, 17001, 4112), (T64, 3, 21, 20003, 1040), (T64x128, 3, 21, 20003, 1008), (T64_deep, 5, 25, 5003, 784),
         (T64x128, 5, 25, 12011, 400), (T128, 9, 111, 4001, 656), (T128, 5, 13, 20000, 1040), (T256, 7, 55, 20002, 400), (T256, 7, 55, 20000, 144), (T256, 15, 100, 8201, 656),
         (T128x256, 4, 64, 32016, 272), (T256, 3, 43, 33007, 1040), (T128x256, 1, 71, 50004, 528)]


@pytest.mark.parametrize("want,n,B,V,d", HEADS)
def test_lm_head_in_every_tile(want, n, B, V, d):
    assert tile(n * B, V, d, head=True) == want
    step.test_draft_step_q8_is_the_bf16_step_where_that_is_exact(n, B, V, d)

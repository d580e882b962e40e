"""The products in 8 bits in their steady state (fp8_shapes.py), and the experts' over enough blocks that every ring of stages is filled
again several times.  Tolerances: those of test_gpu_fp8.py and test_gpu_fp8_sizes.py."""
import pytest
import torch

import test_gpu_fp8_sizes as sizes
from fp8_shapes import LONG, SHORT
from test_gpu_fp8 import check_moe

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("out", DTYPES)
@pytest.mark.parametrize("M,N,K", SHORT + LONG)
def test_product(M, N, K, out):
    sizes.test_product(M, N, K, out)


# few tokens and many, few rows of inner features a use and enough for waves that share x: long reductions of the first product, then of
# the second
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,I,E,n", [(4, 1000, 2048, 16, 4), (16, 1000, 2048, 16, 4), (40, 1000, 2048, 16, 3), (4, 2100, 300, 8, 2), (9, 2100, 300, 8, 2),
                                       (40, 2103, 300, 8, 2), (3, 2000, 1000, 12, 4), (16, 2000, 1000, 12, 4), (40, 2000, 1001, 12, 4), (1, 2000, 1500, 9, 6),
                                       (1, 2000, 1700, 12, 8)])
def test_experts(T, H, I, E, n, dtype):
    check_moe(T, H, I, E, n, dtype)


# the same with 96 MB of weights and more
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,I,E,n", [(4, 1100, 2100, 16, 4), (16, 1100, 2100, 16, 4), (40, 1100, 2048, 16, 3), (64, 1111, 2100, 15, 5)])
def test_experts_of_many_bytes(T, H, I, E, n, dtype):
    sizes.test_experts_of_many_bytes(T, H, I, E, n, dtype)

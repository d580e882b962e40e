"""A row's norm does not depend on how many rows there are: the same bits from every kernel that takes a width."""
import pytest
import torch

import paper_1905_10138_amd as xe
from test_gpu_fp8 import DEV, gen, normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("cols", [5, 500, 513, 600, 1024, 1025, 1300, 1537, 2000, 2049, 4000, 4097, 6001, 6145, 8191, 8193, 9000, 10241, 12000, 12289, 14337, 16384,
                                  16400])
def test_norm_of_many_rows_is_that_of_each(cols, residual, dtype):
    g = gen(cols)
    x, r = normal(g, 515, cols, dtype=dtype).to(DEV), normal(g, 515, cols, dtype=dtype).to(DEV) if residual else None
    w = normal(g, cols).to(DEV)
    whole = xe.add_rmsnorm_fp8(x, w, r, normed=True)
    for rows in (slice(500, 515), slice(514, 515), slice(0, 512)):
        part = xe.add_rmsnorm_fp8(x[rows], w, r[rows] if residual else None, normed=True)
        for a, b in zip(whole, part):
            assert (a is None and b is None) or torch.equal(a[rows].float(), b.float())

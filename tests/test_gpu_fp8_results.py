"""What the calls on 8-bit matrices return, as tensors."""
import io

import pytest
import torch

import paper_1905_10138_amd as xe
import fp8_oracle as ref
from test_gpu_fp8 import DEV, gen, normal

pytestmark = pytest.mark.gpu


# few rows and many: results are tensors of their own, that are saved together, and without what else the call returned
@pytest.mark.parametrize("rows", [1, 40, 3000])
def test_results_can_be_saved(rows):
    g = gen(rows)
    x, r, w = normal(g, rows, 600, dtype=torch.bfloat16).to(DEV), normal(g, rows, 600, dtype=torch.bfloat16).to(DEV), normal(g, 600).to(DEV)
    for got in (xe.quant_fp8(x), xe.quant_fp8(x, block_rows=128), xe.quant_fp8(x[None], block_rows=128), xe.silu_mul_fp8(x),
                xe.add_rmsnorm_fp8(x, w, r, normed=True)):
        file = io.BytesIO()
        torch.save(got, file)
        file.seek(0)
        back = torch.load(file, weights_only=True)
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, back))
        assert len({t.untyped_storage().data_ptr() for t in got}) == len(got)
        for t in got:
            assert t.untyped_storage().nbytes() < t.element_size() * (t.numel() + 16 * rows)
            file = io.BytesIO()
            torch.save(t, file)
            assert len(file.getvalue()) < t.untyped_storage().nbytes() + 4096


def test_normed_rows_that_overlap_are_refused():
    x, w = torch.ones((4, 600), device=DEV), torch.ones(600, device=DEV)
    one = torch.zeros(600 * 4, device=DEV)
    for normed in (one[:600].expand(4, 600), one.as_strided((4, 600), (1, 1)), one.as_strided((4, 600), (599, 1))):
        with pytest.raises(xe.XorencError):
            xe.add_rmsnorm_fp8(x, w, normed=normed)
    assert not one.any()
    for normed in (one[:600].expand(1, 600), one.as_strided((4, 600), (600, 1)), one.as_strided((4, 600), (1, 4))):
        assert torch.equal(xe.add_rmsnorm_fp8(x[:normed.shape[0]], w, normed=normed)[3], xe.add_rmsnorm_fp8(x[:normed.shape[0]], w, normed=True)[3])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T", [1, 3, 5])
def test_logits_of_either_zero_are_equal(T, dtype):
    # products of -1e-60 round to -0, and a sum of them is -0: no less than the 0 of the next expert
    g = gen(T)
    E, H, I = 3, 2048, 40
    x = torch.full((T, H), 1e-30, dtype=dtype, device=DEV)
    W13, S13 = xe.quant_fp8(normal(g, E, 2 * I, H, scale=1e29).to(DEV), block_rows=128)
    W2, S2 = xe.quant_fp8(normal(g, E, H, I).to(DEV), block_rows=128)
    for signs in ((-1.0, 0.0), (0.0, -1.0), (0.0, 0.0), (-1.0, -1.0)):
        router = torch.full((E, H), -1e30, dtype=dtype, device=DEV)
        router[0], router[1] = signs[0] * 1e-30, signs[1] * 1e-30
        Y = xe.moe_fp8(x, router, W13, S13, W2, S2, 1)
        router[:2] = 0.0
        router[1] = -1e30                                                # the first alone
        assert Y.any() and torch.equal(Y, xe.moe_fp8(x, router, W13, S13, W2, S2, 1)), signs


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_gates_whose_logistic_is_subnormal(dtype):
    # 1 / (1 + exp(88)) is 6.1e-39, below the normal numbers of fp32, and 88 times that is none of them; up to exp(-x) = 2^128
    x = torch.cat([-torch.linspace(84.0, 88.7, 512), torch.full((512,), 1e30)]).to(dtype).reshape(1, -1)
    Q, S = xe.silu_mul_fp8(x.to(DEV))
    # as test_gate of test_gpu_fp8.py has it for the exponential's argument (and 2^-26 of it for the constant), and half of a subnormal's
    # last bit: 2^-150 of 2^-128
    ref.check_quantised(ref.silu_mul(x), Q, S, 1, 89 * (2.0 ** -24 + 2.0 ** -26) + 8 * 2.0 ** -24 + 2.0 ** -22)

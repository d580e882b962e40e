"""Operators that end in 8-bit rows: every width at which the work is split another way, and rows that start on any element.
Tolerances: those of test_gpu_fp8.py."""
import pytest
import torch

import paper_1905_10138_amd as xe
import fp8_oracle as ref
from test_gpu_fp8 import DEV, U, gen, normal

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("cols", [2, 7, 9, 511, 513, 1024, 1025, 1535, 1537, 2047, 2049, 4097, 6145, 8191, 8193, 10239, 10241, 12289, 16383, 16385])
def test_norm(cols, residual, dtype):
    g = gen(cols)
    x, r = normal(g, 5, cols, dtype=dtype), normal(g, 5, cols, dtype=dtype) if residual else None
    w = normal(g, cols, dtype=dtype)
    Q, S, total, y = xe.add_rmsnorm_fp8(x.to(DEV), w.to(DEV), r.to(DEV) if residual else None, normed=True)
    t, want = ref.rmsnorm(x, r, w, 1e-6)
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0
    # the sum of squares in a tree: its relative error halves in the root; a handful of roundings beside it
    rel = (2.0 * torch.log2(torch.tensor(float(max(cols, 2)))).item() + 16) * U
    assert ((y.cpu().double() - want).abs() <= (half + rel) * want.abs() + 1e-30).all()
    if residual:
        assert ((total.cpu().double() - t).abs() <= (half + U) * t.abs()).all()
    ref.check_quantised(want, Q, S, 1, rel)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [1, 3, 7, 8, 9, 15, 17, 127, 129, 1000, 1537, 5001])
@pytest.mark.parametrize("start", [0, 1, 3])
def test_rows_that_start_anywhere(cols, start, dtype):
    g = gen(cols + start)
    wide = torch.full((135, 2 * cols + 9), float("nan"), dtype=dtype, device=DEV)
    wide[:, start:start + 2 * cols] = normal(g, 135, 2 * cols, dtype=dtype).to(DEV)
    x, pair = wide[:, start:start + cols], wide[:, start:start + 2 * cols]
    res = wide[:, start + cols:start + 2 * cols]
    w = normal(g, cols + 1, dtype=dtype).to(DEV)[1:]

    def aligned(t):
        out = torch.empty((t.shape[0], -(-t.shape[1] // 16) * 16), dtype=dtype, device=DEV)[:, :t.shape[1]]
        return out.copy_(t)
    for got, want in ((xe.quant_fp8(x), xe.quant_fp8(aligned(x))),
                      (xe.quant_fp8(x, block_rows=128), xe.quant_fp8(aligned(x), block_rows=128)),
                      (xe.silu_mul_fp8(pair), xe.silu_mul_fp8(aligned(pair)))):
        assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
    big = torch.full((137, cols + 3), 9.0, dtype=dtype, device=DEV)
    got = xe.add_rmsnorm_fp8(x, w, res, total=big[1:136, 1:1 + cols], normed=True)
    want = xe.add_rmsnorm_fp8(aligned(x), w.clone(), aligned(res), normed=True)
    assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want))
    big[1:136, 1:1 + cols] = 9.0
    assert (big == 9.0).all()                                            # and nothing beside it
    ref.check_quantised(x.cpu().double(), *xe.quant_fp8(x), 1, 0.0)
    ref.check_quantised(x.cpu().double(), *xe.quant_fp8(x, block_rows=128), 128, 0.0)


# more than 256 MB are read another way: the same values
@pytest.mark.parametrize("dtype,rows,cols", [(torch.bfloat16, 20000, 5003), (torch.float32, 9000, 8000)])
def test_many_rows(dtype, rows, cols):
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn((rows, cols), generator=g, device=DEV).to(dtype)
    r = torch.randn((rows, cols), generator=g, device=DEV).to(dtype)
    w = torch.randn(cols, generator=g, device=DEV)
    both = torch.randn((rows, 2 * cols), generator=g, device=DEV).to(dtype)
    part = slice(128 * 50, 128 * 51)
    for f, rest in ((lambda s: xe.add_rmsnorm_fp8(x[s], w, r[s], normed=True), 0), (lambda s: xe.silu_mul_fp8(both[s]), 0),
                    (lambda s: xe.quant_fp8(both[s]), 0), (lambda s: xe.quant_fp8(both[s], block_rows=128), 1)):
        whole, some = f(slice(None)), f(part)
        assert torch.equal(whole[0][part].float(), some[0].float())
        assert torch.equal(whole[1][50:51] if rest else whole[1][part], some[1])
        if len(whole) == 4:
            assert torch.equal(whole[2][part], some[2]) and torch.equal(whole[3][part], some[3])


# up to 512 rows and beyond: a row's threads, or several rows a workgroup
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("cols", [600, 1300, 2000, 4000, 6001, 9000, 12000])
def test_norm_of_many_rows_is_that_of_each(cols, dtype):
    g = gen(cols)
    x, r = normal(g, 515, cols, dtype=dtype).to(DEV), normal(g, 515, cols, dtype=dtype).to(DEV)
    w = normal(g, cols).to(DEV)
    whole = xe.add_rmsnorm_fp8(x, w, r, normed=True)
    part = xe.add_rmsnorm_fp8(x[500:], w, r[500:], normed=True)
    # two orders of the sum of squares: both within the tolerance of the definition
    _, want = ref.rmsnorm(x[500:].cpu(), r[500:].cpu(), w.cpu(), 1e-6)
    half = 2.0 ** -8 if dtype is torch.bfloat16 else 0.0
    for out in ([t[500:] for t in whole], part):
        assert torch.equal(out[2], (x[500:].float() + r[500:].float()).to(dtype))
        assert ((out[3].cpu().double() - want).abs() <= (half + 40 * U) * want.abs() + 1e-30).all()
        ref.check_quantised(want, out[0], out[1], 1, 40 * U)

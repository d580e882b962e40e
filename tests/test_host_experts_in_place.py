"""A residual that is Y itself has Y's rows: with another leading dimension its rows would lie across those that are written.  Refused before any GPU
call, so no GPU is needed, and no pointer is followed."""
import pytest

from paper_1905_10138_amd import fp8
from test_host_experts import epilogue
from test_host_fp8 import BF16, EINVAL, F32, P, with_changes


@pytest.fixture(scope="module")
def lib():
    return fp8._library()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_combine_onto_the_residual(lib, dtype):
    good = dict(R=P, dt=dtype, ldr=256, pl=P, used=P, sh=P, r=P + 4096, ld=300, T=4, n=2, cols=256, Y=P + 4096, ldy=300, st=None)
    with_changes(lib.xorenc_combine_tokens, good, [({"ld": 256}, EINVAL), ({"ldy": 256}, EINVAL), ({"T": 2, "ld": 1 << 20}, EINVAL)])


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_product_onto_the_residual(lib, dtype):
    good = dict(A=P, lda=256, SA=P, sar=1, sab=4, W=P, ldw=256, SW=P, ldsw=2, M=4, N=128, K=256, e=None, Y=P + 4096, dt=dtype, ldy=160, st=None)
    with_changes(lib.xorenc_linear_fp8, good, [
        ({"e": epilogue(residual=P + 4096, ld=128)}, EINVAL), ({"e": epilogue(bias=None, residual=P + 4096, ld=128)}, EINVAL),
        ({"e": epilogue(residual=P + 4096, ld=161), "M": 2}, EINVAL), ({"e": epilogue(residual=P + 4096, ld=160), "ldy": 128}, EINVAL)])

"""What else the C ABI of the operators in 8 bits refuses, and what it does not (see test_host_fp8.py): no GPU is needed, and no pointer is
followed.  A call whose sizes are accepted is stopped by a later check, of an address that is not aligned, before any launch."""
import pytest

from paper_1905_10138_amd import fp8
from test_host_fp8 import BF16, EALIGN, EINVAL, ELIMIT, F32, P, layer, with_changes

QUANT = dict(X=P, dt=BF16, ldx=256, xs=0, n=1, rows=4, cols=256, br=1, Q=P, ldq=256, qs=0, S=P, sr=1, sb=4, ss=0, st=None)
NORM = dict(X=P, dt=BF16, ldx=256, R=P, ldr=256, w=P, wdt=F32, rows=4, cols=256, eps=1e-6, t=P, ldt=256, Y=P, yr=256, yc=1, Q=P, ldq=256,
            S=P, sr=1, sb=4, st=None)
GATE = dict(g=P, u=P, dt=F32, ldx=512, rows=4, cols=256, Q=P, ldq=256, S=P, sr=1, sb=4, st=None)


@pytest.fixture(scope="module")
def lib():
    return fp8._library()


def test_results_whose_elements_are_one(lib):
    stack = dict(n=2, rows=130, br=128, qs=65536, ss=8, sb=2)
    with_changes(lib.xorenc_quant_fp8, QUANT, [
        ({"sr": 0}, EINVAL), ({"sb": 0}, EINVAL), ({"sr": 1, "sb": 3}, EINVAL), ({"sr": 2, "sb": 6}, EINVAL),
        ({**stack, "qs": 0}, EINVAL), ({**stack, "ss": 0}, EINVAL), ({**stack, "sb": 1}, EINVAL)])
    with_changes(lib.xorenc_silu_mul_fp8, GATE, [({"sr": 0}, EINVAL), ({"sb": 0}, EINVAL), ({"sr": 1, "sb": 1}, EINVAL)])
    with_changes(lib.xorenc_add_rmsnorm_fp8, NORM, [
        ({"sr": 0}, EINVAL), ({"yr": 0}, EINVAL), ({"yr": 255}, EINVAL), ({"yr": 1, "yc": 3}, EINVAL), ({"yr": 2, "yc": 4}, EINVAL)])


def test_rows_whose_blocks_exceed_64_bits(lib):
    # 2^57 + 1 rows of 128 blocks are 2^64 + 128 blocks
    wide = dict(rows=(1 << 57) + 1, cols=16384, ldx=16384, ldq=16384)
    with_changes(lib.xorenc_quant_fp8, QUANT, [({**wide, "X": P + 1}, ELIMIT), ({**wide, "rows": (1 << 63) - 1, "br": 128, "X": P}, ELIMIT)])
    with_changes(lib.xorenc_silu_mul_fp8, GATE, [({**wide, "u": P + 2}, ELIMIT)])
    with_changes(lib.xorenc_add_rmsnorm_fp8, NORM, [({**wide, "ldr": 16384, "ldt": 16384, "yr": 16384, "X": P + 1}, ELIMIT)])


def test_squares_have_their_own_limit(lib):
    # 2^21 x 2^14 is 2^28 blocks of 1 x 128, and 2^21 of 128 x 128; 2^24 of those are too many
    tall = dict(br=128, cols=16384, ldx=16384, ldq=16384, sr=128, sb=1)
    with_changes(lib.xorenc_quant_fp8, QUANT, [
        ({**tall, "rows": 1 << 21, "X": P + 1}, EALIGN), ({**tall, "rows": (1 << 24) - 128, "X": P + 1}, EALIGN), ({**tall, "rows": 1 << 24}, ELIMIT),
        ({**tall, "rows": 1 << 21, "br": 1}, ELIMIT), ({**tall, "rows": (1 << 21) - 1, "br": 1, "X": P + 1}, EALIGN)])


def test_strides_of_products(lib):
    good = dict(A=P, lda=256, SA=P, sar=1, sab=4, W=P, ldw=256, SW=P, ldsw=2, M=4, N=128, K=256, Y=P, dt=BF16, ldy=128, st=None)
    with_changes(lib.xorenc_matmul_fp8, good, [
        ({"lda": (1 << 22) + 16}, ELIMIT), ({"ldw": (1 << 22) + 16}, ELIMIT), ({"sar": (1 << 20) + 1}, ELIMIT), ({"sab": (1 << 28) + 1, "K": 128}, ELIMIT),
        ({"sar": 1 << 20, "sab": 1 << 27}, ELIMIT), ({"M": 1 << 20, "N": 1 << 20, "lda": 256, "ldy": 1 << 20}, ELIMIT)])


def test_strides_of_experts(lib):
    good = dict(L=layer(), X=P, dt=BF16, ldx=256, T=4, n=2, re=1, Y=P, ldy=256, ws=P, wsb=1 << 30, st=None)
    with_changes(lib.xorenc_moe_fp8, good, [
        ({"L": layer(ld13=(1 << 24) + 16)}, ELIMIT), ({"L": layer(ld2=(1 << 24) + 16)}, ELIMIT), ({"L": layer(lds13=(1 << 16) + 1)}, ELIMIT),
        ({"L": layer(lds2=(1 << 16) + 1)}, ELIMIT), ({"L": layer(ld13=1 << 24, ld2=1 << 24, lds13=1 << 16, lds2=1 << 16), "ws": P + 4}, EALIGN)])

"""What the C ABI of the operators in 8 bits refuses, before any GPU call: no GPU is needed, and no pointer is followed."""
import ctypes

import pytest

import paper_1905_10138_amd as xe
from paper_1905_10138_amd import fp8

P = 1 << 20  # an aligned address that nothing reads
EINVAL, EUNSUPPORTED, EALIGN, ELIMIT = -1, -2, -3, -6
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    return fp8._library()


def with_changes(call, good, changes):
    for change, code in changes:
        args = dict(good)
        args.update(change)
        assert call(*args.values()) == code, change


def test_quant(lib):
    good = dict(X=P, dt=BF16, ldx=256, xs=0, n=1, rows=4, cols=256, br=1, Q=P, ldq=256, qs=0, S=P, sr=1, sb=4, ss=0, st=None)
    with_changes(lib.xorenc_quant_fp8, good, [
        ({"X": None}, EINVAL), ({"Q": None}, EINVAL), ({"S": None}, EINVAL), ({"rows": -1}, EINVAL), ({"cols": 0}, EINVAL),
        ({"ldx": 255}, EINVAL), ({"ldq": 255}, EINVAL), ({"n": -1}, EINVAL), ({"sr": -1}, EINVAL), ({"n": 2, "xs": -1}, EINVAL),
        ({"dt": 2}, EUNSUPPORTED), ({"br": 2}, EUNSUPPORTED), ({"br": 0}, EUNSUPPORTED), ({"Q": P + 8}, EALIGN), ({"ldq": 264}, EALIGN),
        ({"X": P + 1}, EALIGN), ({"S": P + 2}, EALIGN), ({"n": 2, "qs": 8}, EALIGN), ({"rows": 1 << 40}, ELIMIT),
        ({"br": 128, "rows": 1 << 31}, ELIMIT), ({"rows": 0}, 0), ({"n": 0}, 0), ({"rows": 0, "X": None}, 0)])


def test_norm(lib):
    good = dict(X=P, dt=BF16, ldx=256, R=P, ldr=256, w=P, wdt=F32, rows=4, cols=256, eps=1e-6, t=P, ldt=256, Y=P, yr=256, yc=1, Q=P, ldq=256,
                S=P, sr=1, sb=4, st=None)
    with_changes(lib.xorenc_add_rmsnorm_fp8, good, [
        ({"X": None}, EINVAL), ({"w": None}, EINVAL), ({"Q": None}, EINVAL), ({"ldr": 1}, EINVAL), ({"ldt": 1}, EINVAL), ({"yc": 0}, EINVAL),
        ({"eps": -1.0}, EINVAL), ({"eps": float("nan")}, EINVAL), ({"dt": 7}, EUNSUPPORTED), ({"wdt": -1}, EUNSUPPORTED), ({"R": P + 1}, EALIGN),
        ({"t": P + 1}, EALIGN), ({"Y": P + 1}, EALIGN), ({"w": P + 2}, EALIGN), ({"rows": 1 << 22}, ELIMIT), ({"rows": 0}, 0)])


def test_gate(lib):
    good = dict(g=P, u=P, dt=F32, ldx=512, rows=4, cols=256, Q=P, ldq=256, S=P, sr=1, sb=4, st=None)
    with_changes(lib.xorenc_silu_mul_fp8, good, [
        ({"g": None}, EINVAL), ({"u": None}, EINVAL), ({"ldx": 2}, EINVAL), ({"dt": 3}, EUNSUPPORTED), ({"u": P + 2}, EALIGN), ({"rows": 0}, 0)])


def test_product(lib):
    good = dict(A=P, lda=256, SA=P, sar=1, sab=4, W=P, ldw=256, SW=P, ldsw=2, M=4, N=128, K=256, Y=P, dt=BF16, ldy=128, st=None)
    with_changes(lib.xorenc_matmul_fp8, good, [
        ({"A": None}, EINVAL), ({"SA": None}, EINVAL), ({"W": None}, EINVAL), ({"SW": None}, EINVAL), ({"Y": None}, EINVAL), ({"M": -1}, EINVAL),
        ({"N": 0}, EINVAL), ({"K": 0}, EINVAL), ({"lda": 240}, EINVAL), ({"ldw": 240}, EINVAL), ({"ldy": 127}, EINVAL), ({"ldsw": 1}, EINVAL),
        ({"sar": -1}, EINVAL), ({"dt": 9}, EUNSUPPORTED), ({"A": P + 1}, EALIGN), ({"lda": 260}, EALIGN), ({"W": P + 8}, EALIGN),
        ({"ldw": 264}, EALIGN), ({"Y": P + 1}, EALIGN), ({"SA": P + 1}, EALIGN), ({"M": 65535 * 64 + 1}, ELIMIT),
        ({"K": (1 << 24) + 1, "lda": 1 << 25, "ldw": 1 << 25, "ldsw": 1 << 18}, ELIMIT), ({"M": 0}, 0)])


def layer(**change):
    f = dict(size=fp8._MOE_BYTES, E=8, H=256, I=128, router=P, ldr=256, W13=P, ld13=256, st13=65536, S13=P, lds13=2, ss13=4, W2=P, ld2=128, st2=32768,
             S2=P, lds2=1, ss2=2)
    f.update(change)
    f = {k: 0 if v is None else v for k, v in f.items()}
    return fp8._pack_moe(*f.values())


def test_moe(lib):
    need = ctypes.c_int64()
    assert lib.xorenc_moe_workspace(4, 256, 128, 8, 2, BF16, ctypes.byref(need)) == 0 and need.value > 0
    assert lib.xorenc_moe_workspace(4, 256, 128, 8, 2, BF16, None) == EINVAL
    assert lib.xorenc_moe_workspace(65, 256, 128, 8, 2, BF16, ctypes.byref(need)) == ELIMIT
    assert lib.xorenc_moe_workspace(4, 256, 128, 257, 2, BF16, ctypes.byref(need)) == ELIMIT
    assert lib.xorenc_moe_workspace(4, 256, 128, 64, 17, BF16, ctypes.byref(need)) == ELIMIT
    assert lib.xorenc_moe_workspace(4, 256, 128, 8, 9, BF16, ctypes.byref(need)) == EINVAL
    assert lib.xorenc_moe_workspace(4, 256, 128, 8, 2, 2, ctypes.byref(need)) == EUNSUPPORTED
    good = dict(L=layer(), X=P, dt=BF16, ldx=256, T=4, n=2, re=1, Y=P, ldy=256, ws=P, wsb=1 << 30, st=None)
    with_changes(lib.xorenc_moe_fp8, good, [
        ({"L": None}, EINVAL), ({"L": layer(size=64)}, EINVAL), ({"L": layer(router=None)}, EINVAL), ({"L": layer(W2=None)}, EINVAL),
        ({"L": layer(ld13=240)}, EINVAL), ({"L": layer(lds13=1)}, EINVAL), ({"L": layer(st2=-16)}, EINVAL), ({"L": layer(E=0)}, EINVAL),
        ({"L": layer(E=300)}, ELIMIT), ({"L": layer(W13=P + 8)}, EALIGN), ({"L": layer(st13=8)}, EALIGN), ({"L": layer(router=P + 1)}, EALIGN),
        ({"X": None}, EINVAL), ({"Y": None}, EINVAL), ({"ws": None}, EINVAL), ({"wsb": 64}, EINVAL), ({"ws": P + 4}, EALIGN), ({"ldx": 200}, EINVAL),
        ({"n": 0}, EINVAL), ({"n": 9}, EINVAL), ({"T": 65}, ELIMIT), ({"T": -1}, EINVAL), ({"dt": 5}, EUNSUPPORTED), ({"T": 0}, 0)])


def test_limits_of_the_header():
    with open(xe.library_path().replace("paper_1905_10138_amd/libxorenc.so", "include/xorenc.h")) as f:
        text = f.read()
    for name, value in (("XORENC_FP8_BLOCK", xe.FP8_BLOCK), ("XORENC_MOE_MAX_TOKENS", xe.MOE_MAX_TOKENS),
                        ("XORENC_MOE_MAX_EXPERTS", xe.MOE_MAX_EXPERTS), ("XORENC_MOE_MAX_PICKS", xe.MOE_MAX_PICKS)):
        assert f"#define {name} {value}\n" in text

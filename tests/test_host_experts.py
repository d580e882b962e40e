"""What the C ABI of sorted tokens and of products with an epilogue refuses, before any GPU call: no GPU is needed, and no pointer is followed."""
import ctypes
import struct

import pytest

import paper_1905_10138_amd as xe
from paper_1905_10138_amd import fp8
from test_host_fp8 import BF16, EALIGN, EINVAL, ELIMIT, EUNSUPPORTED, F32, P, with_changes

I32, I64 = 0, 1
BIG = 1 << 40


@pytest.fixture(scope="module")
def lib():
    return fp8._library()


def test_pick(lib):
    good = dict(l=P, dt=BF16, ldl=64, T=4, E=64, n=6, re=1, ids=P, sh=P, st=None)
    with_changes(lib.xorenc_pick_experts, good, [
        ({"l": None}, EINVAL), ({"ids": None}, EINVAL), ({"sh": None}, EINVAL), ({"ldl": 63}, EINVAL), ({"T": -1}, EINVAL), ({"E": 0}, EINVAL),
        ({"n": 0}, EINVAL), ({"n": 65}, EINVAL), ({"n": 17}, ELIMIT), ({"E": 257, "ldl": 257}, ELIMIT), ({"T": 1 << 24}, ELIMIT),
        ({"T": (1 << 24) // 6 + 1}, ELIMIT), ({"dt": 2}, EUNSUPPORTED), ({"l": P + 1}, EALIGN), ({"dt": F32, "l": P + 2}, EALIGN),
        ({"ids": P + 2}, EALIGN), ({"sh": P + 1}, EALIGN), ({"T": 0}, 0), ({"T": 0, "l": None}, 0)])


def test_sort(lib):
    need = ctypes.c_int64(-1)
    call = lib.xorenc_sort_tokens_workspace
    assert call(0, 2, 8, ctypes.byref(need)) == 0 and need.value == 0
    assert call(4, 2, 8, ctypes.byref(need)) == 0 and need.value == 0
    assert call(100000, 8, 256, ctypes.byref(need)) == 0 and need.value > 0
    assert call(4, 2, 8, None) == EINVAL
    for sizes, code in (((-1, 2, 8), EINVAL), ((4, 0, 8), EINVAL), ((4, 2, 0), EINVAL), ((4, 17, 20), ELIMIT), ((4, 2, 257), ELIMIT), ((1 << 24, 1, 8), ELIMIT)):
        assert call(*sizes, ctypes.byref(need)) == code
    good = dict(ids=P, it=I32, T=100000, n=8, E=8, pl=P, rows=P, off=P, ws=P, wsb=1 << 30, st=None)
    with_changes(lib.xorenc_sort_tokens, good, [
        ({"ids": None}, EINVAL), ({"pl": None}, EINVAL), ({"off": None}, EINVAL), ({"ws": None}, EINVAL), ({"wsb": 64}, EINVAL), ({"it": 2}, EUNSUPPORTED),
        ({"ids": P + 2}, EALIGN), ({"it": I64, "ids": P + 4}, EALIGN), ({"pl": P + 2}, EALIGN), ({"rows": P + 2}, EALIGN), ({"off": P + 1}, EALIGN),
        ({"ws": P + 2}, EALIGN), ({"n": 17}, ELIMIT), ({"E": 300}, ELIMIT), ({"T": 0, "off": None}, EINVAL)])


ROWS = [({"T": -1}, EINVAL), ({"n": 0}, EINVAL), ({"cols": 0}, EINVAL), ({"pl": None}, EINVAL), ({"used": None}, EINVAL), ({"dt": 3}, EUNSUPPORTED),
        ({"n": 17}, ELIMIT), ({"T": 1 << 23}, ELIMIT), ({"cols": (1 << 20) + 1, "ldx": BIG, "ldr": BIG, "ldy": BIG, "ld": BIG}, ELIMIT),
        ({"T": 1 << 22, "cols": 1 << 13, "ldx": BIG, "ldr": BIG, "ldy": BIG, "ld": BIG}, ELIMIT), ({"pl": P + 2}, EALIGN), ({"used": P + 1}, EALIGN),
        ({"sh": P + 2}, EALIGN), ({"T": 0}, 0), ({"T": 0, "pl": None}, 0)]


def changes_of(good):
    return [({k: v for k, v in change.items() if k in good}, code) for change, code in ROWS]


def test_gather(lib):
    good = dict(X=P, dt=BF16, ldx=256, pl=P, used=P, sh=P, T=4, n=2, cols=256, R=P, ldr=256, st=None)
    with_changes(lib.xorenc_gather_tokens, good, changes_of(good) + [
        ({"X": None}, EINVAL), ({"R": None}, EINVAL), ({"ldx": 255}, EINVAL), ({"ldr": 255}, EINVAL), ({"X": P + 1}, EALIGN), ({"R": P + 1}, EALIGN)])


def test_combine(lib):
    good = dict(R=P, dt=F32, ldr=256, pl=P, used=P, sh=P, r=P, ld=256, T=4, n=2, cols=256, Y=P, ldy=256, st=None)
    with_changes(lib.xorenc_combine_tokens, good, changes_of(good) + [
        ({"R": None}, EINVAL), ({"Y": None}, EINVAL), ({"ldr": 255}, EINVAL), ({"ldy": 255}, EINVAL), ({"ld": 255}, EINVAL), ({"R": P + 2}, EALIGN),
        ({"Y": P + 1}, EALIGN), ({"r": P + 2}, EALIGN)])


def test_gradient(lib):
    good = dict(dY=P, dt=F32, ldy=256, R=P, ldr=256, pl=P, used=P, sh=P, T=4, n=2, cols=256, dR=P + 4096, ld=256, ds=P, st=None)
    with_changes(lib.xorenc_combine_tokens_grad, good, changes_of(good) + [
        ({"dY": None}, EINVAL), ({"R": None}, EINVAL), ({"sh": None}, EINVAL), ({"dR": None}, EINVAL), ({"ds": None}, EINVAL), ({"ldr": 255}, EINVAL),
        ({"ldy": 255}, EINVAL), ({"ld": 255}, EINVAL), ({"dR": P, "ld": 300}, EINVAL), ({"dR": P + 2}, EALIGN), ({"ds": P + 2}, EALIGN)])


def epilogue(size=None, act=0, bias=P, bdt=F32, stride=128, residual=None, ld=128):
    fmt = "IiPiqPq"
    return struct.pack(fmt, struct.calcsize(fmt) if size is None else size, act, bias or 0, bdt, stride, residual or 0, ld)


EPILOGUES = [({"e": epilogue(size=8)}, EINVAL), ({"e": epilogue(act=5)}, EUNSUPPORTED), ({"e": epilogue(act=-1)}, EUNSUPPORTED),
             ({"e": epilogue(bdt=2)}, EUNSUPPORTED), ({"e": epilogue(bias=P + 2)}, EALIGN), ({"e": epilogue(bias=P + 1, bdt=BF16)}, EALIGN)]


def test_product_with_epilogue(lib):
    good = dict(A=P, lda=256, SA=P, sar=1, sab=4, W=P, ldw=256, SW=P, ldsw=2, M=4, N=128, K=256, e=epilogue(residual=P), Y=P, dt=BF16, ldy=128, st=None)
    with_changes(lib.xorenc_linear_fp8, good, EPILOGUES + [
        ({"A": None}, EINVAL), ({"SW": None}, EINVAL), ({"Y": None}, EINVAL), ({"M": -1}, EINVAL), ({"ldy": 127}, EINVAL), ({"lda": 240}, EINVAL),
        ({"dt": 9}, EUNSUPPORTED), ({"W": P + 8}, EALIGN), ({"lda": 260}, EALIGN), ({"Y": P + 1}, EALIGN), ({"M": 65535 * 64 + 1}, ELIMIT),
        ({"e": epilogue(residual=P, ld=127)}, EINVAL), ({"e": epilogue(residual=P + 1)}, EALIGN), ({"dt": F32, "e": epilogue(residual=P + 2)}, EALIGN),
        ({"M": 0}, 0), ({"M": 0, "e": None}, 0)])


def test_products_of_experts(lib):
    good = dict(A=P, lda=256, SA=P, sar=1, sab=4, ar=4, rows=P, off=P, E=8, W=P, ldw=256, ws=32768, SW=P, ldsw=2, ss=2, N=128, K=256, e=epilogue(), Y=P,
                dt=BF16, ldy=128, yr=8, st=None)
    with_changes(lib.xorenc_experts_fp8, good, EPILOGUES + [
        ({"A": None}, EINVAL), ({"W": None}, EINVAL), ({"off": None}, EINVAL), ({"E": 0}, EINVAL), ({"ws": -16}, EINVAL), ({"ss": -1}, EINVAL),
        ({"rows": None}, EINVAL), ({"ar": -1}, EINVAL), ({"ar": 0}, EINVAL), ({"yr": -1}, EINVAL), ({"lda": 240}, EINVAL),
        ({"e": epilogue(residual=P)}, EINVAL), ({"e": epilogue(stride=-1)}, EINVAL), ({"ws": 8}, EALIGN), ({"off": P + 2}, EALIGN), ({"rows": P + 2}, EALIGN),
        ({"lda": 260}, EALIGN), ({"E": 257}, ELIMIT), ({"lda": 1 << 20, "ar": 1 << 11}, ELIMIT), ({"sar": 1 << 10, "ar": 1 << 19}, ELIMIT), ({"yr": 0}, 0)])


def test_the_extension_has_them():
    native = fp8._load()
    for name, count in (("pick", 3), ("sort", 2), ("gather", 5), ("combine", 6), ("combine_grad", 6), ("linear", 9), ("experts", 10)):
        with pytest.raises(TypeError, match=f"{count} arguments"):
            getattr(native, name)()


def test_they_are_public():
    for name in ("pick_experts", "sort_tokens", "gather_tokens", "combine_tokens", "combine_tokens_grad", "linear_fp8", "experts_fp8"):
        assert name in xe.__all__ and callable(getattr(xe, name))

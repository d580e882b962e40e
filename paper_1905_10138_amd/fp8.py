"""Dense layers in 8 bits: the calls of include/xorenc.h on e4m3 matrices with a scale per block of 128, argument marshalling only.

An 8-bit matrix is a pair of tensors: the values (torch.float8_e4m3fn, rows on 16-byte boundaries) and the scales (float32,
one for each 1 x 128 block of activations or 128 x 128 block of weights).  All tensors are on the current device, the
work goes to its current stream, and nothing waits.
"""
import ctypes
import struct

from .binding import X_BF16, X_F32, _check, _stream_ptr, load_library

FP8_BLOCK = 128
MOE_MAX_TOKENS, MOE_MAX_EXPERTS, MOE_MAX_PICKS = 64, 256, 16

_pack_moe = struct.Struct("I3iP q P2q P2q P2q P2q").pack
_MOE_BYTES = struct.calcsize("I3iP q P2q P2q P2q P2q")
_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = load_library()
        vp, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float
        lib.xorenc_quant_fp8.restype = i32
        lib.xorenc_quant_fp8.argtypes = [vp, i32, i64, i64, i32, i64, i32, i32, vp, i64, i64, vp, i64, i64, i64, vp]
        lib.xorenc_add_rmsnorm_fp8.restype = i32
        lib.xorenc_add_rmsnorm_fp8.argtypes = [vp, i32, i64, vp, i64, vp, i32, i64, i32, f32, vp, i64, vp, i64, i64, vp, i64,
                                               vp, i64, i64, vp]
        lib.xorenc_silu_mul_fp8.restype = i32
        lib.xorenc_silu_mul_fp8.argtypes = [vp, vp, i32, i64, i64, i32, vp, i64, vp, i64, i64, vp]
        lib.xorenc_matmul_fp8.restype = i32
        lib.xorenc_matmul_fp8.argtypes = [vp, i64, vp, i64, i64, vp, i64, vp, i64, i32, i32, i32, vp, i32, i64, vp]
        lib.xorenc_moe_workspace.restype = i32
        lib.xorenc_moe_workspace.argtypes = [i32, i32, i32, i32, i32, i32, vp]
        lib.xorenc_moe_fp8.restype = i32
        lib.xorenc_moe_fp8.argtypes = [ctypes.c_char_p, vp, i32, i64, i32, i32, i32, vp, i64, vp, i64, vp]
        _lib = lib
    return _lib


def _device():
    import torch
    return torch._C._cuda_getDevice()


def _dtype(t, what):
    import torch
    if t.dtype is torch.bfloat16:
        return X_BF16
    if t.dtype is torch.float32:
        return X_F32
    raise ValueError(f"{what} must be float32 or bfloat16")


def _rows(t, dims, what, device):
    """Checks a row-major matrix (or stack of matrices) on the current device; returns its leading dimension."""
    if t.dim() != dims:
        raise ValueError(f"{what} must have {dims} dimensions")
    if t.get_device() != device:
        raise ValueError(f"{what} is not on the current GPU")
    rows, cols = t.shape[-2:]
    if cols == 0:
        raise ValueError(f"{what} has no columns")
    stride = t.stride()
    if cols > 1 and stride[-1] != 1:
        raise ValueError(f"the columns of {what} must be contiguous")
    return stride[-2] if rows > 1 else (cols + 15) // 16 * 16


def _values(t, dims, what, device):
    import torch
    if t.dtype is not torch.float8_e4m3fn:
        raise ValueError(f"{what} must be float8_e4m3fn")
    return _rows(t, dims, what, device)


def _scales(t, shape, what, device):
    import torch
    if t.dtype is not torch.float32 or t.shape != shape or t.get_device() != device:
        raise ValueError(f"{what} must be float32 of shape {tuple(shape)} on the current GPU")
    return t.stride()


def _new_values(rows, cols, device):
    import torch
    if cols % 16 == 0:
        return torch.empty((rows, cols), dtype=torch.float8_e4m3fn, device=device)
    return torch.empty_strided((rows, cols), ((cols + 15) // 16 * 16, 1), dtype=torch.float8_e4m3fn, device=device)


def _new_scales(rows, cols, device):
    """Scales of activations: block column by block column."""
    import torch
    return torch.empty_strided((rows, -(-cols // FP8_BLOCK)), (1, max(rows, 1)), dtype=torch.float32, device=device)


def quant_fp8(X, block_rows: int = 1):
    """xorenc_quant_fp8: X (rows, cols), or a stack of such matrices, float32 or bfloat16 -> (Q, S) in blocks of
    block_rows (1: activations, 128: weights) x 128."""
    import torch
    dims, device = X.dim(), _device()
    if dims not in (2, 3):
        raise ValueError("X must be a matrix or a stack of matrices")
    ldx, dtype = _rows(X, dims, "X", device), _dtype(X, "X")
    rows, cols = X.shape[-2:]
    n = X.shape[0] if dims == 3 else 1
    dev = X.device
    if dims == 2:
        Q = _new_values(rows, cols, dev)
        S = _new_scales(rows, cols, dev) if block_rows == 1 else torch.empty((-(-rows // FP8_BLOCK), -(-cols // FP8_BLOCK)), device=dev)
        ss = (0,) + S.stride()
    else:
        ld = (cols + 15) // 16 * 16
        Q = torch.empty_strided((n, rows, cols), (rows * ld, ld, 1), dtype=torch.float8_e4m3fn, device=dev)
        S = torch.empty((n, -(-rows // block_rows) if block_rows > 0 else 0, -(-cols // FP8_BLOCK)), device=dev)
        ss = S.stride()
    qs = Q.stride()
    ldq = qs[-2] if rows > 1 else (cols + 15) // 16 * 16
    rc = _library().xorenc_quant_fp8(X.data_ptr(), dtype, ldx, X.stride(0) if n > 1 else 0, n, rows, cols, block_rows,
                                     Q.data_ptr(), ldq, qs[0] if dims == 3 else 0, S.data_ptr(), ss[1], ss[2], ss[0], _stream_ptr())
    if rc:
        _check(rc, "xorenc_quant_fp8")
    return Q, S


def add_rmsnorm_fp8(X, weight, residual=None, eps: float = 1e-6, total=None, normed=False):
    """xorenc_add_rmsnorm_fp8: t = X + residual, y = t / sqrt(mean(t^2) + eps) * weight in 8 bits.  Returns (Q, S, t, y).

    X (tokens, features), residual and t float32 or bfloat16, of one type; weight (features,) of either.  t is `total`, which may
    be X or residual, or a new tensor; None where there is no residual and no `total`.  normed: True to have y too, in
    the type of X, or the tensor that takes it, in any order (the transpose of a (features, tokens) tensor, say, which is
    what `spmm` multiplies); else y is None."""
    import torch
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    rows, cols = X.shape
    w_dtype = _dtype(weight, "weight")
    if weight.shape != (cols,) or weight.stride(0) != 1 and cols > 1 or weight.get_device() != device:
        raise ValueError("weight must be (features,), contiguous, on the current GPU")
    dev, res, ldr, tot, ldt, yp, ys = X.device, 0, 0, 0, 0, 0, (0, 1)
    if residual is not None:
        ldr = _rows(residual, 2, "residual", device)
        if residual.shape != X.shape or residual.dtype is not X.dtype:
            raise ValueError("residual must have the shape and type of X")
        res = residual.data_ptr()
        if total is None:
            total = torch.empty((rows, cols), dtype=X.dtype, device=dev)
    if total is not None:
        ldt = _rows(total, 2, "total", device)
        if total.shape != X.shape or total.dtype is not X.dtype:
            raise ValueError("total must have the shape and type of X")
        tot = total.data_ptr()
    y = None
    if normed is not False:
        y = torch.empty((rows, cols), dtype=X.dtype, device=dev) if normed is True else normed
        if y.shape != X.shape or y.dtype is not X.dtype or y.get_device() != device:
            raise ValueError("normed must have the shape and type of X, on the current GPU")
        yp, ys = y.data_ptr(), y.stride()
        if cols == 1:
            ys = (ys[0], 1)
    Q, S = _new_values(rows, cols, dev), _new_scales(rows, cols, dev)
    rc = _library().xorenc_add_rmsnorm_fp8(X.data_ptr(), dtype, ldx, res, ldr, weight.data_ptr(), w_dtype, rows, cols, eps, tot, ldt,
                                           yp, ys[0], ys[1], Q.data_ptr(), Q.stride(0), S.data_ptr(), 1, S.stride(1), _stream_ptr())
    if rc:
        _check(rc, "xorenc_add_rmsnorm_fp8")
    return Q, S, total, y


def silu_mul_fp8(X):
    """xorenc_silu_mul_fp8: X (tokens, 2 n) float32 or bfloat16, gates before ups -> (Q, S) of silu(gate) * up, (tokens, n)."""
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    rows, cols = X.shape
    if cols % 2:
        raise ValueError("X must have as many gates as ups")
    cols //= 2
    Q, S = _new_values(rows, cols, X.device), _new_scales(rows, cols, X.device)
    at = X.data_ptr()
    rc = _library().xorenc_silu_mul_fp8(at, at + cols * (2 if dtype == X_BF16 else 4), dtype, ldx, rows, cols, Q.data_ptr(), Q.stride(0),
                                        S.data_ptr(), 1, S.stride(1), _stream_ptr())
    if rc:
        _check(rc, "xorenc_silu_mul_fp8")
    return Q, S


def matmul_fp8(A, SA, W, SW, out_dtype=None, Y=None):
    """xorenc_matmul_fp8: Y = A W^T with A (tokens, inputs) in blocks of 1 x 128 and W (outputs, inputs) in blocks of
    128 x 128.  Y is float32 or bfloat16 (out_dtype, bfloat16 unless given)."""
    import torch
    device = _device()
    lda, ldw = _values(A, 2, "A", device), _values(W, 2, "W", device)
    M, K = A.shape
    N = W.shape[0]
    if W.shape[1] != K:
        raise ValueError("A and W must have as many columns")
    blocks = -(-K // FP8_BLOCK)
    sa = _scales(SA, (M, blocks), "SA", device)
    sw = _scales(SW, (-(-N // FP8_BLOCK), blocks), "SW", device)
    if blocks > 1 and sw[1] != 1:
        raise ValueError("the columns of SW must be contiguous")
    if Y is None:
        Y = torch.empty((M, N), dtype=out_dtype or torch.bfloat16, device=A.device)
    elif Y.shape != (M, N) or out_dtype not in (None, Y.dtype):
        raise ValueError("Y must be (tokens, outputs) of the type asked for")
    ldy, y_dtype = _rows(Y, 2, "Y", device), _dtype(Y, "Y")
    rc = _library().xorenc_matmul_fp8(A.data_ptr(), lda, SA.data_ptr(), sa[0], sa[1], W.data_ptr(), ldw, SW.data_ptr(),
                                      sw[0] if N > FP8_BLOCK else blocks, M, N, K, Y.data_ptr(), y_dtype, ldy, _stream_ptr())
    if rc:
        _check(rc, "xorenc_matmul_fp8")
    return Y


def moe_fp8(X, router, W13, S13, W2, S2, picks: int, renormalise: bool = True, Y=None):
    """xorenc_moe_fp8: a mixture-of-experts layer for at most MOE_MAX_TOKENS tokens.

    X (tokens, hidden) float32 or bfloat16, router (experts, hidden) of the same type; W13 (experts, 2 inner, hidden), the gates'
    rows before the ups', and W2 (experts, hidden, inner) in blocks of 128 x 128, as quant_fp8 lays stacks out.  Every token
    takes the `picks` experts with its largest logits; their softmax shares are made to sum to one unless renormalise is
    False.  Returns Y (tokens, hidden) of X's type (Y may be X)."""
    import torch
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    ldr = _rows(router, 2, "router", device)
    ld13, ld2 = _values(W13, 3, "W13", device), _values(W2, 3, "W2", device)
    T, H = X.shape
    E, _, I = W2.shape
    if router.dtype is not X.dtype or router.shape != (E, H):
        raise ValueError("router must be (experts, hidden) of the type of X")
    if W2.shape[1] != H or W13.shape != (E, 2 * I, H):
        raise ValueError("W13 must be (experts, 2 inner, hidden) and W2 (experts, hidden, inner)")
    hb, ib = -(-H // FP8_BLOCK), -(-I // FP8_BLOCK)
    s13 = _scales(S13, (E, -(-2 * I // FP8_BLOCK), hb), "S13", device)
    s2 = _scales(S2, (E, hb, ib), "S2", device)
    if hb > 1 and s13[2] != 1 or ib > 1 and s2[2] != 1:
        raise ValueError("the columns of S13 and S2 must be contiguous")
    if Y is None:
        Y = torch.empty((T, H), dtype=X.dtype, device=X.device)
    elif Y.shape != X.shape or Y.dtype is not X.dtype:
        raise ValueError("Y must have the shape and type of X")
    ldy = _rows(Y, 2, "Y", device)
    lib = _library()
    need = ctypes.c_int64(0)
    rc = lib.xorenc_moe_workspace(T, H, I, E, picks, dtype, ctypes.byref(need))
    if rc:
        _check(rc, "xorenc_moe_workspace")
    ws = torch.empty(need.value, dtype=torch.uint8, device=X.device)
    many = E > 1
    layer = _pack_moe(_MOE_BYTES, E, H, I, router.data_ptr(), ldr, W13.data_ptr(), ld13, W13.stride(0) if many else 0,
                      S13.data_ptr(), s13[1] if 2 * I > FP8_BLOCK else hb, s13[0] if many else 0, W2.data_ptr(), ld2,
                      W2.stride(0) if many else 0, S2.data_ptr(), s2[1] if H > FP8_BLOCK else ib, s2[0] if many else 0)
    rc = lib.xorenc_moe_fp8(layer, X.data_ptr(), dtype, ldx, T, picks, 1 if renormalise else 0, Y.data_ptr(), ldy, ws.data_ptr(),
                            need.value, _stream_ptr())
    if rc:
        _check(rc, "xorenc_moe_fp8")
    return Y

"""Dense layers in 8 bits: the calls of include/xorenc.h on e4m3 matrices with a scale per block of 128, argument marshalling only.

An 8-bit matrix is a pair of tensors: the values (torch.float8_e4m3fn, rows on 16-byte boundaries) and the scales (float32,
one for each 1 x 128 block of activations or 128 x 128 block of weights).  All tensors are on the current device, the
work goes to its current stream, and nothing waits.
"""
import ctypes
import struct

from .binding import X_BF16, X_F32, _check, load_library

FP8_BLOCK = 128
MOE_MAX_TOKENS, MOE_MAX_EXPERTS, MOE_MAX_PICKS = 64, 256, 16

_pack_moe = struct.Struct("I3iP q P2q P2q P2q P2q").pack
_MOE_BYTES = struct.calcsize("I3iP q P2q P2q P2q P2q")
# What the calls need of torch and the library, looked up once: an import statement in each call costs as much as a launch.
_lib = _new = _device = _stream = _BF16 = _F32 = _F8 = None
_X_DTYPE = {}


def _library():
    global _lib, _new, _device, _stream, _BF16, _F32, _F8
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
        import torch
        try:  # a new tensor on the current GPU: sizes, strides, type (0.8 us; torch.empty_strided: 1.3)
            _new = torch._C._dynamo.guards._empty_strided_cuda
        except AttributeError:
            def _new(sizes, strides, dtype):
                return torch.empty_strided(sizes, strides, dtype=dtype, device="cuda")
        _device, _stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream
        _BF16, _F32, _F8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
        _X_DTYPE.update({_BF16: X_BF16, _F32: X_F32})
        _lib = lib
    return _lib


def _dtype(t, what):
    d = _X_DTYPE.get(t.dtype)
    if d is None:
        raise ValueError(f"{what} must be float32 or bfloat16")
    return d


def _rows(t, dims, what, device):
    """Checks a row-major matrix (or stack of matrices) on the current device; returns its leading dimension."""
    shape, stride = t.shape, t.stride()
    if len(shape) != dims:
        raise ValueError(f"{what} must have {dims} dimensions")
    if t.get_device() != device:
        raise ValueError(f"{what} is not on the current GPU")
    cols = shape[-1]
    if stride[-1] != 1 and cols != 1:
        raise ValueError(f"the columns of {what} must be contiguous")
    if cols == 0:
        raise ValueError(f"{what} has no columns")
    return stride[-2] if shape[-2] > 1 else (cols + 15) // 16 * 16


def _values(t, dims, what, device):
    if t.dtype is not _F8:
        raise ValueError(f"{what} must be float8_e4m3fn")
    return _rows(t, dims, what, device)


def _scales(t, shape, what, device):
    if t.dtype is not _F32 or t.shape != shape or t.get_device() != device:
        raise ValueError(f"{what} must be float32 of shape {tuple(shape)} on the current GPU")
    return t.stride()


def _new_values(rows, cols):
    """e4m3 values whose rows start on 16-byte boundaries, and their leading dimension."""
    ld = (cols + 15) & -16
    return _new((rows, cols), (ld, 1), _F8), ld


def _new_scales(rows, cols):
    """Scales of activations: block column by block column."""
    return _new((rows, -(-cols // FP8_BLOCK)), (1, rows or 1), _F32)


def quant_fp8(X, block_rows: int = 1):
    """xorenc_quant_fp8: X (rows, cols), or a stack of such matrices, float32 or bfloat16 -> (Q, S) in blocks of
    block_rows (1: activations, 128: weights) x 128."""
    lib = _lib or _library()
    shape, device = X.shape, _device()
    dims = len(shape)
    if dims not in (2, 3):
        raise ValueError("X must be a matrix or a stack of matrices")
    ldx, dtype = _rows(X, dims, "X", device), _dtype(X, "X")
    rows, cols = shape[-2:]
    blocks = -(-cols // FP8_BLOCK)
    n = x_mat = q_mat = s_mat = 0
    if dims == 2:
        n = 1
        Q, ldq = _new_values(rows, cols)
        if block_rows == 1:
            S, s_row, s_blk = _new_scales(rows, cols), 1, rows or 1
        else:
            S, s_row, s_blk = _new((-(-rows // FP8_BLOCK), blocks), (blocks, 1), _F32), blocks, 1
    else:
        n, ldq, x_mat = shape[0], (cols + 15) & -16, X.stride(0)
        q_mat, s_rows = rows * ldq, rows if block_rows == 1 else -(-rows // FP8_BLOCK)
        s_mat, s_row, s_blk = s_rows * blocks, blocks, 1
        Q, S = _new((n, rows, cols), (q_mat, ldq, 1), _F8), _new((n, s_rows, blocks), (s_mat, blocks, 1), _F32)
    rc = lib.xorenc_quant_fp8(X.data_ptr(), dtype, ldx, x_mat, n, rows, cols, block_rows, Q.data_ptr(), ldq, q_mat, S.data_ptr(), s_row,
                              s_blk, s_mat, _stream(device))
    if rc:
        _check(rc, "xorenc_quant_fp8")
    return Q, S


def add_rmsnorm_fp8(X, weight, residual=None, eps: float = 1e-6, total=None, normed=False):
    """xorenc_add_rmsnorm_fp8: t = X + residual, y = t / sqrt(mean(t^2) + eps) * weight in 8 bits.  Returns (Q, S, t, y).

    X (tokens, features), residual and t float32 or bfloat16, of one type; weight (features,) of either.  t is `total`, which may
    be X or residual, or a new tensor; None where there is no residual and no `total`.  normed: True to have y too, in
    the type of X, or the tensor that takes it, in any order (the transpose of a (features, tokens) tensor, say, which is
    what `spmm` multiplies); else y is None."""
    lib = _lib or _library()
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    shape = X.shape
    rows, cols = shape
    w_dtype = _dtype(weight, "weight")
    if weight.shape != (cols,) or weight.stride(0) != 1 and cols > 1 or weight.get_device() != device:
        raise ValueError("weight must be (features,), contiguous, on the current GPU")
    res = ldr = tot = ldt = yp = y_row = 0
    y_col, y = 1, None
    if residual is not None:
        ldr = _rows(residual, 2, "residual", device)
        if residual.shape != shape or residual.dtype is not X.dtype:
            raise ValueError("residual must have the shape and type of X")
        res = residual.data_ptr()
        if total is None:
            total = _new((rows, cols), (cols, 1), X.dtype)
            tot, ldt = total.data_ptr(), cols
    if total is not None and not tot:
        ldt = _rows(total, 2, "total", device)
        if total.shape != shape or total.dtype is not X.dtype:
            raise ValueError("total must have the shape and type of X")
        tot = total.data_ptr()
    if normed is True:
        y = _new((rows, cols), (cols, 1), X.dtype)
        yp, y_row = y.data_ptr(), cols
    elif normed is not False:
        y = normed
        if y.shape != shape or y.dtype is not X.dtype or y.get_device() != device:
            raise ValueError("normed must have the shape and type of X, on the current GPU")
        yp, (y_row, y_col) = y.data_ptr(), y.stride()
        if cols == 1:
            y_col = 1
    Q, ldq = _new_values(rows, cols)
    S = _new_scales(rows, cols)
    rc = lib.xorenc_add_rmsnorm_fp8(X.data_ptr(), dtype, ldx, res, ldr, weight.data_ptr(), w_dtype, rows, cols, eps, tot, ldt or cols, yp,
                                    y_row, y_col, Q.data_ptr(), ldq, S.data_ptr(), 1, rows or 1, _stream(device))
    if rc:
        _check(rc, "xorenc_add_rmsnorm_fp8")
    return Q, S, total, y


def silu_mul_fp8(X):
    """xorenc_silu_mul_fp8: X (tokens, 2 n) float32 or bfloat16, gates before ups -> (Q, S) of silu(gate) * up, (tokens, n)."""
    lib = _lib or _library()
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    rows, cols = X.shape
    if cols % 2:
        raise ValueError("X must have as many gates as ups")
    cols //= 2
    Q, ldq = _new_values(rows, cols)
    S = _new_scales(rows, cols)
    at = X.data_ptr()
    rc = lib.xorenc_silu_mul_fp8(at, at + cols * (2 if dtype == X_BF16 else 4), dtype, ldx, rows, cols, Q.data_ptr(), ldq, S.data_ptr(),
                                 1, rows or 1, _stream(device))
    if rc:
        _check(rc, "xorenc_silu_mul_fp8")
    return Q, S


def matmul_fp8(A, SA, W, SW, out_dtype=None, Y=None):
    """xorenc_matmul_fp8: Y = A W^T with A (tokens, inputs) in blocks of 1 x 128 and W (outputs, inputs) in blocks of
    128 x 128.  Y is float32 or bfloat16 (out_dtype, bfloat16 unless given)."""
    lib = _lib or _library()
    device = _device()
    lda, ldw = _values(A, 2, "A", device), _values(W, 2, "W", device)
    M, K = A.shape
    N, k = W.shape
    if k != K:
        raise ValueError("A and W must have as many columns")
    blocks = -(-K // FP8_BLOCK)
    sa_row, sa_blk = _scales(SA, (M, blocks), "SA", device)
    ldsw, one = _scales(SW, (-(-N // FP8_BLOCK), blocks), "SW", device)
    if one != 1 and blocks > 1:
        raise ValueError("the columns of SW must be contiguous")
    if Y is None:
        Y, ldy = _new((M, N), (N, 1), out_dtype or _BF16), N
    else:
        ldy = _rows(Y, 2, "Y", device)
        if Y.shape != (M, N) or out_dtype not in (None, Y.dtype):
            raise ValueError("Y must be (tokens, outputs) of the type asked for")
    rc = lib.xorenc_matmul_fp8(A.data_ptr(), lda, SA.data_ptr(), sa_row, sa_blk if blocks > 1 else 0, W.data_ptr(), ldw, SW.data_ptr(),
                               ldsw if N > FP8_BLOCK else blocks, M, N, K, Y.data_ptr(), _dtype(Y, "Y"), ldy, _stream(device))
    if rc:
        _check(rc, "xorenc_matmul_fp8")
    return Y


def moe_fp8(X, router, W13, S13, W2, S2, picks: int, renormalise: bool = True, Y=None):
    """xorenc_moe_fp8: a mixture-of-experts layer for at most MOE_MAX_TOKENS tokens.

    X (tokens, hidden) float32 or bfloat16, router (experts, hidden) of the same type; W13 (experts, 2 inner, hidden), the gates'
    rows before the ups', and W2 (experts, hidden, inner) in blocks of 128 x 128, as quant_fp8 lays stacks out.  Every token
    takes the `picks` experts with its largest logits; their softmax shares are made to sum to one unless renormalise is
    False.  Returns Y (tokens, hidden) of X's type (Y may be X)."""
    lib = _lib or _library()
    device = _device()
    ldx, dtype = _rows(X, 2, "X", device), _dtype(X, "X")
    ldr = _rows(router, 2, "router", device)
    ld13, ld2 = _values(W13, 3, "W13", device), _values(W2, 3, "W2", device)
    T, H = X.shape
    E, h, I = W2.shape
    if router.dtype is not X.dtype or router.shape != (E, H):
        raise ValueError("router must be (experts, hidden) of the type of X")
    if h != H or W13.shape != (E, 2 * I, H):
        raise ValueError("W13 must be (experts, 2 inner, hidden) and W2 (experts, hidden, inner)")
    hb, ib = -(-H // FP8_BLOCK), -(-I // FP8_BLOCK)
    e13, l13, one13 = _scales(S13, (E, -(-2 * I // FP8_BLOCK), hb), "S13", device)
    e2, l2, one2 = _scales(S2, (E, hb, ib), "S2", device)
    if hb > 1 and one13 != 1 or ib > 1 and one2 != 1:
        raise ValueError("the columns of S13 and S2 must be contiguous")
    if Y is None:
        Y, ldy = _new((T, H), (H, 1), X.dtype), H
    else:
        ldy = _rows(Y, 2, "Y", device)
        if Y.shape != X.shape or Y.dtype is not X.dtype:
            raise ValueError("Y must have the shape and type of X")
    need = ctypes.c_int64(0)
    rc = lib.xorenc_moe_workspace(T, H, I, E, picks, dtype, ctypes.byref(need))
    if rc:
        _check(rc, "xorenc_moe_workspace")
    ws = _new((need.value // 4 + 1,), (1,), _F32)
    m13, m2 = (W13.stride(0), W2.stride(0)) if E > 1 else (0, 0)
    layer = _pack_moe(_MOE_BYTES, E, H, I, router.data_ptr(), ldr, W13.data_ptr(), ld13, m13, S13.data_ptr(),
                      l13 if 2 * I > FP8_BLOCK else hb, e13, W2.data_ptr(), ld2, m2, S2.data_ptr(), l2 if H > FP8_BLOCK else ib, e2)
    rc = lib.xorenc_moe_fp8(layer, X.data_ptr(), dtype, ldx, T, picks, 1 if renormalise else 0, Y.data_ptr(), ldy, ws.data_ptr(),
                            need.value, _stream(device))
    if rc:
        _check(rc, "xorenc_moe_fp8")
    return Y

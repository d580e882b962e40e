"""Dense layers in 8 bits: the calls of include/xorenc.h on e4m3 matrices with a scale per block of 128, argument marshalling only.

An 8-bit matrix is a pair of tensors: the values (torch.float8_e4m3fn, rows on 16-byte boundaries) and the scales (float32,
one for each 1 x 128 block of activations or 128 x 128 block of weights).  All tensors are on the current device, the
work goes to its current stream, and nothing waits.  The marshalling is in csrc/xorenc_torch_fp8.cpp.
"""
import os
import struct

from .binding import library_path, load_library as _library

FP8_BLOCK = 128
MOE_MAX_TOKENS, MOE_MAX_EXPERTS, MOE_MAX_PICKS = 64, 256, 16

# The bytes of struct xorenc_moe, for calls of the C ABI through ctypes.
_pack_moe = struct.Struct("I3iP q P2q P2q P2q P2q").pack
_MOE_BYTES = struct.calcsize("I3iP q P2q P2q P2q P2q")

_native = None


def _load():
    """The extension, which like the library is built by `python -m paper_1905_10138_amd.build`."""
    global _native
    if _native is None:
        path = os.path.join(os.path.dirname(library_path()), "_fp8.so")
        if not os.path.exists(path):
            raise RuntimeError(f"{path} is missing: build it with `python -m paper_1905_10138_amd.build` (there is no fallback path)")
        _library()
        import torch  # noqa: F401  (the extension's symbols)
        from . import _fp8
        _native = _fp8
    return _native


def quant_fp8(X, block_rows: int = 1):
    """xorenc_quant_fp8: X (rows, cols), or a stack of such matrices, float32 or bfloat16 -> (Q, S) in blocks of
    block_rows (1: activations, 128: weights) x 128."""
    return (_native or _load()).quant(X, block_rows)


def add_rmsnorm_fp8(X, weight, residual=None, eps: float = 1e-6, total=None, normed=False):
    """xorenc_add_rmsnorm_fp8: t = X + residual, y = t / sqrt(mean(t^2) + eps) * weight in 8 bits.  Returns (Q, S, t, y).

    X (tokens, features), residual and t float32 or bfloat16, of one type; weight (features,) of either.  t is `total`, which may
    be X or residual, or a new tensor; None where there is no residual and no `total`.  normed: True to have y too, in
    the type of X, or the tensor that takes it, in any order (the transpose of a (features, tokens) tensor, say, which is
    what `spmm` multiplies); else y is None."""
    return (_native or _load()).norm(X, weight, residual, eps, total, normed)


def silu_mul_fp8(X):
    """xorenc_silu_mul_fp8: X (tokens, 2 n) float32 or bfloat16, gates before ups -> (Q, S) of silu(gate) * up, (tokens, n)."""
    return (_native or _load()).gate(X)


def matmul_fp8(A, SA, W, SW, out_dtype=None, Y=None):
    """xorenc_matmul_fp8: Y = A W^T with A (tokens, inputs) in blocks of 1 x 128 and W (outputs, inputs) in blocks of
    128 x 128.  Y is float32 or bfloat16 (out_dtype, bfloat16 unless given); float32 adds exact products in fp32, bfloat16
    products that are aligned to a block's largest (include/xorenc.h), which results that cancel to far less than their terms show."""
    return (_native or _load()).matmul(A, SA, W, SW, out_dtype, Y)


def moe_fp8(X, router, W13, S13, W2, S2, picks: int, renormalise: bool = True, Y=None):
    """xorenc_moe_fp8: a mixture-of-experts layer for at most MOE_MAX_TOKENS tokens.

    X (tokens, hidden) float32 or bfloat16, router (experts, hidden) of the same type; W13 (experts, 2 inner, hidden), the gates'
    rows before the ups', and W2 (experts, hidden, inner) in blocks of 128 x 128, as quant_fp8 lays stacks out.  Every token
    takes the `picks` experts with its largest logits; their softmax shares are made to sum to one unless renormalise is
    False.  Returns Y (tokens, hidden) of X's type (Y may be X)."""
    return (_native or _load()).moe(X, router, W13, S13, W2, S2, picks, renormalise, Y)

"""Dense layers in 8 bits: the calls of include/xorenc.h on e4m3 matrices with a scale per block of 128, argument marshalling only.

An 8-bit matrix is a pair of tensors: the values (torch.float8_e4m3fn, rows on 16-byte boundaries) and the scales (float32,
one for each 1 x 128 block of activations or 128 x 128 block of weights).  All tensors are on the current device, the
work goes to its current stream, and nothing waits.  No call records anything for torch's gradients.  The marshalling is in
csrc/xorenc_torch_fp8.cpp and csrc/xorenc_torch_experts.h.

Experts for any number of tokens, as a layer runs them:

    ids, shares = pick_experts(logits, picks)
    places, tokens, offsets = sort_tokens(ids, experts)
    u = experts_fp8(Q, S, *W13, offsets, tokens)
    d = experts_fp8(*silu_mul_fp8(u), *W2, offsets)
    y = combine_tokens(d, places, offsets, shares, residual)
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


def linear_fp8(A, SA, W, SW, bias=None, activation=None, residual=None, out_dtype=None, Y=None):
    """xorenc_linear_fp8: Y = residual + f(A W^T + bias), matmul_fp8 with an epilogue that is computed in fp32 before the only rounding.

    bias (outputs,) float32 or bfloat16; activation None, 'relu', 'silu', 'gelu' (with the error function) or 'gelu_tanh'; residual (tokens,
    outputs) of the type of Y, which may be Y."""
    return (_native or _load()).linear(A, SA, W, SW, bias, activation, residual, out_dtype, Y)


def pick_experts(logits, picks: int, renormalise: bool = True):
    """xorenc_pick_experts: the experts of each token and their shares -> (ids int32, shares float32), both (tokens, picks).

    logits (tokens, experts) float32 or bfloat16.  The largest logits, the lowest index of equals; an expert whose logit is -inf is
    never picked, and where fewer are left the id is -1 and the share 0.  The shares are the softmax over all experts,
    made to sum to one over the picked ones unless renormalise is False."""
    return (_native or _load()).pick(logits, picks, renormalise)


def sort_tokens(ids, experts: int):
    """xorenc_sort_tokens: the pairs of tokens and experts sorted by expert -> (places, tokens, offsets), int32.

    ids (tokens, picks) int32 or int64.  places (tokens, picks) is the row of each pair, tokens (tokens * picks,) the token of each row, and
    rows offsets[e] .. offsets[e + 1] - 1 are expert e's, in the order of the tokens.  Ids outside 0 .. experts - 1 are pairs without an expert:
    their rows come last, from offsets[experts] on."""
    return (_native or _load()).sort(ids, experts)


def gather_tokens(X, places, offsets, shares=None, R=None):
    """xorenc_gather_tokens: R[places[t, p]] = X[t], times shares[t, p] if they are given; zero for pairs without an expert.

    X (tokens, features) float32 or bfloat16; R (tokens * picks, features) of its type.  Its gradient for X is combine_tokens(dR, places,
    offsets, shares), and for the shares the second result of combine_tokens_grad(X, dR, places, offsets, shares)."""
    return (_native or _load()).gather(X, places, offsets, shares, R)


def combine_tokens(R, places, offsets, shares=None, residual=None, Y=None):
    """xorenc_combine_tokens: Y[t] = sum over p of shares[t, p] R[places[t, p]] (without shares: of the rows alone) + residual[t].

    R (tokens * picks, features) float32 or bfloat16; residual and Y (tokens, features) of its type, Y may be residual.  Pairs without an expert
    add nothing.  Sums are in fp32, in the order of p."""
    return (_native or _load()).combine(R, places, offsets, shares, residual, Y)


def combine_tokens_grad(dY, R, places, offsets, shares, dR=None):
    """xorenc_combine_tokens_grad: the gradients of combine_tokens for R and shares, given that for Y -> (dR, dshares).

    dR (the type of R; it may be R) is zero where a pair has no expert, and so is dshares (float32).  The residual's gradient is dY, and
    without shares R's is gather_tokens(dY, places, offsets)."""
    return (_native or _load()).combine_grad(dY, R, places, offsets, shares, dR)


def experts_fp8(A, SA, W, SW, offsets, tokens=None, bias=None, activation=None, out_dtype=None, Y=None):
    """xorenc_experts_fp8: products of sorted rows with their own expert's matrix, Y[i] = f(A[tokens[i]] W[e]^T + bias[e]) for
    offsets[e] <= i < offsets[e + 1].

    A in blocks of 1 x 128: a row for each token, with `tokens` of sort_tokens, or without it a row for each row of Y.  W (experts, outputs,
    inputs) in blocks of 128 x 128, as quant_fp8 lays stacks out; bias (experts, outputs) and activation as linear_fp8.  Rows of Y from
    offsets[experts] on are left as they are: in a new Y they hold anything."""
    return (_native or _load()).experts(A, SA, W, SW, offsets, tokens, bias, activation, out_dtype, Y)

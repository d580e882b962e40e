"""What an epilogue makes of a bias or a residual that is not finite, in its column, and in no other: the formula's value, residual + f(z + bias), with IEEE
arithmetic (x / (1 + exp(-x)) and x times a distribution function that is 0 are NaN for -infinity)."""
import math

import pytest
import torch

import paper_1905_10138_amd as xe
from test_gpu_experts import ACTIVATIONS, TYPES, operands, random_on_gpu
from test_gpu_fp8 import DEV, gen, normal

pytestmark = pytest.mark.gpu

INF, NAN = math.inf, math.nan
WANT = {None: {INF: INF, -INF: -INF}, "relu": {INF: INF, -INF: 0.0}, "silu": {INF: INF, -INF: NAN}, "gelu": {INF: INF, -INF: NAN},
        "gelu_tanh": {INF: INF, -INF: NAN}}


def same(got, want):
    """Equal, with NaN in the same places."""
    return bool(((got == want) | (got.isnan() & want.isnan())).all())


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("M,N,K", [(1, 70, 200), (40, 70, 200), (300, 260, 600)])
def test_of_one_product(M, N, K, activation, out):
    A, SA, W, SW, b, r = operands(gen(M + N), M, N, K, out, torch.float32, True)
    clean = xe.linear_fp8(A, SA, W, SW, b, activation, r, out_dtype=out)
    for bias_type in (torch.float32, torch.bfloat16):
        clean = xe.linear_fp8(A, SA, W, SW, b.to(bias_type), activation, r, out_dtype=out)
        for v in (NAN, INF, -INF):
            bad = b.to(bias_type)
            bad[11] = v
            want = clean.clone()
            f = NAN if math.isnan(v) else WANT[activation][v]
            want[:, 11] = (f + r[:, 11].float()).to(out)
            assert same(xe.linear_fp8(A, SA, W, SW, bad, activation, r, out_dtype=out), want), v
            # and against a residual that is the other infinity
            other = r.clone()
            other[:, 11] = -INF
            want[:, 11] = NAN if f in (INF,) or math.isnan(f) else -INF
            assert same(xe.linear_fp8(A, SA, W, SW, bad, activation, other, out_dtype=out), want), v


@pytest.mark.parametrize("out", TYPES)
@pytest.mark.parametrize("activation", ACTIVATIONS)
@pytest.mark.parametrize("T", [3, 90, 1200])
def test_of_experts(T, activation, out):
    g = gen(T)
    P, E, N, K = 2, 5, 140, 260
    ids = torch.rand((T, E), generator=g).argsort(1)[:, :P].to(torch.int32).contiguous()
    ids[0, 0] = -1
    _, tokens, offsets = xe.sort_tokens(ids.to(DEV), E)
    A, SA = random_on_gpu(1, T, K, block_rows=1)
    W, SW = random_on_gpu(2, E, N, K, block_rows=128)
    b = normal(g, E, N).to(DEV)
    Y = torch.full((T * P, N), 9.0, dtype=out, device=DEV)
    clean = xe.experts_fp8(A, SA, W, SW, offsets, tokens, b, activation, Y=Y).clone()
    at = offsets.tolist()
    e = max(range(E), key=lambda e: at[e + 1] - at[e])
    for v in (NAN, INF, -INF):
        bad = b.clone()
        bad[e, 77] = v
        want = clean.clone()
        want[at[e]:at[e + 1], 77] = NAN if math.isnan(v) else WANT[activation][v]
        assert same(xe.experts_fp8(A, SA, W, SW, offsets, tokens, bad, activation, Y=Y), want), v

"""The operators as a program uses them: examples/feed_forward.py, each part against 64-bit arithmetic on the part's own inputs.

Rounding a normal value to e4m3 is off by at most 2^-4 of it and by 0.026 of it in the root mean square (a half step of
2^-4 of the binade's start, uniform: 2^-3 / sqrt(12) over a mean significand of 1.4); the sum of a product of many
independent terms is off by as much in the 2-norm.  Two operands rounded so: 0.037.  The limits are 1.5 times these."""
import importlib.util
import os

import pytest
import torch

import paper_1905_10138_amd as xe
import fp8_oracle as ref
from synth_inputs import CONFIGS, make_workload

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "feed_forward.py")
    spec = importlib.util.spec_from_file_location("feed_forward_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.fixture(scope="module")
def layers(example):
    workload = make_workload(CONFIGS["large_q1"], m=512, n=384)
    return example.build(workload, experts=6, picks=2, inner=200)


@pytest.mark.parametrize("tokens", [1, 7, 64, 65, 130])
def test_the_parts(example, layers, tokens):
    gated, moe, draw = layers
    x, r = draw(tokens, 384), draw(tokens, 384)
    t, u = gated.up(x, r)
    want_t, want_n = ref.rmsnorm(x.cpu(), r.cpu(), gated.norm.cpu(), 1e-6)
    assert (t.cpu().double() - want_t).abs().max() <= 2.0 ** -8 * want_t.abs().max()
    W13 = xe.decode(gated.encrypted, xe.OUT_F32).cpu().double()
    want_u = want_n @ W13.t()
    # the norm in 16 bits (2^-8 at most, 0.0016 in the root mean square; fp32 sums), or activations and weights in 8 bits and the result in 16
    limit = 1.5 * 2.0 ** -9 if tokens <= example.MOST_ENCRYPTED else 1.5 * 0.037
    assert u.shape == (tokens, 512) and example.off_by(u.cpu(), want_u) <= limit
    # the activations in 8 bits (the weights are what they are), the result in 16
    d = gated.down(u)
    want_d = ref.silu_mul(u.cpu()) @ ref.dense(*gated.W2, 128).t()
    assert example.off_by(d.cpu(), want_d) <= 1.5 * 0.026
    assert example.compare(gated, moe, x, r) == pytest.approx((example.off_by(u.cpu(), want_u), example.off_by(d.cpu(), want_d)), rel=1e-3)


@pytest.mark.parametrize("tokens", [1, 7, 65])
def test_the_experts(example, layers, tokens):
    gated, moe, draw = layers
    n = draw(tokens, 384)
    y = moe.experts(n)
    W13 = torch.stack([ref.dense(q, s, 128) for q, s in zip(*moe.W13)])
    W2 = torch.stack([ref.dense(q, s, 128) for q, s in zip(*moe.W2)])
    want, _ = ref.moe(n.cpu(), moe.router.cpu(), W13, W2, 2, True)
    assert example.off_by(y.cpu(), want) <= 2.0 ** -8  # what lies between the products holds 16 bits or more; the result is rounded to 16


@pytest.mark.parametrize("tokens", [1, 64, 200])
def test_the_whole(example, layers, tokens):
    gated, moe, draw = layers
    x, r = draw(tokens, 384), draw(tokens, 384)
    y = example.forward(gated, moe, x, r)
    t, d = gated(x, r)
    s, e = moe(d, t)
    assert torch.equal(y, s + e) and torch.equal(s, (d.float() + t.float()).to(s.dtype)) and torch.isfinite(y).all()


def test_arguments_that_are_no_tensors_of_the_call():
    x = torch.zeros(4, 256, device="cuda")
    Q, S = xe.quant_fp8(x)
    W, SW = xe.quant_fp8(x, block_rows=128)
    for call in (lambda: xe.quant_fp8(None), lambda: xe.silu_mul_fp8([1.0]), lambda: xe.matmul_fp8(Q, S, W, 1), lambda: xe.quant_fp8(x, "1"),
                 lambda: xe.add_rmsnorm_fp8(x, x[0], eps="1"), lambda: xe.add_rmsnorm_fp8(x, x[0], normed="yes")):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: xe.quant_fp8(x, 1 << 40), lambda: xe.matmul_fp8(Q, S, W, SW, out_dtype=3), lambda: xe.quant_fp8(x.to_sparse()),
                 lambda: xe.quant_fp8(x[:, None, None]), lambda: xe.quant_fp8(x.to("meta")), lambda: xe.add_rmsnorm_fp8(x, x[0], normed=x.cpu())):
        with pytest.raises(ValueError):
            call()

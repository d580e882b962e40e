"""The example's experts give results of their input's type, whichever way they take.

Rows of 32 bits are off by the activations' rounding to 8 bits where they are sorted, as in test_gpu_feed_forward_many.py: 0.047, and the limit is
1.5 times that."""
import pytest
import torch

import paper_1905_10138_amd as xe
import fp8_oracle as ref
from test_gpu_feed_forward import example, layers  # noqa: F401  (fixtures)

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wide(example, layers):  # noqa: F811
    """The layer of experts with a router and rows of 32 bits, and weights of its own."""
    _, moe, draw = layers
    W13, W2 = draw(6, 400, 384, scale=384 ** -0.5), draw(6, 384, 200, scale=200 ** -0.5)
    return example.ExpertLayer(moe.router.float(), W13, W2, moe.norm, 2)


@pytest.mark.parametrize("tokens", [1, 129, 300])
def test_sorted_experts_keep_their_rows_type(example, layers, wide, tokens):  # noqa: F811
    _, _, draw = layers
    n = draw(tokens, 384, dtype=torch.float32)
    y = wide.sorted_experts(n, *xe.quant_fp8(n))
    assert y.shape == n.shape and y.dtype is torch.float32
    W13 = torch.stack([ref.dense(q, s, 128) for q, s in zip(*wide.W13)])
    W2 = torch.stack([ref.dense(q, s, 128) for q, s in zip(*wide.W2)])
    want, _ = ref.moe(n.cpu(), wide.router.cpu(), W13, W2, 2, True)
    assert example.off_by(y.cpu(), want) <= 1.5 * 0.047
    # results that were rounded to 16 bits would all be equal to what this rounds them to; of others one in 2^16 is
    assert (y.to(torch.bfloat16).float() != y).float().mean() > 0.9


@pytest.mark.parametrize("tokens", [64, 129, 300])
def test_the_layer_keeps_its_rows_type(example, layers, wide, tokens):  # noqa: F811
    _, _, draw = layers
    x = draw(tokens, 384, dtype=torch.float32)
    t, y = wide(x, x)
    assert t.dtype is y.dtype is torch.float32 and y.shape == x.shape

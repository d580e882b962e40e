"""Whoever makes the example's layer of experts chooses from how many tokens on its activations are rounded to 8 bits: none chosen, none rounded."""
import sys

import pytest
import torch

import paper_1905_10138_amd as xe
from test_gpu_feed_forward import example, layers  # noqa: F401  (fixtures)


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [64, 129, 300])
def test_a_layer_of_no_choice_rounds_nothing(example, layers, tokens):  # noqa: F811
    _, moe, draw = layers
    W13, W2 = draw(6, 400, 384, scale=384 ** -0.5), draw(6, 384, 200, scale=200 ** -0.5)
    x = draw(tokens, 384)
    Q, S, t, n = xe.add_rmsnorm_fp8(x, moe.norm, x, normed=True)
    exact = example.ExpertLayer(moe.router, W13, W2, moe.norm, 2)
    got = exact(x, x)
    assert torch.equal(got[0], t) and torch.equal(got[1], exact.experts(n))
    rounded = example.ExpertLayer(moe.router, W13, W2, moe.norm, 2, most_unrounded=tokens - 1)
    assert torch.equal(rounded(x, x)[1], rounded.sorted_experts(n, Q, S))
    at_most = example.ExpertLayer(moe.router, W13, W2, moe.norm, 2, most_unrounded=tokens)
    assert torch.equal(at_most(x, x)[1], got[1])


class Asked(Exception):
    pass


@pytest.mark.parametrize("words,limit", [([], None), (["--tokens", "1024"], None), (["--most-unrounded", "128"], 128), (["--most-unrounded", "0"], 0)])
def test_the_command_rounds_nothing_unless_told(example, monkeypatch, words, limit):  # noqa: F811
    def build(*args, most_unrounded="nothing", **more):
        raise Asked(most_unrounded)
    monkeypatch.setattr(example, "build", build)
    monkeypatch.setattr(example, "make_workload", lambda config: None)
    monkeypatch.setattr(sys, "argv", ["feed_forward.py", *words])
    with pytest.raises(Asked) as asked:
        example.main()
    assert asked.value.args == (limit,)

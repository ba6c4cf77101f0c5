"""The mixture-of-experts example: it learns, repeats itself bit by bit, and its decode step gives
what its training forward gives."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mx4_experts", os.path.join(ROOT, "examples", "mx4_experts.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_training_lowers_the_loss_and_repeats(example):
    _, a = example.train(steps=12, experts=4, dim=128, hidden=256, tokens=500)
    _, b = example.train(steps=12, experts=4, dim=128, hidden=256, tokens=500)
    assert a == b
    assert a[-1] < 0.8 * a[0] and all(x > 0 for x in a)


@pytest.mark.parametrize("tokens", [1, 5, 300])
def test_decode_gives_the_training_forward(example, tokens):
    layer = example.Experts(4, 160, 224, 2)
    x = torch.randn(tokens, 160, device="cuda").bfloat16()
    # the same rows in other places: blocks of 32 lie along the columns in both
    assert torch.equal(layer.forward(x), layer.forward(x, keep=True))

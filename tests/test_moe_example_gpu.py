"""The example of the expert layer: dispatch, sort, gather, products, scatter, combine and the backward pass together."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

# e4m3 keeps 3 bits of fraction: a rounding is off by at most 2^-4 and on average (2-norm, values spread evenly over a
# binade) by about 2^-4 / sqrt(3) * 0.72 = 0.026 of its value.  An output passes 4 independent roundings (x, w1, h, w2),
# a gradient at most 9 (those of the forward pass that it saw, the gradient's own, and the transposed weights'), and
# the activation passes the gate's error on by a factor below 1.1: 1.1 * sqrt(9) * 0.026 = 0.086, and half as much again
# for values that one block's scale puts near the smallest ones.
MOST = 0.13


@pytest.mark.parametrize("sizes", [
    dict(ranks=8, tokens=32, hidden=512, inner=256, experts=32, topk=4),
    dict(ranks=2, tokens=77, hidden=200, inner=136, experts=6, topk=2),
    dict(ranks=4, tokens=1, hidden=128, inner=128, experts=64, topk=8)])
def test_example(sizes):
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "expert_layer.py")
    spec = importlib.util.spec_from_file_location("expert_layer_example", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    example.nuna.init()
    errors = example.run(**sizes)
    assert set(errors) == {"out", "dx", "dweights", "dw1", "dw2"}
    assert all(e < MOST for e in errors.values()), errors

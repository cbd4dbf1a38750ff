"""The operators of a layer together, as examples/adapted_layer.py uses them."""
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))


def test_training_finds_the_adapters():
    from adapted_layer import Layer, train
    losses = train(Layer(K=256, N=192, r=16, G=3, rows=300), steps=40, M=300)
    assert losses[-1] < 0.5 * losses[0]
    assert all(b < 1.02 * a for a, b in zip(losses, losses[1:]))


def test_serving_in_8_bits_is_near_bfloat16():
    from adapted_layer import BF16, Layer
    layer = Layer(K=512, N=320, r=16, G=3, rows=64)
    layer.B.normal_(0, 0.25)
    x, res = (torch.randn(20, 512, device="cuda").to(BF16) for _ in range(2))
    ids = (torch.arange(20, device="cuda") % 4 - 1).to(torch.int32)
    h, _, Y = layer.forward(x, res, ids)
    h8, Y8 = layer.decode(x, res, ids)
    assert torch.equal(h, h8)
    # 127 steps for about four standard deviations on both sides: an error of a
    # hundredth of each operand, independent from product to product
    assert float((Y8.float() - Y.float()).norm() / Y.float().norm()) < 0.03

"""The plain implementations that the products in 4 bits and the heads' norms are tested
against, themselves against other ways to the same values (host only)."""
import itertools

import pytest
import torch

from heads_util import forward64, grad64, turned
from layer_util import gen, randn
from mx4_util import MAG, pack, quant64, rounded64, unpack, value64


def test_codes_round_to_nearest_even():
    """Against the borders between neighbouring codes, one value after another."""
    for e in (-127, -3, 0, 40, 125):
        s = 2.0 ** e
        # a block's largest value is 4 s: its scale is s
        for i, f in itertools.product(range(8), (-1e-9, 0.0, 1e-9)):
            lo = float(MAG[i])
            hi = float(MAG[i + 1]) if i < 7 else 8.0
            x = torch.zeros(1, 32, dtype=torch.float64)
            x[0, 0], x[0, 1] = 4 * s, ((lo + hi) / 2 + f) * s
            if float(x[0, 1]) >= 8 * s:
                continue
            codes, byte = quant64(x)
            assert int(byte[0, 0]) == e + 127
            want = i if i == 7 or f < 0 or (f == 0 and i % 2 == 0) else i + 1
            assert int(codes[0, 1]) == want, (e, i, f)


def test_rounding_is_within_half_a_step_and_idempotent():
    x = randn((40, 300), torch.float32, gen(1)) * torch.exp2(torch.arange(40.0))[:, None]
    y = rounded64(x)
    assert torch.equal(rounded64(y), y)
    amax = torch.nn.functional.pad(x, (0, 20)).view(40, -1, 32).abs().amax(2).double()
    step = torch.exp2(torch.floor(torch.log2(amax)) - 2)      # of a half below 2 scales, 2 above 4
    off = torch.nn.functional.pad((x.double() - y).abs(), (0, 20)).view(40, -1, 32)
    assert bool((off <= step[..., None] * 2).all())
    q, w = pack(*quant64(x))
    assert torch.equal(value64(*unpack(q, w))[:, :300], y)


@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("dim,rot,eps", [(8, 8, 1e-5), (10, 6, 0.0), (7, 4, 1e-2), (6, 0, 1e-5)])
def test_gradients_are_the_formulas_and_the_differences(adjacent, dim, rot, eps):
    g = gen(dim)
    x = randn((3, 2, dim), torch.float64, g).requires_grad_()
    w = randn((dim,), torch.float64, g).requires_grad_()
    dy = randn((3, 2, dim), torch.float64, g)
    angle = randn((3, rot // 2), torch.float64, g, 3.0)
    y, _ = forward64(x, w, angle, rot, adjacent, eps)
    dx, dw = torch.autograd.grad((y * dy).sum(), (x, w))
    got_x, got_w, *_ = grad64(dy, x.detach(), w.detach(), angle, rot, adjacent, eps)
    assert torch.allclose(got_x, dx, rtol=1e-12, atol=1e-13)
    assert torch.allclose(got_w, dw, rtol=1e-12, atol=1e-13)

    def value(x, w):
        return float((forward64(x, w, angle, rot, adjacent, eps)[0] * dy).sum())

    x, w, h = x.detach(), w.detach(), 1e-6
    for i in range(0, x.numel(), 5):
        d = torch.zeros(x.numel(), dtype=torch.float64)
        d[i] = h
        d = d.view(x.shape)
        assert abs((value(x + d, w) - value(x - d, w)) / (2 * h) - float(got_x.flatten()[i])) < 1e-7
    for i in range(dim):
        d = torch.zeros(dim, dtype=torch.float64)
        d[i] = h
        assert abs((value(x, w + d) - value(x, w - d)) / (2 * h) - float(got_w[i])) < 1e-7


def test_rotation_keeps_lengths_and_turns_back():
    v, angle = randn((4, 3, 10), torch.float64, gen(2)), randn((4, 4), torch.float64, gen(3), 9.0)
    for adjacent in (False, True):
        y = turned(v, angle, 8, adjacent)
        assert torch.allclose(y.norm(dim=-1), v.norm(dim=-1), rtol=1e-13)
        assert torch.allclose(turned(y, -angle, 8, adjacent), v, rtol=1e-12, atol=1e-13)

"""tcu_rms_norm and tcu_rms_norm_grad at the ends of their sizes and values."""
import pytest
import torch

from layer_util import DEV, F32
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu


def test_gradient_of_columns_past_a_launch():
    """More columns than a launch of a workgroup for every 32 of them counts (2^27), so
    that the weights' gradient is walked: against binary64 on the device."""
    rows, cols = 2, (1 << 27) + 5
    g = torch.Generator(device=DEV).manual_seed(1)
    dy, h, w = (torch.randn(s, generator=g, device=DEV, dtype=torch.bfloat16)
                for s in ((rows, cols), (rows, cols), (cols,)))
    dx, dw = torch.empty_like(dy), torch.full((cols,), float("nan"), device=DEV)
    work = torch.empty(tcu.tcu_rms_norm_grad_work(rows, cols), dtype=torch.uint8, device=DEV)
    tcu.tcu_rms_norm_grad(dy, cols, h, cols, w, None, 0, dx, cols, dw, work, rows, cols, 1e-5)
    # a lane adds cols / 1024 terms of a row's sums, then trees of 16
    rel = (cols / 1024 + 16) * F32
    want, size = torch.zeros(cols, device=DEV).double(), torch.zeros(cols, device=DEV).double()
    for i in range(rows):
        hi, gi = h[i].double(), dy[i].double() * w.double()
        rstd = float((hi.pow(2).mean() + 1e-5).rsqrt())
        c = rstd ** 2 * float((gi * hi).mean())
        # |mean(g h)| is off by the sums' share of the mean of the magnitudes
        off = rstd ** 3 * float((gi * hi).abs().mean()) * rel * hi.abs()
        excess = (dx[i].double() - rstd * (gi - hi * c)).abs()
        excess -= rstd * (gi - hi * c).abs() * 2.0 ** -8 + off + rstd * (gi.abs() + hi.abs() * abs(c)) * 2 * rel
        assert float(excess.max()) <= 0
        term = dy[i].double() * hi * rstd
        want += term
        size += term.abs()
    assert bool(((dw.double() - want).abs() <= size * (rel + 4 * F32)).all())

"""tcu_rms_norm and tcu_rms_norm_grad at the ends of their sizes and values."""
import pytest
import torch

from layer_util import DEV, F32, ROUND, gen, norm64, norm_grad64, randn, within
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


def sum_bound(cols):
    """Relative error of a binary32 sum of squares and what follows it: a lane adds
    at most 64 terms of a row (of its 8192 vectors' worth), then trees."""
    return (64 + cols / 1024 + 16) * F32


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [5, 600, 1020, 3001, 9000, 17000])
def test_small_rows_without_eps(dtype, cols):
    """eps = 0 and values near 2^-66: rstd is 2^66, its square not in binary32's range."""
    g = gen(cols)
    x, dy, dh = (randn((4, cols), dtype, g) for _ in range(3))
    w = randn((cols,), dtype, g)
    x[1:3] *= 2.0 ** -66
    y, dx = (torch.empty(4, cols, dtype=dtype, device=DEV) for _ in range(2))
    tcu.tcu_rms_norm(x.to(DEV), cols, None, 0, w.to(DEV), None, 0, y, cols, None, 0, None, 4, cols,
                     0.0)
    dw = torch.empty(cols, device=DEV)
    work = torch.empty(tcu.tcu_rms_norm_grad_work(4, cols), dtype=torch.uint8, device=DEV)
    tcu.tcu_rms_norm_grad(dy.to(DEV), cols, x.to(DEV), cols, w.to(DEV), dh.to(DEV), cols, dx, cols,
                          dw, work, 4, cols, 0.0)
    # The squares near 2^-132 are multiples of 2^-149, and so is their mean: each off by
    # 2^-150, rstd by half of twice that over the mean, which is above 2^-135 here.
    low = 2.0 ** -15
    h64, y64 = norm64(x, None, w, 0.0)
    assert float(h64.pow(2).mean(1).min()) > 2.0 ** -135
    within(y, y64, y64.abs() * (ROUND[dtype] + sum_bound(cols) + low))
    x64, w64, xm, wm = norm_grad64(dy, x, w, dh, 0.0)
    within(dx, x64, x64.abs() * ROUND[dtype] + xm * (2 * sum_bound(cols) + 3 * low))
    within(dw, w64, wm * (sum_bound(cols) + 64 * F32 + low))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("cols", [5, 600, 1020, 3001, 9000, 17000])
@pytest.mark.parametrize("size,weight,eps", [(1e13, 1e27, 1e-5), (1e-20, 1e-22, 1e-38)])
def test_eight_bits_where_products_of_h_and_w_leave_the_range(dtype, cols, size, weight, eps):
    """h w near 1e40 or 1e-42, beyond binary32, and y near 1e27 or 1e-23, inside."""
    g = gen(cols)
    x, w = randn((4, cols), dtype, g, size), randn((cols,), dtype, g, weight)
    y = torch.empty(4, cols, dtype=dtype, device=DEV)
    q, s = torch.empty(4, cols, dtype=torch.int8, device=DEV), torch.empty(4, device=DEV)
    tcu.tcu_rms_norm(x.to(DEV), cols, None, 0, w.to(DEV), None, 0, y, cols, q, cols, s, 4, cols,
                     eps)
    _, y64 = norm64(x, None, w, eps)
    # squares near 1e-40 are off by 2^-150 each, of a mean whose eps is 1e-38 > 2^-127; eps is
    # rounded to a multiple of 2^-149 too
    rel = sum_bound(cols) + 2.0 ** -21
    within(y, y64, y64.abs() * (ROUND[dtype] + rel))
    top = y64.abs().amax(1)
    within(s, top / 127, top / 127 * rel)
    off = (q.cpu().double() * (top / 127)[:, None] - y64).abs()
    assert float((off - (0.5 + 127 * 4 * rel) * (top / 127)[:, None]).max()) <= 0
    assert bool((q.abs().amax(1) == 127).all())


@pytest.mark.parametrize("cols", [5, 600, 3001, 17000])
def test_eight_bits_of_a_row_that_overflows(cols):
    """Finite h and w, y beyond binary32: the row has no scale, the others have theirs."""
    g = gen(cols)
    x, w = randn((3, cols), torch.float32, g), randn((cols,), torch.float32, g)
    x[1] = 0
    x[1, 2] = cols            # the norm brings it to sqrt(cols)
    w[2] = 3e38
    x[0, 2] = x[2, 2] = 1e-4
    q, s = torch.empty(3, cols, dtype=torch.int8, device=DEV), torch.empty(3, device=DEV)
    tcu.tcu_rms_norm(x.to(DEV), cols, None, 0, w.to(DEV), None, 0, None, 0, q, cols, s, 3, cols,
                     1e-5)
    assert bool(torch.isnan(s[1])) and bool((q[1] == 0).all())
    for row in (0, 2):
        _, y64 = norm64(x[row:row + 1], None, w, 1e-5)
        top = y64.abs().amax(1)
        within(s[row:row + 1], top / 127, top / 127 * sum_bound(cols))
        assert int(q[row, 2]) == 127

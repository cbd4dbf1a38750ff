"""tcu_rms_norm and tcu_rms_norm_grad against binary64."""
import pytest
import torch

from layer_util import DEV, F32, ROUND, gen, norm64, norm_grad64, pitched, randn, untouched, within
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
EPS = 1e-5
TYPES = [torch.bfloat16, torch.float16, torch.float32]
# every way a row is held: a wave (one or two vectors a lane), a workgroup (one to
# eight), longer; whole vectors and not
COLS = [1, 7, 8, 511, 512, 1000, 1024, 1025, 2048, 4100, 8192, 9999, 16384, 16385, 40003]


def sum_bound(cols):
    """Relative error of a binary32 sum of squares and what follows it: a lane adds
    at most 64 terms of a row (of its 8192 vectors' worth), then trees."""
    return (64 + cols / 1024 + 16) * F32


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("rows,res,pad", [(1, True, 0), (5, False, 3), (9, True, 8)])
def test_norm(dtype, cols, rows, res, pad):
    g = gen(cols + rows)
    x, w = randn((rows, cols), dtype, g), randn((cols,), dtype, g)
    r = randn((rows, cols), dtype, g, 2.0) if res else None
    ld = cols + pad
    _, dx = pitched(x, ld)
    dr = pitched(r, ld)[1] if res else None
    hb, h = pitched(torch.zeros_like(x), ld)
    yb, y = pitched(torch.zeros_like(x), ld)
    qb, q = pitched(torch.zeros(rows, cols, dtype=torch.int8), ld)
    s = torch.full((rows,), -1.0, device=DEV)
    tcu.tcu_rms_norm(dx, ld, dr, ld, w.to(DEV), h, ld, y, ld, q, ld, s, rows, cols, EPS)
    h64, y64 = norm64(x, r, w, EPS)
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0     # its subnormals
    within(h, h64, h64.abs() * (ROUND[dtype] + F32) + tiny)
    rel = sum_bound(cols)
    within(y, y64, y64.abs() * (ROUND[dtype] + rel) + tiny)
    top = y64.abs().amax(1)
    within(s, top / 127, top / 127 * rel)
    # the 8-bit value is within half a step, and the largest is +-127
    q64 = q.cpu().double()
    assert float((q64 * (top / 127)[:, None] - y64).abs().sub(
        (0.5 + 127 * 4 * rel) * (top / 127)[:, None]).max()) <= 0
    assert (q64.abs().amax(1) == 127).all()
    for buf in (hb, yb, qb):
        assert untouched(buf, rows, cols, ld)


@pytest.mark.parametrize("cols", [300, 5000, 20000])
def test_norm_outputs_may_be_absent_and_in_place(cols):
    g = gen(cols)
    x, r, w = (randn(s, torch.bfloat16, g).to(DEV) for s in ((6, cols), (6, cols), (cols,)))
    h, y = torch.empty_like(x), torch.empty_like(x)
    q, s = torch.empty(6, cols, dtype=torch.int8, device=DEV), torch.empty(6, device=DEV)
    tcu.tcu_rms_norm(x, cols, r, cols, w, h, cols, y, cols, q, cols, s, 6, cols, EPS)
    for keep in range(1, 8):
        out = [torch.empty_like(t) if keep >> i & 1 else None for i, t in enumerate((h, y, q))]
        sc = torch.empty_like(s) if out[2] is not None else None
        tcu.tcu_rms_norm(x, cols, r, cols, w, out[0], cols, out[1], cols, out[2], cols, sc, 6,
                         cols, EPS)
        for a, b in zip(out + [sc], (h, y, q, s)):
            assert a is None or torch.equal(a, b)
    for into in (x, r):
        a, b = x.clone(), r.clone()
        t, y2 = (a if into is x else b), torch.empty_like(y)
        tcu.tcu_rms_norm(a, cols, b, cols, w, t, cols, y2, cols, None, 0, None, 6, cols, EPS)
        assert torch.equal(t, h) and torch.equal(y2, y)


@pytest.mark.parametrize("cols", [100, 4096, 17000])
def test_norm_special_rows(cols):
    """Zeros, values near the ends of the range, infinities and NaN: each row by itself."""
    g = gen(3)
    x, w = randn((8, cols), torch.float32, g), randn((cols,), torch.float32, g)
    x[1] = 0
    x[2, cols // 2] = float("inf")
    x[3, 0] = float("nan")
    x[4] *= 1e-30
    x[5] *= 1e15
    q, s = torch.empty(8, cols, dtype=torch.int8, device=DEV), torch.empty(8, device=DEV)
    y = torch.empty(8, cols, device=DEV)
    tcu.tcu_rms_norm(x.to(DEV), cols, None, 0, w.to(DEV), None, 0, y, cols, q, cols, s, 8, cols,
                     EPS)
    _, y64 = norm64(x, None, w, EPS)
    fine = [0, 1, 4, 5, 6, 7]
    within(y[fine], y64[fine], y64[fine].abs() * sum_bound(cols) + 2.0 ** -149)
    assert float(s[1]) == 0 and bool((q[1] == 0).all())
    for row in (2, 3):
        assert bool(torch.isnan(s[row])) and bool((q[row] == 0).all())
    assert bool((q[[0, 4, 5, 6, 7]].abs().amax(1) == 127).all())
    assert bool(torch.isnan(y[3]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("rows,dh,pad", [(1, False, 0), (7, True, 5), (1100, True, 0)])
def test_norm_grad(dtype, cols, rows, dh, pad):
    if rows > 100 and cols > 20000:
        rows = 530     # more rows than parts
    g = gen(cols + rows)
    dy, h = randn((rows, cols), dtype, g), randn((rows, cols), dtype, g, 1.5)
    w = randn((cols,), dtype, g)
    up = randn((rows, cols), dtype, g) if dh else None
    ld = cols + pad
    ddy, dhh = pitched(dy, ld)[1], pitched(h, ld)[1]
    dup = pitched(up, ld)[1] if dh else None
    xb, dx = pitched(torch.zeros_like(dy), ld)
    dw = torch.full((cols,), float("nan"), device=DEV)
    work = torch.full((tcu.tcu_rms_norm_grad_work(rows, cols) + 64,), 255, dtype=torch.uint8,
                      device=DEV)
    args = (ddy, ld, dhh, ld, w.to(DEV), dup, ld, dx, ld, dw, work, rows, cols, EPS)
    tcu.tcu_rms_norm_grad(*args)
    x64, w64, xm, wm = norm_grad64(dy, h, w, up, EPS)
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0
    within(dx, x64, x64.abs() * ROUND[dtype] + xm * 2 * sum_bound(cols) + tiny)
    within(dw, w64, wm * (sum_bound(cols) + (rows / 512 + 64) * F32))
    assert untouched(xb, rows, cols, ld)
    assert bool((work[-64:] == 255).all())
    again = dw.clone()
    tcu.tcu_rms_norm_grad(*args)
    assert torch.equal(dw, again), "another call gives other sums"


def test_norm_grad_no_rows():
    dw = torch.full((50,), 7.0, device=DEV)
    e = torch.empty(0, 50, device=DEV)
    work = torch.empty(tcu.tcu_rms_norm_grad_work(0, 50), dtype=torch.uint8, device=DEV)
    tcu.tcu_rms_norm_grad(e, 50, e, 50, torch.ones(50, device=DEV), None, 0, e, 50, dw, work, 0,
                          50, EPS)
    assert bool((dw == 0).all())


@pytest.mark.parametrize("cols", [64, 1500, 17000])
def test_norm_grad_against_differences(cols):
    """d/dt sum(y(h + t v, w + t u) dy) by central differences of the call itself."""
    g = gen(cols)
    h, dy, w, v, u = (randn(s, torch.float32, g) for s in
                      ((3, cols), (3, cols), (cols,), (3, cols), (cols,)))

    def loss(t):
        y = torch.empty(3, cols, device=DEV)
        tcu.tcu_rms_norm((h + t * v).to(DEV), cols, None, 0, (w + t * u).to(DEV), None, 0, y, cols,
                         None, 0, None, 3, cols, EPS)
        return float((y.cpu().double() * dy.double()).sum())

    t = 2.0 ** -8
    slope = (loss(t) - loss(-t)) / (2 * t)
    dx, dw = torch.empty(3, cols, device=DEV), torch.empty(cols, device=DEV)
    work = torch.empty(tcu.tcu_rms_norm_grad_work(3, cols), dtype=torch.uint8, device=DEV)
    tcu.tcu_rms_norm_grad(dy.to(DEV), cols, h.to(DEV), cols, w.to(DEV), None, 0, dx, cols, dw,
                          work, 3, cols, EPS)
    got = float((dx.cpu().double() * v.double()).sum() + (dw.cpu().double() * u.double()).sum())
    # the loss has about 3 cols terms of size 1, each with a few binary32 roundings; the
    # third derivative of a normalised value along a direction of its own size is below 30
    size = (3 * cols) ** 0.5
    assert abs(got - slope) <= size * (8 * sum_bound(cols) / t + 30 * t * t)


def test_norm_wide_offsets():
    """Rows more than 2^32 bytes apart."""
    ld, cols = (1 << 31) + 8, 3000
    g = gen(1)
    x, w = randn((3, cols), torch.bfloat16, g), randn((cols,), torch.bfloat16, g)
    buf = torch.zeros(2 * ld + cols, dtype=torch.bfloat16, device=DEV)
    view = buf.as_strided((3, cols), (ld, 1))
    view.copy_(x)
    y = torch.empty(3, cols, dtype=torch.bfloat16, device=DEV)
    tcu.tcu_rms_norm(view, ld, None, 0, w.to(DEV), view, ld, y, cols, None, 0, None, 3, cols, EPS)
    _, y64 = norm64(x, None, w, EPS)
    within(y, y64, y64.abs() * (2.0 ** -8 + sum_bound(cols)))
    assert torch.equal(view.cpu(), x)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [5, 600, 3001, 17000])
def test_zero_rows_without_eps(dtype, cols):
    """eps = 0: a row of zeros stays zero, its gradient is dh alone; others as ever."""
    g = gen(cols)
    x, w, dy, dh = (randn(s, dtype, g) for s in ((3, cols), (cols,), (3, cols), (3, cols)))
    x[1] = 0
    y = torch.empty(3, cols, dtype=dtype, device=DEV)
    q, s = torch.empty(3, cols, dtype=torch.int8, device=DEV), torch.empty(3, device=DEV)
    tcu.tcu_rms_norm(x.to(DEV), cols, None, 0, w.to(DEV), None, 0, y, cols, q, cols, s, 3, cols,
                     0.0)
    assert bool((y[1] == 0).all()) and bool((q[1] == 0).all()) and float(s[1]) == 0
    tiny = 2.0 ** -24 if dtype == torch.float16 else 0.0
    _, y64 = norm64(x[::2], None, w, 0.0)
    within(y[::2], y64, y64.abs() * (ROUND[dtype] + sum_bound(cols)) + tiny)
    dx, dw = torch.empty(3, cols, dtype=dtype, device=DEV), torch.empty(cols, device=DEV)
    work = torch.empty(tcu.tcu_rms_norm_grad_work(3, cols), dtype=torch.uint8, device=DEV)
    tcu.tcu_rms_norm_grad(dy.to(DEV), cols, x.to(DEV), cols, w.to(DEV), dh.to(DEV), cols, dx, cols,
                          dw, work, 3, cols, 0.0)
    assert torch.equal(dx[1].cpu(), dh[1])
    _, w64, _, wm = norm_grad64(dy[::2], x[::2], w, dh[::2], 0.0)
    within(dw, w64, wm * (sum_bound(cols) + 64 * F32))

"""tcu_qk_norm and tcu_qk_norm_grad against binary64.

A head's sum of squares is off by at most (dim + 4) 2^-24 of itself, its inverse root by
half of that and three roundings more; see heads_util.TURN for the rotation."""
import pytest
import torch

from heads_util import TURN, Case, bound, forward64, grad64, laid, only
from layer_util import DEV, F32 as EPS, within
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def forward(c, adjacent, eps, layout="tokens", out="tokens", in_place=False):
    _, q = laid(c.q, layout)
    _, k = laid(c.k, layout)
    qb, yq = laid(torch.zeros_like(c.q), out)
    kb, yk = laid(torch.zeros_like(c.k), out)
    if in_place:
        yq, yk = q, k
    tcu.tcu_qk_norm(q, k, *c.vectors(), yq, yk, c.T, c.hq, c.hk, c.dim, c.rot, eps,
                    tcu.TCU_ROPE_ADJACENT if adjacent else 0)
    if not in_place:
        assert only(qb, yq) and only(kb, yk)
    for y, x, w in ((yq, c.q, c.wq), (yk, c.k, c.wk)):
        want, mag = forward64(x, w, c.angle, c.rot, adjacent, eps)
        within(y, want, bound(want, mag * ((c.dim / 2 + 8) * EPS + TURN), c.dtype))
    return yq, yk


def backward(c, adjacent, eps, layout="tokens", out="tokens", over=None):
    ops = {n: laid(getattr(c, n), layout)[1] for n in ("dyq", "dyk", "q", "k")}
    qb, dq = laid(torch.zeros_like(c.q), out)
    kb, dk = laid(torch.zeros_like(c.k), out)
    if over:
        dq, dk = (ops["dyq"], ops["dyk"]) if over == "dy" else (ops["q"], ops["k"])
    dw = torch.full((2, c.dim), float("nan"), device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(c.T, c.hq, c.hk, c.dim), dtype=torch.uint8,
                       device=DEV)
    tcu.tcu_qk_norm_grad(ops["dyq"], ops["dyk"], ops["q"], ops["k"], *c.vectors(), dq, dk, dw[0],
                         dw[1], work, c.T, c.hq, c.hk, c.dim, c.rot, eps,
                         tcu.TCU_ROPE_ADJACENT if adjacent else 0)
    if not over:
        assert only(qb, dq) and only(kb, dk)
    rel = (c.dim + 20) * EPS + TURN
    for d, w, dy, x, weight, H in ((dq, dw[0], c.dyq, c.q, c.wq, c.hq),
                                   (dk, dw[1], c.dyk, c.k, c.wk, c.hk)):
        dx64, dw64, xm, wm = grad64(dy, x, weight, c.angle, c.rot, adjacent, eps)
        within(d, dx64, bound(dx64, xm * 2 * rel, c.dtype))
        within(w, dw64, wm * (rel + c.T * H * EPS))
    return dq, dk, dw


SIZES = [  # tokens, hq, hk, dim, rot
    (1, 1, 1, 1, 0), (1, 32, 8, 128, 128), (3, 2, 1, 2, 2), (5, 3, 2, 7, 4), (4, 5, 5, 16, 16),
    (7, 4, 1, 32, 16), (9, 6, 2, 64, 64), (13, 3, 1, 80, 40), (6, 15, 5, 80, 80), (10, 4, 4, 96, 48),
    (11, 5, 1, 100, 100), (11, 5, 1, 100, 50), (8, 2, 2, 128, 64), (3, 9, 3, 129, 128),
    (5, 7, 1, 192, 192), (4, 3, 3, 250, 90), (6, 2, 1, 256, 256), (3, 2, 2, 300, 4),
    (2, 3, 1, 512, 512), (3, 1, 2, 577, 96), (2, 2, 2, 1024, 1024), (2, 1, 1, 1023, 1022),
    (300, 8, 2, 64, 32), (2100, 3, 1, 128, 128)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("adjacent", [False, True])
def test_forward(dtype, size, adjacent):
    c = Case(*size, dtype)
    forward(c, adjacent, 1e-6)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("adjacent", [False, True])
def test_backward(dtype, size, adjacent):
    c = Case(*size, dtype)
    backward(c, adjacent, 1e-6)


@pytest.mark.parametrize("layout,out", [("tokens", "heads"), ("heads", "tokens"),
                                        ("padded", "padded"), ("padded", "heads")])
@pytest.mark.parametrize("size", [(5, 4, 2, 128, 128), (6, 3, 1, 80, 40), (4, 2, 2, 33, 20),
                                  (1, 3, 2, 64, 64), (7, 1, 1, 64, 64)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(layout, out, size, dtype):
    c = Case(*size, dtype)
    forward(c, False, 1e-6, layout, out)
    backward(c, False, 1e-6, layout, out)


@pytest.mark.parametrize("size", [(5, 4, 2, 128, 128), (4, 2, 2, 33, 20), (3, 1, 1, 300, 300)])
@pytest.mark.parametrize("adjacent", [False, True])
@pytest.mark.parametrize("layout", ["tokens", "heads", "padded"])
def test_in_place(size, adjacent, layout):
    c = Case(*size, BF16)
    a, b = forward(c, adjacent, 1e-6, layout), forward(c, adjacent, 1e-6, layout, in_place=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    a = backward(c, adjacent, 1e-6, layout)
    for over in ("dy", "x"):
        b = backward(c, adjacent, 1e-6, layout, over=over)
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("adjacent", [False, True])
def test_views_of_packed_rows(adjacent):
    """Queries and keys in place in rows that hold the values too, which stay as they are."""
    c = Case(17, 6, 2, 64, 64, BF16)
    qkv = torch.cat((c.q, c.k, torch.full((17, 2, 64), 3.0, dtype=BF16)), 1).to(DEV)
    q, k = qkv[:, :6], qkv[:, 6:8]
    tcu.tcu_qk_norm(q, k, *c.vectors(), q, k, 17, 6, 2, 64, 64, 1e-6, int(adjacent))
    yq, yk = forward(c, adjacent, 1e-6)
    assert torch.equal(q, yq) and torch.equal(k, yk)
    assert bool((qkv[:, 8:] == 3).all())


@pytest.mark.parametrize("T", [1, 40])
def test_far_positions(T):
    """Angles of positions over all of int32, in binary32 outputs."""
    c = Case(T, 4, 2, 128, 128, F32, far=True)
    c.pos[0] = -2 ** 31
    c.pos[-1] = 2 ** 31 - 1
    c.angle = c.pos.double()[:, None] * c.freq.double()
    forward(c, False, 1e-6)
    backward(c, False, 1e-6)


@pytest.mark.parametrize("one", ["q", "k"])
def test_queries_or_keys_alone(one):
    c = Case(9, 5 if one == "q" else 0, 0 if one == "q" else 3, 64, 32, BF16)
    wq, wk, freq, pos = c.vectors()
    x, w, dy = (c.q, wq, c.dyq) if one == "q" else (c.k, wk, c.dyk)
    x, dy = x.to(DEV), dy.to(DEV)
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(64, device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(9, c.hq, c.hk, 64), dtype=torch.uint8, device=DEV)
    pair = (lambda t: (t, None)) if one == "q" else (lambda t: (None, t))
    tcu.tcu_qk_norm(*pair(x), *pair(w), freq, pos, *pair(y), 9, c.hq, c.hk, 64, 32, 1e-6)
    tcu.tcu_qk_norm_grad(*pair(dy), *pair(x), *pair(w), freq, pos, *pair(dx), *pair(dw), work, 9,
                         c.hq, c.hk, 64, 32, 1e-6)
    want, mag = forward64(x.cpu(), w.cpu(), c.angle, 32, False, 1e-6)
    within(y, want, bound(want, mag * (40 * EPS + TURN), BF16))
    dx64, dw64, xm, wm = grad64(dy.cpu(), x.cpu(), w.cpu(), c.angle, 32, False, 1e-6)
    within(dx, dx64, bound(dx64, xm * 2 * (84 * EPS + TURN), BF16))
    within(dw, dw64, wm * (130 * EPS + TURN))


def test_no_rotation_needs_no_tables():
    c = Case(6, 3, 1, 64, 0, BF16)
    q, k = c.q.to(DEV), c.k.to(DEV)
    yq, yk = torch.empty_like(q), torch.empty_like(k)
    tcu.tcu_qk_norm(q, k, c.wq.to(DEV), c.wk.to(DEV), None, None, yq, yk, 6, 3, 1, 64, 0, 1e-6)
    want, _ = forward64(c.q, c.wq, c.angle, 0, False, 1e-6)
    within(yq, want, bound(want, want.abs() * 50 * EPS, BF16))


@pytest.mark.parametrize("dim", [64, 50])
def test_zero_heads_and_heads_that_are_not_finite(dim):
    """A head of zeros without an eps has zeros; NaN and infinity stay in their head."""
    c = Case(6, 3, 1, dim, dim, F32)
    clean = [t.cpu() for t in forward(c, False, 0.0)]
    cdx = [t.cpu() for t in backward(c, False, 0.0)]
    q = c.q.clone()
    q[1, 2] = 0
    q[2, 0, 5] = float("inf")
    q[4, 1, 3] = float("nan")
    dq, k = q.to(DEV), c.k.to(DEV)
    yq, yk = torch.empty_like(dq), torch.empty_like(k)
    tcu.tcu_qk_norm(dq, k, *c.vectors(), yq, yk, 6, 3, 1, dim, dim, 0.0)
    yq = yq.cpu()
    assert bool((yq[1, 2] == 0).all()) and bool(torch.isnan(yq[2, 0, 5]))
    assert bool(torch.isnan(yq[4, 1]).all())
    keep = torch.ones(6, 3, dtype=torch.bool)
    keep[1, 2] = keep[2, 0] = keep[4, 1] = False
    assert torch.equal(yq[keep], clean[0][keep]) and torch.equal(yk.cpu(), clean[1])
    dx, dk = torch.empty_like(dq), torch.empty_like(k)
    dw = torch.empty(2, dim, device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(6, 3, 1, dim), dtype=torch.uint8, device=DEV)
    tcu.tcu_qk_norm_grad(c.dyq.to(DEV), c.dyk.to(DEV), dq, k, *c.vectors(), dx, dk, dw[0], dw[1],
                         work, 6, 3, 1, dim, dim, 0.0)
    dx = dx.cpu()
    assert bool((dx[1, 2] == 0).all()) and bool(torch.isnan(dx[4, 1]).all())
    assert torch.equal(dx[keep], cdx[0][keep]) and torch.equal(dk.cpu(), cdx[1])
    assert bool(torch.isnan(dw[0]).all()) and torch.equal(dw[1].cpu(), cdx[2][1])


def test_no_tokens():
    """The weights' gradients of no tokens are zeros."""
    e = torch.empty(0, 3, 32, dtype=BF16, device=DEV)
    w = torch.ones(32, dtype=BF16, device=DEV)
    f, p = torch.ones(16, device=DEV), torch.empty(0, dtype=torch.int32, device=DEV)
    dw = torch.full((2, 32), float("nan"), device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(0, 3, 3, 32), dtype=torch.uint8, device=DEV)
    tcu.tcu_qk_norm(e, e, w, w, f, p, e.clone(), e.clone(), 0, 3, 3, 32, 32, 1e-6)
    tcu.tcu_qk_norm_grad(e, e, e, e, w, w, f, p, e.clone(), e.clone(), dw[0], dw[1], work, 0, 3, 3,
                         32, 32, 1e-6)
    assert bool((dw == 0).all())

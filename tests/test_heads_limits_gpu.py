"""tcu_qk_norm and tcu_qk_norm_grad at the ends of their sizes and values: many tokens (several
to a wave), values that are not finite among them, ends of binary32's range, pitches past
2^31 elements, the same bits on every call."""
import pytest
import torch

from heads_util import Case, angles, bound, forward64, TURN
from layer_util import DEV, F32 as EPS, within
from paper_1908_06649_amd import tcu
from test_heads_gpu import backward, forward

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32

MANY = [(4097, 15, 3, 128, 128), (9001, 3, 1, 64, 64), (20011, 2, 1, 16, 8), (8200, 5, 2, 80, 40),
        (17000, 1, 1, 7, 4), (12289, 3, 2, 48, 48), (33000, 1, 2, 32, 0)]


@pytest.mark.parametrize("size", MANY)
@pytest.mark.parametrize("dtype,adjacent", [(BF16, False), (F16, True), (F32, False)])
def test_many_tokens(size, dtype, adjacent):
    c = Case(*size, dtype)
    forward(c, adjacent, 1e-6, layout="padded", out="heads")
    backward(c, adjacent, 1e-6)


def outputs(c, q, k, dyq, dyk):
    q, k, dyq, dyk = (t.to(DEV) for t in (q, k, dyq, dyk))
    yq, yk, dq, dk = (torch.empty_like(t) for t in (q, k, q, k))
    dw = torch.empty(2, c.dim, device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(c.T, c.hq, c.hk, c.dim), dtype=torch.uint8,
                       device=DEV)
    tcu.tcu_qk_norm(q, k, *c.vectors(), yq, yk, c.T, c.hq, c.hk, c.dim, c.rot, 1e-6)
    tcu.tcu_qk_norm_grad(dyq, dyk, q, k, *c.vectors(), dq, dk, dw[0], dw[1], work, c.T, c.hq, c.hk,
                         c.dim, c.rot, 1e-6)
    return [t.cpu() for t in (yq, yk, dq, dk, dw[0], dw[1])]


@pytest.mark.parametrize("size", [(9001, 2, 1, 64, 64), (9001, 3, 3, 16, 16), (3, 2, 2, 50, 50),
                                  (9000, 1, 2, 20, 20)])
def test_values_that_are_not_finite_stay_in_their_heads(size):
    """Also where a wave holds queries and keys of several tokens at once: the other weights'
    gradients are the clean ones' bits."""
    c = Case(*size, F32)
    clean = outputs(c, c.q, c.k, c.dyq, c.dyk)
    q, dyq = c.q.clone(), c.dyq.clone()
    hit = torch.zeros(c.T, c.hq, dtype=torch.bool)
    for t, v in ((1, float("nan")), (c.T // 2, float("inf")), (c.T - 1, float("nan"))):
        q[t, t % c.hq, t % c.dim] = v
        hit[t, t % c.hq] = True
    y = outputs(c, q, c.k, dyq, c.dyk)
    assert torch.equal(y[0][~hit], clean[0][~hit]) and not torch.isfinite(y[0][hit]).all(-1).any()
    assert torch.equal(y[2][~hit], clean[2][~hit]) and bool(torch.isnan(y[4]).any())
    assert all(torch.equal(y[i], clean[i]) for i in (1, 3, 5))
    # and in the keys' gradient
    dyk = c.dyk.clone()
    dyk[c.T // 3, 0] = float("nan")
    y = outputs(c, c.q, c.k, c.dyq, dyk)
    assert all(torch.equal(y[i], clean[i]) for i in (0, 1, 2, 4))
    assert bool(torch.isnan(y[3][c.T // 3, 0]).all()) and bool(torch.isnan(y[5]).all())


def test_ends_of_the_range():
    """Without an eps: squares' sums past binary32's range and below it make a head's outputs
    and gradients 0, the heads beside it as they are."""
    c = Case(6, 2, 1, 64, 64, F32)
    q = c.q.clone()
    q[0, 0], q[1, 1], q[2, 0] = 1e25, 1e-30, -3e38
    q, k = q.to(DEV), c.k.to(DEV)
    outs = [torch.full_like(t, float("nan")) for t in (q, k, q, k)]
    dw = torch.empty(2, 64, device=DEV)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(6, 2, 1, 64), dtype=torch.uint8, device=DEV)
    tcu.tcu_qk_norm(q, k, *c.vectors(), outs[0], outs[1], 6, 2, 1, 64, 64, 0.0)
    tcu.tcu_qk_norm_grad(c.dyq.to(DEV), c.dyk.to(DEV), q, k, *c.vectors(), outs[2], outs[3], dw[0],
                         dw[1], work, 6, 2, 1, 64, 64, 0.0)
    for t in (outs[0], outs[2]):
        for at in ((0, 0), (1, 1), (2, 0)):
            assert bool((t[at] == 0).all())
    assert all(bool(torch.isfinite(t).all()) for t in (*outs, dw))
    keep = torch.ones(6, 2, dtype=torch.bool)
    keep[0, 0] = keep[1, 1] = keep[2, 0] = False
    want, mag = forward64(c.q, c.wq, c.angle, 64, False, 0.0)
    within(outs[0].cpu()[keep], want[keep], bound(want, mag * (40 * EPS + TURN), F32)[keep])


def test_pitches_past_31_bits():
    """Tokens 2^31 elements apart, read and written."""
    c = Case(2, 2, 1, 64, 64, BF16)
    ld = 2 ** 31 + 64
    buf = torch.empty(ld + 256, dtype=BF16, device=DEV)
    q, k = buf.as_strided((2, 2, 64), (ld, 64, 1)), buf.as_strided((2, 1, 64), (ld, 64, 1), 128)
    q.copy_(c.q)
    k.copy_(c.k)
    yq, yk = torch.empty(2, 2, 64, dtype=BF16, device=DEV), torch.empty(2, 1, 64, dtype=BF16, device=DEV)
    tcu.tcu_qk_norm(q, k, *c.vectors(), yq, yk, 2, 2, 1, 64, 64, 1e-6)
    tcu.tcu_qk_norm(q, k, *c.vectors(), q, k, 2, 2, 1, 64, 64, 1e-6)
    assert torch.equal(q, yq) and torch.equal(k, yk)
    want, mag = forward64(c.q, c.wq, c.angle, 64, False, 1e-6)
    within(yq, want, bound(want, mag * (40 * EPS + TURN), BF16))


def test_the_same_bits_on_every_call():
    c = Case(3001, 6, 2, 96, 96, BF16)
    first = outputs(c, c.q, c.k, c.dyq, c.dyk)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(outputs(c, c.q, c.k, c.dyq, c.dyk), first))


def test_the_same_head_in_both_places():
    """Two weights of one tensor, queries and keys one tensor: allowed where only outputs must
    be apart."""
    c = Case(33, 2, 2, 64, 64, BF16)
    q = c.q.to(DEV)
    wq, wk, f, p = c.vectors()
    yq, yk = torch.empty_like(q), torch.empty_like(q)
    tcu.tcu_qk_norm(q, q, wq, wq, f, p, yq, yk, 33, 2, 2, 64, 64, 1e-6)
    assert torch.equal(yq, yk)
    want, mag = forward64(c.q, c.wq, angles(c.pos, c.freq), 64, False, 1e-6)
    within(yq, want, bound(want, mag * (40 * EPS + TURN), BF16))

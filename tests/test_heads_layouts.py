"""Where the heads' norms' outputs may lie (fake pointers that are never dereferenced): between
other operands' heads, as in packed rows of each head's query, key and value, but never on a
byte of another operand."""
import random

import pytest
import torch

from paper_1908_06649_amd import tcu
from test_mx4_abi import CALLS, OVER, P, QK, QKG

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="valid arguments with fake pointers")
FREE = tcu.TCU_ERR_NO_DEVICE       # every argument check passed
D = 64


def packed(kind, T, H, each=3, more=0):
    """(pitch of tokens, pitch of heads, elements of the buffer) of `each` operands' heads side
    by side: token by token, or head by head."""
    if kind == "tokens":
        return H * each * D + more, each * D, T * (H * each * D + more)
    return each * D, T * each * D + more, H * (T * each * D + more)


def forward(q, k, yq, yk, T, hq, hk):
    """q .. yk: (address, pitch of tokens, pitch of heads)."""
    change = {}
    for n, (p, ld, hd) in dict(q=q, k=k, yq=yq, yk=yk).items():
        change.update({n: p, "ld" + n: ld, "hd" + n: hd})
    return getattr(tcu.lib(), QK)(*{**CALLS[QK], **change, "tokens": T, "hq": hq, "hk": hk}.values())


def backward(dyq, dyk, q, k, dq, dk, T, hq, hk):
    change = {}
    for n, (p, ld, hd) in dict(dyq=dyq, dyk=dyk, q=q, k=k, dq=dq, dk=dk).items():
        change.update({n: p, "ld" + n: ld, "hd" + n: hd})
    return getattr(tcu.lib(), QKG)(*{**CALLS[QKG], **change, "tokens": T, "hq": hq,
                                     "hk": hk}.values())


def parts(base, layout, *which):
    return [(base + 2 * D * i, *layout[:2]) for i in which]


@pytest.mark.parametrize("kind", ["tokens", "heads"])
@pytest.mark.parametrize("T,H", [(1, 4), (7, 4), (7, 1), (2, 2)])
@pytest.mark.parametrize("each,more", [(2, 0), (3, 0), (3, 5)])
def test_packed_heads(kind, T, H, each, more):
    at = packed(kind, T, H, each, more)
    q, k = parts(P[0], at, 0, 1)
    yq, yk = parts(P[5], at, 0, 1)
    assert forward(q, k, q, k, T, H, H) == FREE
    assert forward(q, k, yq, yk, T, H, H) == FREE
    assert forward(q, k, yk, yq, T, H, H) == FREE
    dq, dk = parts(P[6], at, 0, 1)
    assert backward(q, k, yq, yk, dq, dk, T, H, H) == FREE
    assert backward(q, k, yq, yk, q, k, T, H, H) == FREE
    assert backward(q, k, yq, yk, yq, yk, T, H, H) == FREE
    # one value to the side, and each other's places
    side = (k[0] - 2, *k[1:])
    assert forward(q, k, yq, (yk[0] - 2, *yk[1:]), T, H, H) == OVER
    assert forward(q, k, q, side, T, H, H) == OVER
    assert forward(q, k, k, q, T, H, H) == OVER
    assert backward(q, k, yq, yk, dq, (dk[0] - 2, *dk[1:]), T, H, H) == OVER
    assert backward(q, k, yq, yk, k, dk, T, H, H) == OVER


@pytest.mark.parametrize("T,hq,hk", [(7, 4, 1), (7, 4, 2), (1, 4, 1), (5, 1, 1)])
@pytest.mark.parametrize("more", [0, 5])
def test_fewer_keys(T, hq, hk, more):
    """Queries and keys in rows, or one after the other head by head, beside values."""
    rows = (hq + 2 * hk) * D + more
    q, k = (P[0], rows, D), (P[0] + 2 * hq * D, rows, D)
    assert forward(q, k, q, k, T, hq, hk) == FREE
    assert forward(q, k, q, (k[0] - 2, *k[1:]), T, hq, hk) == OVER
    # each head's tokens, a query (or key) and something else in turn
    q, k = (P[0], 2 * D, T * 2 * D + more), (P[0] + 2 * D, 2 * D, T * 2 * D + more)
    assert forward(q, k, q, k, T, hq, hk) == FREE
    assert forward(q, k, q, (k[0] - 2, *k[1:]), T, hq, hk) == OVER


def bytes_of(p, ld, hd, T, H, dim, es):
    return {p + (t * ld + h * hd) * es + b for t in range(T) for h in range(H)
            for b in range(dim * es)}


def nested(rng, T, H, dim):
    """Pitches of tokens and heads that do not run into each other."""
    inner = dim + rng.choice([0, 0, 1, dim, 2 * dim])
    n, m = (H, T) if rng.random() < 0.5 else (T, H)
    outer = (n - 1) * inner + dim + rng.choice([0, inner - dim, inner - dim, 1, dim, inner + 3])
    return (outer, inner) if n == H else (inner, outer)


def test_against_every_byte():
    """Small layouts: what shares a byte is refused, and of equal pitches nothing else."""
    rng = random.Random(5)
    seen = {FREE: 0, OVER: 0}
    for _ in range(20000):
        T, hq, hk, dim = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 3)
        at = nested(rng, T, max(hq, hk), dim)
        same = rng.random() < 0.7
        to = at if same else nested(rng, T, max(hq, hk), dim)
        yk = P[0] + 2 * rng.randint(-30, 60)
        q, y = bytes_of(P[0], *at, T, hq, dim, 2), bytes_of(yk, *to, T, hk, dim, 2)
        change = dict(q=P[0], ldq=at[0], hdq=at[1], yk=yk, ldyk=to[0], hdyk=to[1], k=P[7], ldk=9999,
                      hdk=99, yq=P[8], ldyq=9999, hdyq=99, tokens=T, hq=hq, hk=hk, dim=dim, rot=0)
        got = getattr(tcu.lib(), QK)(*{**CALLS[QK], **change}.values())
        want = OVER if q & y else FREE
        if want == OVER or same:
            assert got == want, (change, sorted(q & y))
        else:
            assert got in (FREE, OVER)
        seen[want] += 1
    assert min(seen.values()) > 3000


def test_vectors_against_every_byte():
    """A gradient of the weights anywhere about an operand's heads."""
    rng = random.Random(6)
    seen = {FREE: 0, OVER: 0}
    for _ in range(10000):
        T, hq, dim = rng.randint(1, 5), rng.randint(1, 4), rng.randint(1, 3)
        ld, hd = nested(rng, T, hq, dim)
        dw = P[0] + 4 * rng.randint(-8, 40)
        change = dict(q=P[0], ldq=ld, hdq=hd, dyq=P[1], lddyq=ld, hddyq=hd, dq=P[2], lddq=ld, hddq=hd,
                      hk=0, k=0, dyk=0, dk=0, wk=0, dwk=0, wq=P[3], dwq=dw, work=P[6], tokens=T, hq=hq,
                      dim=dim, rot=0)
        got = getattr(tcu.lib(), QKG)(*{**CALLS[QKG], **change}.values())
        shared = bytes_of(P[0], ld, hd, T, hq, dim, 2) & set(range(dw, dw + 4 * dim))
        assert got == OVER if shared else got in (FREE, OVER), change
        seen[got] += 1
    assert min(seen.values()) > 2000

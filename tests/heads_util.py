"""Norms of queries and keys with rotation in binary64, their magnitudes, and seeded
operands in the layouts that the tests use."""
import torch

from layer_util import DEV, ROUND, gen, randn

# Binary32 rotation: a share of a turn is at most 1/2 and rounded once (2^-26 of a turn,
# 2^-23.3 of an angle), sine and cosine are within 2 units of 2^-24, two products and
# their sum round three times: together below 2^-21 of |a| + |b|.
TURN = 2.0 ** -21


def bound(want, err, dtype):
    """What a result may be off that is within err of want before it is rounded once: half a
    step relative to the value that is rounded, and binary16's values below 2^-14 are
    multiples of 2^-24, so half of that."""
    return err + (want.abs() + err) * ROUND[dtype] + (2.0 ** -25 if dtype == torch.float16 else 0)


def partner(v, rot, adjacent):
    """The other element of every rotated pair, 0 elsewhere."""
    p = torch.zeros_like(v)
    if adjacent:
        p[..., 0:rot:2], p[..., 1:rot:2] = v[..., 1:rot:2], v[..., 0:rot:2]
    else:
        p[..., :rot // 2], p[..., rot // 2:rot] = v[..., rot // 2:rot], v[..., :rot // 2]
    return p


def turned(v, angle, rot, adjacent):
    """v (tokens x heads x dim, binary64) with its pairs turned (angle: tokens x rot/2)."""
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    rest = v[..., rot:]
    if adjacent:
        a, b = v[..., 0:rot:2], v[..., 1:rot:2]
        y = torch.stack((a * c - b * s, a * s + b * c), -1).flatten(-2)
    else:
        a, b = v[..., :rot // 2], v[..., rot // 2:rot]
        y = torch.cat((a * c - b * s, a * s + b * c), -1)
    return torch.cat((y, rest), -1)


def forward64(x, w, angle, rot, adjacent, eps):
    """(y, v's magnitude with its partner's)."""
    x = x.double()
    v = x / (x.pow(2).mean(-1, keepdim=True) + eps).sqrt() * w.double()
    return turned(v, angle, rot, adjacent), v.abs() + partner(v.abs(), rot, adjacent)


def grad64(dy, x, w, angle, rot, adjacent, eps):
    """dx, dw and the magnitudes of what their sums are made of."""
    x, w, dy = x.double(), w.double(), dy.double()
    rstd = (x.pow(2).mean(-1, keepdim=True) + eps).rsqrt()
    n = x * rstd
    dv, dvm = turned(dy, -angle, rot, adjacent), dy.abs() + partner(dy.abs(), rot, adjacent)
    g, gm = dv * w, dvm * w.abs()
    dx = rstd * (g - n * (g * n).mean(-1, keepdim=True))
    xm = rstd * (gm + n.abs() * (gm * n.abs()).mean(-1, keepdim=True))
    return dx, (dv * n).sum((0, 1)), xm, (dvm * n.abs()).sum((0, 1))


def angles(pos, freq):
    return pos.double()[:, None] * freq.double()


class Case:
    """Seeded operands on the host: q, k, weights, positions, frequencies, gradients."""

    def __init__(self, T, hq, hk, dim, rot, dtype, seed=0, far=False):
        g = gen(seed + T + hq * 7 + dim)
        self.T, self.hq, self.hk, self.dim, self.rot, self.dtype = T, hq, hk, dim, rot, dtype
        self.q, self.k = (randn((T, h, dim), dtype, g, 1.5) for h in (hq, hk))
        self.dyq, self.dyk = (randn((T, h, dim), dtype, g) for h in (hq, hk))
        self.wq, self.wk = (randn((dim,), dtype, g) for _ in range(2))
        i = torch.arange(0, rot, 2, dtype=torch.float64)
        self.freq = (10000.0 ** (-i / max(rot, 1))).float()
        lo, hi = (-2 ** 31, 2 ** 31) if far else (0, 5000)
        self.pos = torch.randint(lo, hi, (T,), generator=g).to(torch.int32)
        self.angle = angles(self.pos, self.freq)

    def vectors(self):
        return tuple(t.to(DEV) for t in (self.wq, self.wk, self.freq, self.pos))


def laid(t, layout, fill=float("nan")):
    """(buffer, device view of t): "tokens" contiguous, "heads" head by head, "padded" with
    pitches that nothing is a multiple of, the rest of the buffer filled."""
    T, H, D = t.shape
    if layout == "tokens":
        ld, hd = H * D, D
    elif layout == "heads":
        ld, hd = D, T * D
    else:
        hd = D + 3
        ld = H * hd + 5
    n = max(T - 1, 0) * ld + max(H - 1, 0) * hd + D if T and H else 0
    buf = torch.full((n + 11,), fill, dtype=t.dtype, device=DEV)
    v = buf[1 if layout == "padded" else 0:].as_strided((T, H, D), (ld, hd, 1),
                                                        1 if layout == "padded" else 0)
    v.copy_(t)
    return buf, v


def only(buf, view, fill=float("nan")):
    """Whether everything of the buffer outside the view is as filled."""
    b = buf.clone()
    b.as_strided(view.shape, view.stride(), view.storage_offset()).fill_(fill)
    return bool(torch.isnan(b).all())

"""The 4-bit format in binary64 from its definition, on the host, and device buffers in
it for the tests."""
import math

import torch

from layer_util import DEV

MAG = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def groups(n):
    return -(-n // 128)


def quant64(x):
    """(codes: rows x 128 groups int64, scale bytes: rows x 4 groups int64) of x's rows."""
    rows, cols = x.shape
    v = torch.zeros(rows, groups(cols) * 128, dtype=torch.float64)
    v[:, :cols] = x.double()
    v = v.view(rows, -1, 32)
    bad = ~torch.isfinite(v).all(2, keepdim=True)
    v = torch.where(bad, 0.0, v)
    amax = v.abs().amax(2, keepdim=True)
    # frexp is exact: amax = m 2^e with m in [1/2, 1), so floor(log2 amax) = e - 1
    e = torch.where(amax > 0, torch.frexp(amax).exponent.double() - 1 - 2, -127.0)
    e = e.clamp(min=-127)
    u = v / torch.exp2(e)
    # the nearest magnitude, of two equally near ones that of the even code
    d = (u.abs()[..., None] - MAG).abs()
    best = d.amin(-1, keepdim=True)
    near = d == best
    even = near & (torch.arange(8) % 2 == 0)
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = code + torch.where(torch.signbit(v) , 8, 0)
    code = torch.where(bad, 0, code)
    byte = torch.where(bad, 255, (e + 127).long())[..., 0]
    return code.view(rows, -1), byte


def value64(codes, byte):
    """What codes and scale bytes stand for."""
    rows = codes.shape[0]
    v = MAG[codes & 7] * torch.where(codes >= 8, -1.0, 1.0).double()
    s = torch.where(byte == 255, math.nan, torch.exp2(byte.double() - 127))
    return (v.view(rows, -1, 32) * s[..., None]).view(rows, -1)


def rounded64(x):
    return value64(*quant64(x))[:, :x.shape[1]]


def pack(codes, byte):
    """Codes and bytes as the library holds them: uint8 rows, int32 words group by group."""
    rows = codes.shape[0]
    c = codes.to(torch.uint8).view(rows, -1, 2)
    q = (c[..., 0] | (c[..., 1] << 4)).contiguous()
    return q, byte.to(torch.uint8).contiguous().view(torch.int32).t().contiguous()


def unpack(q, words):
    """The inverse of pack."""
    q, rows = q.cpu(), q.shape[0]
    codes = torch.stack((q & 15, q >> 4), 2).view(rows, -1).long()
    byte = (words.cpu().t()[:, :, None] >> torch.tensor([0, 8, 16, 24])) & 255
    byte = byte.reshape(rows, -1).long()
    return codes, byte


class Held:
    """A matrix in 4 bits on the device, in buffers of larger pitches filled with 0x71."""

    def __init__(self, rows, cols, codes=None, byte=None, more=16, more_words=3):
        g = groups(cols)
        self.rows, self.cols, self.ld, self.lds = rows, cols, 64 * g + more, rows + more_words
        self.qbuf = torch.full((rows * self.ld + 64,), 113, dtype=torch.uint8, device=DEV)
        self.sbuf = torch.full((g * self.lds + 16,), 113, dtype=torch.int32, device=DEV)
        self.q = self.qbuf[:rows * self.ld].view(rows, self.ld)[:, :64 * g]
        self.s = self.sbuf[:g * self.lds].view(g, self.lds)[:, :rows]
        if codes is not None:
            q, s = pack(codes, byte)
            self.q.copy_(q)
            self.s.copy_(s)

    def untouched(self):
        a, b = self.qbuf.clone(), self.sbuf.clone()
        g = groups(self.cols)
        a[:self.rows * self.ld].view(self.rows, self.ld)[:, :64 * g] = 113
        b[:g * self.lds].view(g, self.lds)[:, :self.rows] = 113
        return bool((a == 113).all()) and bool((b == 113).all())

    def args(self):
        return self.q, self.ld, self.s, self.lds

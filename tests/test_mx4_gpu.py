"""tcu_mx4_quant, tcu_mx4_dequant: exact against the format's definition."""
import pytest
import torch

from layer_util import DEV, gen, pitched, randn, untouched
from mx4_util import Held, groups, quant64, rounded64, unpack, value64
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def quantise(x, along=True, across=True, pad=0):
    """x (on the host) through the library; checks that nothing else is written."""
    rows, cols = x.shape
    buf, v = pitched(x, cols + pad)
    a, b = Held(rows, cols), Held(cols, rows)
    tcu.tcu_mx4_quant(v, cols + pad, *(a.args() if along else (None, 0, None, 0)),
                      *(b.args() if across else (None, 0, None, 0)), rows, cols)
    assert a.untouched() and b.untouched()
    return a, b


def same(held, x):
    codes, byte = unpack(held.q, held.s)
    want_codes, want_byte = quant64(x)
    assert torch.equal(byte, want_byte), "scales differ"
    # (the sign of a zero is x's)
    assert torch.equal(codes, want_codes), "codes differ"


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 32), (2, 33), (5, 127), (31, 129), (64, 512),
                                       (129, 640), (257, 1003), (1, 4096), (1000, 7)])
@pytest.mark.parametrize("pad", [0, 3])
def test_quant(dtype, rows, cols, pad):
    x = randn((rows, cols), dtype, gen(rows * cols))
    x *= torch.exp2(torch.randint(-9, 6, (rows, 1), generator=gen(3))).to(dtype)
    a, b = quantise(x, pad=pad)
    same(a, x)
    same(b, x.t())
    one, _ = quantise(x, across=False, pad=pad)
    _, other = quantise(x, along=False, pad=pad)
    assert torch.equal(one.q, a.q) and torch.equal(one.s, a.s)
    assert torch.equal(other.q, b.q) and torch.equal(other.s, b.s)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_every_value(dtype):
    """Every 16-bit pattern, beside the largest of its block from the same exponent to 2^6
    times that, and in any order (so NaN and infinities spoil some blocks)."""
    bits = torch.arange(-32768, 32768).to(torch.int16)
    x = bits.view(dtype)
    finite = x[torch.isfinite(x)]
    parts = []
    for k in range(7):
        n = len(finite) // 31 * 31
        v = finite[torch.randperm(len(finite), generator=gen(k))[:n]]
        order = v.abs().double().sort().indices
        v = v[order].view(-1, 31)        # blocks of neighbours
        top = (v.abs().double().amax(1, keepdim=True) * 2.0 ** k).to(dtype)
        top = torch.where(torch.isfinite(top), top, v.abs().amax(1, keepdim=True))
        parts.append(torch.cat((v, top), 1))
    parts.append(x[torch.randperm(65536, generator=gen(9))].view(-1, 32))
    x = torch.cat(parts)
    a, b = quantise(x)
    same(a, x)
    same(b, x.t())


def test_half_way_and_tiny_values_in_binary32():
    """Values on and next to every border between two codes, at scales from the smallest to
    the largest; subnormal ones among them; NaN, infinities and zeros."""
    mids = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=torch.float64)
    rows = []
    for e in (-127, -126, -125, -110, -96, -95, -94, -30, -1, 0, 1, 50, 125):
        s = 2.0 ** e
        v = [m * s * f for m in mids.tolist() for f in (1, 1 - 2.0 ** -20, 1 + 2.0 ** -20, -1)]
        v = torch.tensor(v + [4.0 * s, 6.0 * s, 7.5 * s, -7.999 * s], dtype=torch.float64)
        assert len(v) == 32
        rows.append(v.to(F32))
    tiny = torch.full((32,), 2.0 ** -149)
    tiny[::3] = 0
    tiny[5] = -3 * 2.0 ** -149
    odd = torch.zeros(32, dtype=F32)
    odd[1] = -0.0
    odd[2] = 0.0
    nan, inf = torch.ones(32), torch.ones(32)
    nan[17] = float("nan")
    inf[3] = -float("inf")
    huge = torch.full((32,), torch.finfo(F32).max)
    x = torch.stack(rows + [tiny, odd, nan, inf, huge])
    a, b = quantise(x)
    same(a, x)
    same(b, x.t())
    y = torch.empty(x.shape, device=DEV)
    tcu.tcu_mx4_dequant(*a.args(), y, 32, *x.shape)
    assert torch.equal(torch.nan_to_num(y.cpu().double(), nan=-1),
                       torch.nan_to_num(rounded64(x), nan=-1))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_dequant_of_every_code_and_scale(dtype):
    """256 scale bytes x 16 codes, rounded once to the output's type (binary16 to its
    infinity or zero where the value is out of its range)."""
    codes = torch.arange(16).repeat(256, 2)
    byte = torch.arange(256)[:, None].expand(256, 1)
    codes = torch.nn.functional.pad(codes, (0, 96))
    byte = torch.nn.functional.pad(byte, (0, 3))
    h = Held(256, 32, codes, byte)
    buf, y = pitched(torch.zeros(256, 32, dtype=dtype), 35)
    tcu.tcu_mx4_dequant(*h.args(), y, 35, 256, 32)
    want = value64(codes, byte)[:, :32].to(F32).to(dtype)     # to binary32: exact, or infinite
    got = y.cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(got.double()), torch.nan_to_num(want.double()))
    assert untouched(buf, 256, 32, 35)


@pytest.mark.parametrize("rows,cols", [(1, 1), (33, 517), (300, 1003)])
def test_dequant_sizes(rows, cols):
    x = randn((rows, cols), BF16, gen(1))
    h = Held(rows, cols, *quant64(x))
    for dtype in (BF16, F32, F16):
        buf, y = pitched(torch.zeros(rows, cols, dtype=dtype), cols + 5)
        tcu.tcu_mx4_dequant(*h.args(), y, cols + 5, rows, cols)
        assert torch.equal(y.cpu().double(), rounded64(x))
        assert untouched(buf, rows, cols, cols + 5)


def test_nothing_to_do():
    """No rows or no columns: nothing is read or written."""
    for rows, cols in ((0, 40), (40, 0), (0, 0)):
        x = torch.zeros(rows, cols, dtype=BF16, device=DEV)
        q = torch.zeros(rows, 64 * groups(cols), dtype=torch.uint8, device=DEV)
        s = torch.zeros(groups(cols), rows, dtype=torch.int32, device=DEV)
        tcu.tcu_mx4_quant(x, cols, q, 64 * groups(cols), s, rows, None, 0, None, 0, rows, cols)
        tcu.tcu_mx4_dequant(q, 64 * groups(cols), s, rows, x, cols, rows, cols)

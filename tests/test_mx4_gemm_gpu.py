"""tcu_mx4_gemm and tcu_mx4_linear against binary64.

Products of codes and scales are exact; a sum of K binary32 terms is off by at most
(K + 8) 2^-24 of the terms' magnitudes in any order, the stored C (accumulating) being
one more term, and the result is rounded once."""
import pytest
import torch

from layer_util import DEV, F32 as EPS, ROUND, gen, pitched, randn, untouched, within
from mx4_util import Held, quant64, value64
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def matrix(rows, cols, g, dtype=BF16, scale=1.0):
    x = randn((rows, cols), dtype, g, scale)
    return x, quant64(x)


def work(M, K, N):
    return torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=torch.uint8, device=DEV)


def check(M, K, N, dtype, acc=False, pad=0, seed=0):
    g = gen(seed + M + K + N)
    _, a = matrix(M, K, g)
    _, b = matrix(N, K, g, scale=max(K, 1) ** -0.5)
    A, B = Held(M, K, *a), Held(N, K, *b)
    C0 = randn((M, N), dtype, g)
    buf, C = pitched(C0, N + pad)
    tcu.tcu_mx4_gemm(*A.args(), *B.args(), C, N + pad, work(M, K, N), M, K, N,
                     tcu.TCU_ACCUMULATE if acc else 0)
    va, vb = value64(*a), value64(*b)
    want = va @ vb.t()
    mag = va.abs() @ vb.abs().t()
    if acc:
        want, mag = want + C0.double(), mag + C0.double().abs()
    within(C, want, (K + 8) * EPS * mag + want.abs() * ROUND[dtype])
    assert untouched(buf, M, N, N + pad)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("M,K,N", [
    # single rows and columns, K below, at and past a group
    (1, 1, 1), (1, 32, 16), (1, 128, 5), (3, 129, 33), (16, 1000, 100), (17, 2048, 48),
    (32, 512, 40), (33, 300, 70), (64, 4096, 257),
    # tiles, cut along K or not, odd numbers of groups
    (65, 128, 64), (100, 129, 100), (130, 384, 300), (200, 640, 129), (257, 1003, 260),
    (128, 8192, 128), (300, 5000, 77)])
@pytest.mark.parametrize("acc,pad", [(False, 0), (True, 3)])
def test_sizes(dtype, M, K, N, acc, pad):
    check(M, K, N, dtype, acc, pad)


@pytest.mark.parametrize("M,K,N", [(4096, 640, 4096), (4100, 384, 4353), (33000, 130, 600)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_large_tiles(M, K, N, dtype):
    check(M, K, N, dtype, pad=5)


@pytest.mark.parametrize("M", [3, 50, 300])
def test_nothing_to_add(M):
    """K = 0: zeros, or C as it is."""
    h = Held(M, 0), Held(20, 0)
    C = torch.full((M, 20), 2.5, device=DEV)
    tcu.tcu_mx4_gemm(*h[0].args(), *h[1].args(), C, 20, work(M, 0, 20), M, 0, 20,
                     tcu.TCU_ACCUMULATE)
    assert bool((C == 2.5).all())
    tcu.tcu_mx4_gemm(*h[0].args(), *h[1].args(), C, 20, work(M, 0, 20), M, 0, 20, 0)
    assert bool((C == 0).all())
    X = torch.empty(M, 0, dtype=BF16, device=DEV)
    C.fill_(1)
    tcu.tcu_mx4_linear(X, 0, *h[1].args(), C, 20, work(M, 0, 20), M, 0, 20, 0)
    assert bool((C == 0).all())


@pytest.mark.parametrize("M", [5, 40, 200])
def test_blocks_that_are_not_finite(M):
    """A NaN block makes its row's (or column's) results NaN and no other."""
    K, N = 700, 90
    g = gen(M)
    _, (ca, ba) = matrix(M, K, g)
    _, (cb, bb) = matrix(N, K, g)
    ba[2, 3] = 255
    bb[7, 21] = 255
    A, B = Held(M, K, ca, ba), Held(N, K, cb, bb)
    C = torch.empty(M, N, device=DEV)
    tcu.tcu_mx4_gemm(*A.args(), *B.args(), C, N, work(M, K, N), M, K, N)
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[2] = bad[:, 7] = True
    assert torch.equal(torch.isnan(C).cpu(), bad)


@pytest.mark.parametrize("M", [5, 40, 200])
def test_scales_of_all_sizes(M):
    """Scales from 2^-127 to 2^127 on one side and their inverses on the other: every term
    is of ordinary size."""
    K, N = 1024, 64
    g = gen(M + 1)
    _, (ca, _) = matrix(M, K, g)
    _, (cb, _) = matrix(N, K, g)
    e = torch.randint(0, 255, (K // 32,), generator=g)
    ba, bb = e.expand(M, -1).contiguous(), (254 - e).expand(N, -1).contiguous()
    A, B = Held(M, K, ca, ba), Held(N, K, cb, bb)
    C = torch.empty(M, N, device=DEV)
    tcu.tcu_mx4_gemm(*A.args(), *B.args(), C, N, work(M, K, N), M, K, N)
    va, vb = value64(ca, ba), value64(cb, bb)
    within(C, va @ vb.t(), (K + 8) * EPS * (va.abs() @ vb.abs().t()))


@pytest.mark.parametrize("xtype,ytype", [(BF16, BF16), (BF16, F32), (F16, F16), (F16, F32)])
@pytest.mark.parametrize("M,K,N", [(1, 1, 1), (1, 4096, 256), (2, 1003, 50), (4, 130, 33),
                                   (5, 512, 64), (16, 2000, 40), (64, 640, 100), (65, 1003, 70),
                                   (300, 256, 515)])
@pytest.mark.parametrize("acc,pad", [(False, 0), (True, 5)])
def test_linear(xtype, ytype, M, K, N, acc, pad):
    g = gen(M + K + N)
    X, a = matrix(M, K, g, xtype)
    _, b = matrix(N, K, g, scale=K ** -0.5)
    B = Held(N, K, *b)
    Y0 = randn((M, N), ytype, g)
    _, dX = pitched(X, K + pad)
    buf, Y = pitched(Y0, N + pad)
    tcu.tcu_mx4_linear(dX, K + pad, *B.args(), Y, N + pad, work(M, K, N), M, K, N,
                       tcu.TCU_ACCUMULATE if acc else 0)
    va, vb = value64(*a), value64(*b)
    want, mag = va @ vb.t(), va.abs() @ vb.abs().t()
    if acc:
        want, mag = want + Y0.double(), mag + Y0.double().abs()
    within(Y, want, (K + 8) * EPS * mag + want.abs() * ROUND[ytype])
    assert untouched(buf, M, N, N + pad)


@pytest.mark.parametrize("M", [1, 3, 30, 130])
def test_linear_rows_that_are_not_finite(M):
    """An infinity or NaN in X makes its row NaN and no other."""
    K, N = 300, 40
    g = gen(M)
    X, _ = matrix(M, K, g)
    X[0, 299] = float("inf")
    if M > 2:
        X[2, 5] = float("nan")
    _, b = matrix(N, K, g)
    B, Y = Held(N, K, *b), torch.empty(M, N, device=DEV)
    tcu.tcu_mx4_linear(X.to(DEV), K, *B.args(), Y, N, work(M, K, N), M, K, N)
    bad = torch.zeros(M, N, dtype=torch.bool)
    bad[0] = True
    bad[2:3] = True
    assert torch.equal(torch.isnan(Y).cpu(), bad)

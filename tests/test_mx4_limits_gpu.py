"""The products in 4 bits at the ends of their pitches: codes, scales, inputs and outputs whose
rows lie past 32 bits of bytes, and batches far past one launch's rounds."""
import pytest
import torch

from layer_util import DEV, F32 as EPS, gen, randn, within
from mx4_util import rounded64
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


def spread(rows, cols, ld, dtype):
    """A view of `rows` rows, ld elements apart, of a buffer of its own."""
    return torch.empty((rows - 1) * ld + cols, dtype=dtype, device=DEV).as_strided((rows, cols),
                                                                                   (ld, 1))


@pytest.mark.parametrize("M", [3, 70])
def test_codes_and_scales_far_apart(M):
    """Rows of codes 2^26 bytes apart (70 of them: 4.7 GB), words of the second group 2^30
    words behind the first's."""
    g = gen(M)
    N, K, lds = 70, 200, 2 ** 30 + 8
    X, W = randn((M, K), BF16, g), randn((N, K), BF16, g)
    q, s = spread(N, 128, 2 ** 26, U8), spread(2, N, lds, I32)
    tcu.tcu_mx4_quant(W.to(DEV), K, q, 2 ** 26, s, lds, None, 0, None, 0, N, K)
    back = torch.empty(N, K, device=DEV)
    tcu.tcu_mx4_dequant(q, 2 ** 26, s, lds, back, K, N, K)
    W4, X4 = rounded64(W), rounded64(X)
    assert torch.equal(back.cpu().double(), W4)
    want, mag = X4 @ W4.t(), X4.abs() @ W4.abs().t()
    work = torch.empty(max(tcu.tcu_mx4_work(M, K, N), tcu.tcu_mx4_work(N, K, M)), dtype=U8,
                       device=DEV)
    Y = torch.empty(M, N, device=DEV)
    tcu.tcu_mx4_linear(X.to(DEV), K, q, 2 ** 26, s, lds, Y, N, work, M, K, N)
    within(Y, want, (K + 8) * EPS * mag)
    # as the left operand too: the product's transpose
    a, b = torch.empty(M, 128, dtype=U8, device=DEV), torch.empty(2, M, dtype=I32, device=DEV)
    tcu.tcu_mx4_quant(X.to(DEV), K, a, 128, b, M, None, 0, None, 0, M, K)
    Z = torch.empty(N, M, device=DEV)
    tcu.tcu_mx4_gemm(q, 2 ** 26, s, lds, a, 128, b, M, Z, M, work, N, K, M)
    within(Z, want.t(), (K + 8) * EPS * mag.t())


@pytest.mark.parametrize("M", [3, 66])
def test_inputs_and_outputs_far_apart(M):
    """Rows of X and of Y 2^30 or 2^26 elements apart, past 4 GiB in all."""
    g = gen(M)
    K, N = 130, 40
    ld = 2 ** 30 + 16 if M == 3 else 2 ** 26 + 8
    X, W = randn((M, K), BF16, g), randn((N, K), BF16, g)
    x, y = spread(M, K, ld, BF16), spread(M, N, ld, F32)
    x.copy_(X)
    q, s = torch.empty(N, 128, dtype=U8, device=DEV), torch.empty(2, N, dtype=I32, device=DEV)
    tcu.tcu_mx4_quant(W.to(DEV), K, q, 128, s, N, None, 0, None, 0, N, K)
    work = torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=U8, device=DEV)
    tcu.tcu_mx4_linear(x, ld, q, 128, s, N, y, ld, work, M, K, N)
    W4, X4 = rounded64(W), rounded64(X)
    want, mag = X4 @ W4.t(), X4.abs() @ W4.abs().t()
    within(y, want, (K + 8) * EPS * mag)
    # both ways from rows far apart
    G = tcu.tcu_mx4_row_bytes(M)
    qx, sx = torch.empty(M, 128, dtype=U8, device=DEV), torch.empty(2, M, dtype=I32, device=DEV)
    qt, st = torch.empty(K, G, dtype=U8, device=DEV), torch.empty(1, K, dtype=I32, device=DEV)
    tcu.tcu_mx4_quant(x, ld, qx, 128, sx, M, qt, G, st, K, M, K)
    back, turned = torch.empty(M, K, device=DEV), torch.empty(K, M, device=DEV)
    tcu.tcu_mx4_dequant(qx, 128, sx, M, back, K, M, K)
    tcu.tcu_mx4_dequant(qt, G, st, K, turned, M, K, M)
    assert torch.equal(back.cpu().double(), X4)
    assert torch.equal(turned.cpu().double(), rounded64(X.t()))


@pytest.mark.parametrize("M,N", [(2 ** 21 + 5, 3), (5, 2 ** 21 + 5), (300000, 130)])
def test_many_rows(M, N):
    """Of either operand, K of one group; every row's results by those of 16 distinct ones."""
    K = 96
    g = gen(N)
    big = max(M, N)
    base = randn((16, K), BF16, g)
    small = randn((min(M, N), K), BF16, g)
    X = base.to(DEV)[torch.arange(big, device=DEV) % 16]
    q, s = torch.empty(big, 64, dtype=U8, device=DEV), torch.empty(1, big, dtype=I32, device=DEV)
    tcu.tcu_mx4_quant(X, K, q, 64, s, big, None, 0, None, 0, big, K)
    n = min(M, N)
    p, t = torch.empty(n, 64, dtype=U8, device=DEV), torch.empty(1, n, dtype=I32, device=DEV)
    tcu.tcu_mx4_quant(small.to(DEV), K, p, 64, t, n, None, 0, None, 0, n, K)
    C = torch.empty(M, N, device=DEV)
    work = torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=U8, device=DEV)
    left, right = ((q, 64, s, big), (p, 64, t, n)) if M > N else ((p, 64, t, n), (q, 64, s, big))
    tcu.tcu_mx4_gemm(*left, *right, C, N, work, M, K, N)
    R = C if M > N else C.t()
    a, b = rounded64(base), rounded64(small)
    want, mag = a @ b.t(), a.abs() @ b.abs().t()
    within(R[:16], want, (K + 8) * EPS * mag)
    # (rows of one value everywhere, whatever tile they are in)
    at = torch.arange(big, device=DEV) % 16
    off = (R - R[:16][at]).abs()
    assert bool((off <= 2 * (K + 8) * EPS * mag.float().to(DEV)[at]).all())


def test_one_workspace_in_turn():
    """Products that follow each other share the largest one's workspace."""
    g = gen(1)
    work = torch.empty(tcu.tcu_mx4_work(64, 8192, 64), dtype=U8, device=DEV)
    for M, K, N in ((64, 8192, 64), (1, 8192, 64), (64, 32, 1), (33, 8000, 50), (64, 8192, 64)):
        X, W = randn((M, K), BF16, g), randn((N, K), BF16, g)
        G = tcu.tcu_mx4_row_bytes(K)
        q = torch.empty(N, G, dtype=U8, device=DEV)
        s = torch.empty(G // 64, N, dtype=I32, device=DEV)
        tcu.tcu_mx4_quant(W.to(DEV), K, q, G, s, N, None, 0, None, 0, N, K)
        Y = torch.empty(M, N, device=DEV)
        assert tcu.tcu_mx4_work(M, K, N) <= work.numel()
        tcu.tcu_mx4_linear(X.to(DEV), K, q, G, s, N, Y, N, work, M, K, N)
        X4, W4 = rounded64(X), rounded64(W)
        within(Y, X4 @ W4.t(), (K + 8) * EPS * (X4.abs() @ W4.abs().t()))

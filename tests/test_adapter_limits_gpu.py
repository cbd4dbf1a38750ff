"""The adapter operators at the ends of their sizes and values."""
import pytest
import torch

from layer_util import DEV, Layer, within
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu


def forward(d, out):
    X, W, A, B, alpha, ids = (t.to(DEV) for t in (d.X, d.W, d.A, d.B, d.alpha, d.ids))
    Y = torch.empty(d.M, d.N, dtype=out, device=DEV)
    work = torch.empty(tcu.tcu_adapter_work(d.M, d.K, d.N, d.r, d.G), dtype=torch.uint8, device=DEV)
    tcu.tcu_adapter_gemm(X, d.K, W, d.N, A, B, alpha, ids, Y, d.N, work, d.M, d.K, d.N, d.r, d.G)
    return Y


@pytest.mark.parametrize("r", [16, 32])
@pytest.mark.parametrize("M", [4, 100, 500])
def test_infinite_rank_beside_large_ones(M, r):
    """binary16: one rank of T infinite, the others beyond binary16's range but finite."""
    d = Layer(M, 512, 64, r, 2, torch.float16, M)
    d.X = (d.X.float() * 100).to(torch.float16)
    d.A = (d.A.float() * 1000).to(torch.float16)
    d.A[0, 0, 7] = float("inf")
    d.X[:, 7] = d.X[:, 7].abs() + 1
    d.B[0, :, 0] = d.B[0, :, 0].abs() + 1
    assert float((d.X.double() @ d.A[0, 1:].double().t()).abs().max()) > 65504
    y, e = d.forward64()
    assert bool((y[d.ids == 0] == float("inf")).all()) and bool(torch.isfinite(y[d.ids != 0]).all())
    within(forward(d, torch.float32), y, e)


@pytest.mark.parametrize("M", [1, 57, 128, 256, 400])
def test_scratch_of_a_larger_batch(M):
    """Every call on the scratch of 512 rows, whatever it holds."""
    K, N, r, G = 4096, 2048, 16, 4
    d = Layer(M, K, N, r, G, torch.bfloat16, M)
    n = tcu.tcu_adapter_work(512, K, N, r, G)
    work = torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV)
    X, W, A, B, alpha, ids, dY = (t.to(DEV) for t in (d.X, d.W, d.A, d.B, d.alpha, d.ids, d.dY))
    Y = torch.empty(M, N, device=DEV)
    tcu.tcu_adapter_gemm(X, K, W, N, A, B, alpha, ids, Y, N, work[:n], M, K, N, r, G)
    within(Y, *d.forward64())
    dA, dB = torch.empty(A.shape, device=DEV), torch.empty(B.shape, device=DEV)
    tcu.tcu_adapter_grad(X, K, dY, N, A, B, alpha, ids, dA, dB, work[:n], M, K, N, r, G)
    A64, B64, eA, eB = d.grads64()
    within(dA, A64, eA)
    within(dB, B64, eB)
    dX = torch.empty(M, K, device=DEV)
    tcu.tcu_adapter_input_grad(dY, N, d.W.t().contiguous().to(DEV), K, A, B, alpha, ids, dX, K,
                               work[:n], M, K, N, r, G)
    within(dX, *d.input_grad64())
    assert bool((work[n:] == 255).all())

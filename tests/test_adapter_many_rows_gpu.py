"""Adapters of many rows against binary64: pieces of 32 rows of an adapter, found from
the rows' numbers and from their order, and factor gradients over several chunks."""
import pytest
import torch

from layer_util import DEV, ROUND, Layer, pitched, untouched, within
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
F16, BF16, FL = torch.float16, torch.bfloat16, torch.float32


def work_of(d):
    return torch.empty(tcu.tcu_adapter_work(d.M, d.K, d.N, d.r, d.G), dtype=torch.uint8, device=DEV)


def numbers(M, G, order):
    """Adapters' numbers: row by row in turn, in runs, or almost all of one adapter."""
    i = torch.arange(M)
    return {"mixed": i * 7 % (G + 1) - 1, "runs": i * (G + 1) // M - 1,
            "one": torch.where(i % 97 == 5, i // 97 % (G + 1) - 1, torch.full_like(i, G - 1))}[order]


# (M, K, N, r, G): looked through (up to 8192 rows), by their order past it or past 512
# adapters; K of one step, of a few and ragged; one and two blocks of ranks
@pytest.mark.parametrize("order", ["mixed", "runs", "one"])
@pytest.mark.parametrize("size", [(8100, 64, 40, 16, 33), (8192, 201, 24, 5, 70),
                                  (7000, 650, 16, 30, 9), (5000, 100, 33, 64, 100),
                                  (9000, 130, 24, 16, 6), (8500, 333, 40, 64, 17),
                                  (2000, 96, 16, 128, 520)])
@pytest.mark.parametrize("types", [(F16, FL), (BF16, BF16)])
def test_many_rows(types, size, order):
    M, K, N, r, G = size
    d = Layer(*size, types[0], M + K, numbers(M, G, order))
    y, e = d.forward64()
    X, W = pitched(d.X, K + 3)[1], pitched(d.W, N)[1]
    yb, Y = pitched(torch.zeros(M, N, dtype=types[1]), N + 5)
    tcu.tcu_adapter_gemm(X, K + 3, W, N, d.A.to(DEV), d.B.to(DEV), d.alpha.to(DEV), d.ids.to(DEV), Y,
                         N + 5, work_of(d), M, K, N, r, G)
    within(Y, y, e + y.abs() * ROUND[types[1]])
    assert untouched(yb, M, N, N + 5)


@pytest.mark.parametrize("order", ["mixed", "runs", "one"])
@pytest.mark.parametrize("size", [(9000, 130, 72, 16, 6), (3000, 200, 333, 64, 5),
                                  (1500, 96, 129, 128, 40), (2500, 301, 64, 33, 3),
                                  (900, 7, 5, 3, 2)])
@pytest.mark.parametrize("dtype", [F16, BF16])
def test_factor_gradients(dtype, size, order):
    M, K, N, r, G = size
    d = Layer(*size, dtype, M + K, numbers(M, G, order))
    want_a, want_b, ea, eb = d.grads64()
    dA = torch.full((G, r, K), float("nan"), device=DEV)
    dB = torch.full((G, N, r), float("nan"), device=DEV)
    args = (d.X.to(DEV), K, d.dY.to(DEV), N, d.A.to(DEV), d.B.to(DEV), d.alpha.to(DEV),
            d.ids.to(DEV), dA, dB, work_of(d), M, K, N, r, G)
    tcu.tcu_adapter_grad(*args)
    within(dA, want_a, ea)
    within(dB, want_b, eb)
    first = dA.clone(), dB.clone()
    tcu.tcu_adapter_grad(*args)
    assert torch.equal(first[0], dA) and torch.equal(first[1], dB), "another call gives other sums"

"""tcu_mx4_linear on up to four long rows: one launch up to 16384 inputs, X brought to 4 bits
by a launch of its own above, both against binary64."""
import shutil

import pytest
import torch

import recording as rec
from layer_util import DEV, F32 as EPS, ROUND, gen, randn, within
from mx4_util import Held, quant64, value64
from paper_1908_06649_amd import tcu
from test_mx4_dispatch import kernels, linear

BF16 = torch.bfloat16
ONE, TWO = [("mx4_few", [2, 2, 1, 1])], [("quant_rows", [2]), ("mx4_few", [2, -1, 1, 1])]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("M,K,N,want", [(1, 16384, 1024, ONE), (4, 16384, 4096, ONE),
                                        (1, 16385, 1024, TWO), (4, 32768, 4096, TWO)])
def test_launches(tmp_path, M, K, N, want):
    assert kernels(rec.run(rec.build(tmp_path), [linear(M, K, N)])[0]) == want


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", [(1, 16384, 33), (4, 16384, 20), (1, 16385, 33), (3, 20000, 50),
                                   (4, 32768, 40)])
def test_results(M, K, N):
    g = gen(M + K)
    X, W = randn((M, K), BF16, g), randn((N, K), BF16, g, K ** -0.5)
    a, b = quant64(X), quant64(W)
    B, Y = Held(N, K, *b), torch.empty(M, N, dtype=BF16, device=DEV)
    work = torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=torch.uint8, device=DEV)
    tcu.tcu_mx4_linear(X.to(DEV), K, *B.args(), Y, N, work, M, K, N)
    va, vb = value64(*a), value64(*b)
    want, mag = va @ vb.t(), va.abs() @ vb.abs().t()
    within(Y, want, (K + 8) * EPS * mag * (1 + ROUND[BF16]) + want.abs() * ROUND[BF16])

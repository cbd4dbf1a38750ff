"""The launches that the products in 4 bits and the heads' norms are made of
(tests/recording.py), on a device of 256 compute units."""
import re
import shutil

import pytest

from paper_1908_06649_amd import tcu

import recording as rec

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
P = rec.ptr
BIG = tcu.TCU_MAX_MX4_DIM
FAR = 1 << 50      # past the other addresses


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return rec.build(tmp_path_factory.mktemp("recording"))


def row(n):
    return 64 * ((n + 127) // 128)


def gemm(M, K, N, elem=2, flags=0, **kw):
    return dict(fn="tcu_mx4_gemm", args=[P(0), row(K) or 16, P(1), M, P(2), row(K) or 16, P(3), N,
                                         P(4), N, P(5), M, K, N, flags, elem, None], **kw)


def linear(M, K, N, **kw):
    return dict(fn="tcu_mx4_linear", args=[P(0), K, P(2), row(K), P(3), N, P(4), N, P(5), M, K, N,
                                           0, 2, 2, None], **kw)


def quant(rows, cols, q=True, qt=True, **kw):
    z = [P(1), row(cols), P(2), rows] if q else [None, 0, None, 0]
    zt = [P(3), row(rows), P(4), cols] if qt else [None, 0, None, 0]
    return dict(fn="tcu_mx4_quant", args=[P(0), cols, *z, *zt, rows, cols, 2, None], **kw)


def heads(T, hq, hk, dim, rot, **kw):
    return dict(fn="tcu_qk_norm", args=[P(0), hq * dim, dim, P(1), hk * dim, dim, P(2), P(2), P(3),
                                        P(4), P(5), hq * dim, dim, P(6), hk * dim, dim, T, hq, hk,
                                        dim, rot, 1e-5, 0, 2, None], **kw)


def heads_grad(T, hq, hk, dim, rot, **kw):
    x, y = [hq * dim, dim], [hk * dim, dim]
    return dict(fn="tcu_qk_norm_grad", args=[P(0), *x, P(1), *y, P(2), *x, P(3), *y, P(4), P(4),
                                             P(4), P(4), P(5), *x, P(6), *y, P(7), FAR,
                                             FAR + (1 << 41), T, hq, hk, dim, rot, 1e-5, 0, 2, None], **kw)


def kernels(answer):
    assert answer["rc"] == tcu.TCU_OK, answer["rc"]
    assert all(la["blocks"] * la["threads"] < 1 << 32 for la in answer["launches"])
    out = []
    for la in answer["launches"]:
        name = la["name"].split("_GLOBAL__N_1")[1].lstrip("0123456789")
        base, args = name.split("_kernel", 1)
        out.append((base, [int(a.replace("n", "-")) for a in re.findall(r"L[ib](n?\d+)E", args)]))
    return out


@pytest.mark.parametrize("job,want", [
    # single tokens: one launch, X brought to 4 bits in it
    (linear(1, 4096, 4096), [("mx4_few", [2, 2, 1, 1])]),
    (linear(4, 8192, 8192), [("mx4_few", [2, 2, 1, 2])]),
    # more: X first
    (linear(16, 8192, 8192), [("quant_rows", [2]), ("mx4_few", [2, -1, 1, 2])]),
    (linear(30, 4096, 1024), [("quant_rows", [2]), ("mx4_few", [2, -1, 2, 1])]),
    (linear(1000, 1003, 2005), [("quant_rows", [2]), ("mx4_tile", [2, 4, 2, 1, 2, 1])]),
    (linear(8192, 8192, 8192), [("quant_rows", [2]), ("mx4_tile", [2, 8, 4, 2, 4, 1])]),
    # a matrix in 4 bits: by rows, tiles and the length of the contracted index
    (gemm(1, 4096, 4096), [("mx4_few", [2, -1, 1, 1])]),
    (gemm(64, 1024, 1024), [("mx4_few", [2, -1, 4, 1])]),
    (gemm(64, 8192, 8192), [("mx4_tile", [2, 4, 2, 1, 2, 4])]),
    (gemm(1024, 8192, 1024), [("mx4_tile", [2, 4, 2, 1, 2, 4])]),
    (gemm(2048, 8192, 2048), [("mx4_tile", [2, 4, 4, 2, 2, 2])]),
    (gemm(2048, 512, 2048), [("mx4_tile", [2, 4, 2, 1, 2, 1])]),
    (gemm(4096, 4096, 4096), [("mx4_tile", [2, 8, 4, 2, 4, 1])]),
    (gemm(100, 65536, 64), [("mx4_tile", [3, 4, 2, 1, 2, 4]), ("mx4_join", [2])]),
    # nothing to multiply
    (gemm(100, 0, 64), [("mx4_join", [2])]),
    (quant(300, 500), [("quant_both", [2, 1])]),
    (quant(300, 500, q=False), [("quant_both", [2, 0])]),
    (quant(300, 500, qt=False), [("quant_rows", [2])]),
    # heads: whole vectors, whole vectors that share values, pairs
    (heads(1, 32, 8, 128, 128), [("heads", [2, 8, 1, 0, 0])]),
    (heads(100, 4, 4, 80, 40), [("heads", [2, 8, 1, 0, 1])]),
    (heads(100, 4, 4, 96, 48), [("heads", [2, 8, 1, 0, 0])]),
    (heads(100, 4, 4, 20, 10), [("heads", [2, 1, 1, 0, 0])]),
    (heads(100, 4, 4, 300, 4), [("heads", [2, 1, 8, 0, 0])]),
    (heads_grad(5000, 4, 4, 64, 64), [("heads", [2, 8, 1, 1, 0]), ("head_dw", [])]),
    (heads_grad(0, 4, 4, 64, 64), [("zero_dw", [])])])
def test_launches(so, job, want):
    assert kernels(rec.run(so, [job])[0]) == want


@pytest.mark.parametrize("job", [
    # sizes at their limits: as many launches as it takes, threads counted in 32 bits
    gemm(BIG, 64, 64), gemm(BIG, 256, 2048), gemm(64, 64, BIG), gemm(4, 64, BIG),
    gemm(1 << 20, 300, 1 << 18), quant(BIG, 100), quant(100, BIG), quant(BIG, 100, qt=False),
    quant(1 << 19, 1 << 19), heads(1 << 27, 2, 1, 64, 64), heads_grad(1 << 27, 2, 1, 64, 64)])
def test_large_sizes(so, job):
    assert kernels(rec.run(so, [job])[0])


@pytest.mark.parametrize("job,count", [(linear(16, 512, 512), 2), (gemm(100, 65536, 64), 2),
                                       (quant(64, 64), 1), (heads(5, 2, 2, 64, 64), 1),
                                       (heads_grad(5, 2, 2, 64, 64), 2), (gemm(64, 64, BIG), 4)])
def test_a_failed_launch_is_reported(so, job, count):
    for fail in range(count):
        answer = rec.run(so, [{**job, "fail": fail}])[0]
        assert answer["rc"] == tcu.TCU_ERR_HIP and len(answer["launches"]) == fail + 1

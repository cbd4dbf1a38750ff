"""Every variant of the 4-bit product's tile kernel: which sizes it takes (the launches, on a
device of 256 compute units), and its results on the GPU, exactly.

Codes are multiples of 1/2 up to 6 and scales here 1 or 2: a term is a multiple of 1/4 of at
most 144, and K <= 8192 of them and a C of at most 8 stay below 2^21, so that every sum in
any order is a binary32 number, and the result is the exact one, rounded once."""
import shutil

import pytest
import torch

import recording as rec
from layer_util import DEV, pitched, untouched
from mx4_util import MAG, groups
from paper_1908_06649_amd import tcu
from test_mx4_dispatch import gemm, kernels

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
ELEMS = {F32: 0, F16: 1, BF16: 2}

# (FM, FN, WM, WN, KG) of the kernel: tiles of 256, 128 and 64 with 1, 2 or 4 groups of waves;
# sizes with more tiles than workgroups, ragged edges, odd numbers of groups of 128
V256, V128, V128x2 = (8, 4, 2, 4, 1), (4, 4, 2, 2, 1), (4, 4, 2, 2, 2)
V64, V64x2, V64x4 = (4, 2, 1, 2, 1), (4, 2, 1, 2, 2), (4, 2, 1, 2, 4)
CASES = [
    (V256, 4096, 640, 4096),      # a tile a workgroup
    (V256, 1500, 1003, 6000),     # ragged, a tile a workgroup
    (V256, 6007, 600, 6100),      # 576 tiles, 3 rounds of stages
    (V256, 4500, 2049, 4203),     # 306 tiles, 9 rounds, the last one half
    (V256, 8192, 4096, 4352),     # 544 whole tiles
    (V256, 16400, 300, 16500),    # 4225 tiles of two rounds
    (V128, 4100, 384, 4353),
    (V128, 8000, 300, 4500),      # 2268 tiles
    (V128, 4096, 256, 4224),      # 1056 whole tiles of one round
    (V128x2, 2048, 8192, 2048),   # whole tiles
    (V128x2, 1990, 4100, 2011),   # 17 rounds for two groups, the last one half
    (V128x2, 640, 3000, 5001),
    (V64, 1000, 1003, 2005),
    (V64, 2048, 512, 2048),
    (V64, 6001, 130, 1300),       # 1974 tiles
    (V64x2, 3000, 1003, 520),
    (V64x2, 500, 2100, 2005),
    (V64x4, 1100, 8192, 520),
    (V64x4, 500, 2100, 520),      # 9 rounds for four groups
]
# long contracted indices, their ranges summed by a second launch
RANGES = [(100, 65536, 64), (512, 65536, 512), (77, 40100, 131), (65, 20000, 2)]


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return rec.build(tmp_path_factory.mktemp("recording"))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("variant,M,K,N", CASES)
def test_variant_of_a_size(so, variant, M, K, N):
    for elem in ELEMS.values():
        assert kernels(rec.run(so, [gemm(M, K, N, elem)])[0]) == [("mx4_tile", [elem, *variant])]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("M,K,N", RANGES)
def test_ranges_of_a_size(so, M, K, N):
    assert kernels(rec.run(so, [gemm(M, K, N)])[0]) == [("mx4_tile", [3, *V64x4]), ("mx4_join", [2])]


def held(rows, K, seed, scales=2):
    """((codes, pitch, scales, pitch), the values in binary64) on the device; scales of 1, or 1
    and 2."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    G = groups(K)
    codes = torch.zeros(rows, 128 * G, dtype=torch.uint8, device=DEV)
    codes[:, :K] = torch.randint(0, 16, (rows, K), generator=g, device=DEV, dtype=torch.uint8)
    byte = torch.randint(127, 127 + scales, (rows, 4 * G), generator=g, device=DEV, dtype=torch.uint8)
    q = codes.view(rows, -1, 2)
    q = (q[..., 0] | (q[..., 1] << 4)).contiguous()
    s = byte.view(torch.int32).t().contiguous()
    table = torch.cat((MAG, -MAG)).to(DEV)
    v = table[codes.int()].view(rows, -1, 32) * (byte.double() - 126)[..., None]
    return (q, 64 * G, s, rows), v.view(rows, -1)[:, :K]


def quarters(shape, dtype, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randint(-32, 33, shape, generator=g, device=DEV).to(dtype) / 4


def work(M, K, N):
    return torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=torch.uint8, device=DEV)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N", RANGES)
def test_results_of_ranges(M, K, N):
    """All scales 1: terms of at most 36, their sums below 2^22."""
    check(M, K, N, 1)


@pytest.mark.gpu
@pytest.mark.parametrize("variant,M,K,N", CASES)
def test_results(variant, M, K, N):
    check(M, K, N, 2)


def check(M, K, N, scales):
    A, a = held(M, K, 1, scales)
    B, b = held(N, K, 2, scales)
    ab = a @ b.t()
    for dtype in (F32, BF16, F16):
        for flags, pad in ((0, 0), (0, 3), (tcu.TCU_ACCUMULATE, 0), (tcu.TCU_ACCUMULATE, 3)):
            C0 = quarters((M, N), dtype, 3)
            buf, C = pitched(C0, N + pad)
            tcu.tcu_mx4_gemm(*A, *B, C, N + pad, work(M, K, N), M, K, N, flags)
            want = (ab + C0.double() if flags else ab).to(F32).to(dtype)
            assert torch.equal(C, want), (dtype, flags, pad, int((C != want).sum()))
            assert untouched(buf, M, N, N + pad), (dtype, flags, pad)


@pytest.mark.gpu
@pytest.mark.parametrize("variant,M,K,N", [CASES[i] for i in (2, 3, 6, 10, 12, 16, 18)])
def test_blocks_that_are_not_finite(variant, M, K, N):
    """In the last block of the last row of A and the first of a row of B: their results and
    no others."""
    A, a = held(M, K, 4)
    B, b = held(N, K, 5)
    last = (K - 1) // 32
    A[2][last // 4, M - 1] |= 0xff << 8 * (last % 4) if last % 4 < 3 else -1 << 24
    B[2][0, N // 2] |= 0xff
    C = torch.empty(M, N, device=DEV)
    tcu.tcu_mx4_gemm(*A, *B, C, N, work(M, K, N), M, K, N)
    bad = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    bad[M - 1] = bad[:, N // 2] = True
    assert torch.equal(torch.isnan(C), bad)
    assert torch.equal(C[~bad].double(), (a @ b.t())[~bad])

"""The adapters' part on every kernel that forms a product's tiles: the library's
choice overridden, with rows of several adapters in one tile, ragged edges, rows
at odd addresses, ranges of the contracted index, and few workgroups for many
tiles."""
import pytest
import torch

from gpu_util import PATHS
from layer_util import DEV, F32, ROUND, Layer, gen, pitched, untouched, within
from paper_1908_06649_amd import tcu
from test_adapter_gpu import BF16, F16, FL, dev, work_of

pytestmark = pytest.mark.gpu


def orders(M, G):
    """Rows as prompts lie, and mixed."""
    return {"runs": torch.arange(M) * (G + 1) // max(M, 1) - 1,
            "mixed": torch.randint(-1, G, (M,), generator=gen(M))}


def run(d, out, pad, q8=None):
    yb, Y = pitched(torch.zeros(d.M, d.N, dtype=out), d.N + pad)
    work, low = work_of(d), dev(d.A, d.B, d.alpha, d.ids)
    X = pitched(d.X, d.K + pad)[1]
    if q8:
        xq, wq, xs, ws = q8
        tcu.tcu_adapter_gemm_q8(pitched(xq, d.K + pad)[1], d.K + pad, xs.to(DEV),
                                pitched(wq, d.N + pad)[1], d.N + pad, ws.to(DEV), X, d.K + pad,
                                *low, Y, d.N + pad, work, d.M, d.K, d.N, d.r, d.G)
    else:
        tcu.tcu_adapter_gemm(X, d.K + pad, pitched(d.W, d.N + pad)[1], d.N + pad, *low, Y,
                             d.N + pad, work, d.M, d.K, d.N, d.r, d.G)
    assert untouched(yb, d.M, d.N, d.N + pad) and bool((work[-64:] == 255).all())
    return Y


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("types", [(F16, FL), (BF16, FL), (BF16, BF16)])
@pytest.mark.parametrize("M,K,N,r,pad", [(512, 256, 512, 16, 0), (300, 1003, 517, 8, 0),
                                         (700, 320, 776, 32, 8), (530, 257, 600, 48, 3),
                                         (257, 96, 272, 128, 0)])
def test_tiles(knobs, path, types, M, K, N, r, pad):
    knobs(tcu.TCU_KNOB_GEMM_KERNEL, PATHS[path])
    knobs(tcu.TCU_KNOB_PP_GRID, 3)
    for name, ids in orders(M, 5).items():
        d = Layer(M, K, N, r, 5, types[0], M + K, ids)
        y, e = d.forward64()
        within(run(d, types[1], pad), y, e + y.abs() * ROUND[types[1]])


@pytest.mark.parametrize("path", sorted(PATHS))
@pytest.mark.parametrize("M,K,N,r,pad", [(512, 256, 512, 16, 0), (300, 1003, 517, 8, 0),
                                         (700, 320, 784, 32, 16), (257, 96, 272, 128, 5)])
def test_tiles_q8(knobs, path, M, K, N, r, pad):
    knobs(tcu.TCU_KNOB_GEMM_KERNEL, PATHS[path])
    knobs(tcu.TCU_KNOB_PP_GRID, 3)
    g = gen(M)
    q8 = (torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8),
          torch.randint(-128, 128, (K, N), generator=g, dtype=torch.int8),
          torch.rand(M, generator=g) / 127, torch.rand(N, generator=g) / 127)
    base = (q8[0].double() @ q8[1].double()) * q8[2].double()[:, None] * q8[3].double()
    for name, ids in orders(M, 5).items():
        d = Layer(M, K, N, r, 5, BF16, M + K, ids)
        low, mag = d.adapters64()
        y = base + low
        within(run(d, BF16, pad, q8), y, base.abs() * 4 * F32 + y.abs() * 2.0 ** -8 +
               mag * ((K + r + 8) * F32 + 2.0 ** -16))


@pytest.mark.parametrize("path,knob", [("fast", tcu.TCU_KNOB_SPLIT_K), ("ring", tcu.TCU_KNOB_SPLIT_K),
                                       ("general", tcu.TCU_KNOB_SPLIT_K),
                                       ("fast", tcu.TCU_KNOB_TAIL_SPLIT)])
def test_ranges_add_the_adapters_once(knobs, path, knob):
    knobs(tcu.TCU_KNOB_GEMM_KERNEL, PATHS[path])
    knobs(knob, 3)
    knobs(tcu.TCU_KNOB_PP_GRID, 4)
    for types in ((F16, FL), (BF16, FL)):
        d = Layer(768, 2048, 512, 16, 4, types[0], 5, orders(768, 4)["mixed"])
        y, e = d.forward64()
        within(run(d, FL, 0), y, e)


@pytest.mark.parametrize("path", ["fast", "ring"])
def test_tiles_keep_rows_apart(knobs, path):
    knobs(tcu.TCU_KNOB_GEMM_KERNEL, PATHS[path])
    for types in ((F16, FL), (BF16, BF16)):
        d = Layer(600, 128, 264, 16, 4, types[0], 6, orders(600, 4)["mixed"])
        clean = run(d, types[1], 0).cpu()
        d.A[1, 3, 5] = float("nan")
        d.B[2, 7, 2] = float("inf")
        got = run(d, types[1], 0).cpu()
        fine = (d.ids != 1) & (d.ids != 2)
        assert torch.equal(got[fine], clean[fine])
        assert bool(torch.isnan(got[d.ids == 1]).all())
        two = got[d.ids == 2]
        assert not bool(torch.isfinite(two[:, 7]).any())
        two[:, 7] = 0
        assert bool(torch.isfinite(two).all())

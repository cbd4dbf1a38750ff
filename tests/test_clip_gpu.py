"""tcu_clip_grads against binary64."""
import math

import pytest
import torch

from layer_util import DEV, F32, ROUND, gen, randn
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def clip(grads, max_norm, outs=None):
    outs = [torch.empty_like(t) for t in grads] if outs is None else outs
    result = torch.full((2,), -1.0, device=DEV)
    work = torch.full((tcu.tcu_clip_grads_work() + 64,), 255, dtype=torch.uint8, device=DEV)
    tcu.tcu_clip_grads(grads, outs, max_norm, result, work)
    assert bool((work[-64:] == 255).all())
    return outs, float(result[0]), float(result[1])


def check(grads, max_norm):
    outs, norm, coef = clip(grads, max_norm)
    want = math.sqrt(sum(float(t.double().pow(2).sum()) for t in grads))
    c = min(1.0, max_norm / (want + 1e-6))
    # summed in binary64, rounded once
    assert abs(norm - want) <= 2 * F32 * want
    assert abs(coef - c) <= 2 * F32 * c + 2.0 ** -149     # binary32's smallest step
    for t, o in zip(grads, outs):
        ref = t.double() * c
        tiny = 2.0 ** -24 if t.dtype == torch.float16 else 2.0 ** -133
        assert float(((o.double() - ref).abs() - (ref.abs() * (ROUND[t.dtype] + 4 * F32) + tiny))
                     .max() if t.numel() else 0.0) <= 0
    return outs


@pytest.mark.parametrize("max_norm", [0.0, 0.5, 1e9])
@pytest.mark.parametrize("sizes", [[1], [7, 8, 9], [8192, 8191, 8193, 1], [100003], [0, 5, 0],
                                   [3 * i + 1 for i in range(300)]])
def test_clip(sizes, max_norm):
    g = gen(len(sizes))
    check([randn((n,), TYPES[i % 3], g).to(DEV) for i, n in enumerate(sizes)], max_norm)


def test_clip_large():
    g = torch.Generator(device=DEV).manual_seed(4)
    check([torch.randn(n, generator=g, device=DEV) for n in (30_000_001, 5, 12_345_678)], 3.0)


def test_clip_no_tensors():
    assert clip([], 1.0)[1:] == (0.0, 1.0)


def test_clip_any_address_and_in_place():
    g = gen(9)
    base = {t: randn((5000,), t, g).to(DEV) for t in TYPES}
    grads = [base[t][k:k + n] for t in TYPES for k, n in ((1, 17), (19, 1003), (1025, 3001))]
    ref = check(grads, 2.0)
    rest = {t: b.clone() for t, b in base.items()}
    outs, _, coef = clip(grads, 2.0, grads)
    assert coef < 1 and all(torch.equal(a, b) for a, b in zip(outs, ref))
    for t in TYPES:      # the elements between the views
        for at in (0, 18, 1022, 1023, 1024, 4026, 4999):
            assert float(base[t][at]) == float(rest[t][at])
    before = [t.clone() for t in grads]
    assert clip(grads, 1e9, grads)[2] == 1.0
    assert all(torch.equal(a, b) for a, b in zip(grads, before))


def test_clip_squares_past_binary32():
    grads = [torch.full((1000,), 2e30, device=DEV), torch.full((10,), 1e38, device=DEV,
                                                               dtype=torch.bfloat16)]
    check(grads, 1.0)
    check([torch.full((1000,), 1e-30, device=DEV)], 1.0)


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_clip_not_finite(bad):
    x = torch.randn(3000, device=DEV)
    x[1234] = bad
    (o,), norm, coef = clip([x], 1.0)
    if math.isinf(bad):
        assert math.isinf(norm) and coef == 0
        assert bool(torch.isnan(o[1234])) and float(o[:1234].abs().max()) == 0
    else:
        assert math.isnan(norm) and math.isnan(coef) and bool(torch.isnan(o).all())


def test_clip_repeats_and_graph():
    g = gen(2)
    grads = [randn((n,), TYPES[i % 3], g).to(DEV) for i, n in enumerate([50000, 3, 700, 90001])]
    outs = [torch.empty_like(t) for t in grads]
    result = torch.empty(2, device=DEV)
    work = torch.empty(tcu.tcu_clip_grads_work(), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        tcu.tcu_clip_grads(grads, outs, 1.0, result, work)
    for k in range(4):
        for t in grads:
            t.mul_(1.0 + k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t, r in zip(got, clip(grads, 1.0)[0]):
            assert torch.equal(t, r)

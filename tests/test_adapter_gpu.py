"""The adapter operators against binary64."""
import pytest
import torch

from layer_util import DEV, F32, ROUND, Layer, gen, pitched, randn, untouched, within
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
F16, BF16, FL = torch.float16, torch.bfloat16, torch.float32
PAIRS = [(F16, FL), (BF16, FL), (BF16, BF16)]
# from one token to several tiles; one of K, N, r, G odd or small in turn
SIZES = [(1, 64, 64, 16, 1), (1, 1000, 257, 8, 4), (3, 512, 1024, 16, 3), (8, 4096, 512, 16, 8),
         (16, 100, 96, 4, 2), (17, 33, 31, 1, 3), (40, 2048, 640, 32, 40), (64, 1024, 1000, 16, 5),
         (65, 257, 129, 20, 2), (100, 8, 8, 64, 3), (130, 640, 300, 128, 2), (256, 512, 512, 16, 1),
         (300, 1003, 517, 8, 7), (513, 320, 768, 32, 4), (1000, 256, 264, 16, 30),
         (2, 3, 5, 3, 2), (33, 1, 1, 2, 2), (700, 4096, 256, 16, 2), (128, 4096, 256, 16, 5),
         (256, 2048, 200, 8, 3), (64, 8192, 72, 128, 4), (200, 3001, 100, 64, 9)]


def work_of(d):
    n = tcu.tcu_adapter_work(d.M, d.K, d.N, d.r, d.G)
    return torch.full((n + 64,), 255, dtype=torch.uint8, device=DEV)


def dev(*ts):
    return [t.to(DEV) for t in ts]


def forward(d, out, pad=0, work=None):
    X, W = pitched(d.X, d.K + pad)[1], pitched(d.W, d.N + pad)[1]
    yb, Y = pitched(torch.zeros(d.M, d.N, dtype=out), d.N + pad)
    work = work_of(d) if work is None else work
    tcu.tcu_adapter_gemm(X, d.K + pad, W, d.N + pad, *dev(d.A, d.B, d.alpha, d.ids), Y, d.N + pad,
                         work, d.M, d.K, d.N, d.r, d.G)
    assert untouched(yb, d.M, d.N, d.N + pad)
    assert bool((work[-64:] == 255).all())
    return Y


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("size", SIZES)
def test_adapter(size, types):
    d = Layer(*size, types[0], sum(size))
    y, e = d.forward64()
    for pad in (0, 8, 3):
        within(forward(d, types[1], pad), y, e + y.abs() * ROUND[types[1]])


@pytest.mark.parametrize("M", [1, 5, 16, 50, 128, 129, 700])
def test_adapter_rows_without_one(M):
    """No row has an adapter, G = 0, and numbers far outside: the projection alone."""
    none = torch.full((M,), -1)
    far = torch.tensor([2 ** 31 - 1, -2 ** 31, 4, -7] * M)[:M]
    for G, ids in ((3, none), (3, far), (0, none)):
        d = Layer(M, 300, 200, 16, G, BF16, M, ids)
        y, e = d.forward64()
        within(forward(d, BF16), y, e + y.abs() * ROUND[BF16])
    d = Layer(M, 300, 200, 16, 0, BF16, M, none)
    X, W = dev(d.X, d.W)
    Y = torch.empty(M, 200, device=DEV)
    tcu.tcu_adapter_gemm(X, 300, W, 200, None, None, None, None, Y, 200, work_of(d), M, 300, 200,
                         16, 0)
    y, e = d.forward64()
    within(Y, y, e)


def test_adapter_empty():
    for size in ((0, 64, 64, 16, 2), (5, 0, 64, 16, 2), (5, 64, 0, 16, 2)):
        d = Layer(*size, BF16, 1)
        y, e = d.forward64()
        within(forward(d, FL), y, e)


@pytest.mark.parametrize("M", [2, 16, 40, 200, 600])
@pytest.mark.parametrize("types", PAIRS)
def test_adapter_rows_are_apart(M, types):
    """Values that are not finite in one row, or in an adapter, reach the rows that name
    them and no other."""
    G = 4
    d = Layer(M, 200, 136, 16, G, types[0], M, torch.arange(M) % (G + 1) - 1)
    clean = forward(d, types[1]).cpu()
    d.A[1, 3, 5] = float("nan")
    d.B[2, 7, 2] = float("inf")
    bad = (d.ids == 1) | (d.ids == 2)
    if M > 3:
        d.X[3, 0] = float("inf")
        bad[3] = True
    got = forward(d, types[1]).cpu()
    assert torch.equal(got[~bad], clean[~bad])
    assert bool(torch.isnan(got[d.ids == 1]).all())
    if M > 3 and bool((d.ids[4:] == 2).any()):
        row = int((d.ids[4:] == 2).nonzero()[0]) + 4
        assert not bool(torch.isfinite(got[row, 7])) and bool(torch.isfinite(got[row, :7]).all())


@pytest.mark.parametrize("M", [4, 100, 500])
def test_adapter_large_low_rank_sums(M):
    """X A^T beyond binary16's range with binary16 inputs."""
    d = Layer(M, 512, 64, 16, 2, F16, M)
    d.X = (d.X.float() * 100).to(F16)
    d.A = (d.A.float() * 1000).to(F16)
    assert float((d.X.double() @ d.A[0].double().t()).abs().max()) > 65504
    y, e = d.forward64()
    within(forward(d, FL), y, e)


@pytest.mark.parametrize("size", SIZES)
def test_adapter_q8(size):
    M, K, N, r, G = size
    d = Layer(*size, BF16, sum(size))
    g = gen(5)
    Xq = torch.randint(-127, 128, (M, K), generator=g, dtype=torch.int8)
    Wq = torch.randint(-128, 128, (K, N), generator=g, dtype=torch.int8)
    xs, ws = torch.rand(M, generator=g) / 127, torch.rand(N, generator=g) / 127
    low, mag = d.adapters64()
    base = (Xq.double() @ Wq.double()) * xs.double()[:, None] * ws.double()
    y = base + low
    e = base.abs() * 4 * F32 + mag * ((K + r + 8) * F32 + 2.0 ** -16) + y.abs() * 2.0 ** -8
    for pad in (0, 16, 5):
        a, b, x = pitched(Xq, K + pad)[1], pitched(Wq, N + pad)[1], pitched(d.X, K + pad)[1]
        yb, Y = pitched(torch.zeros(M, N, dtype=BF16), N + pad)
        work = work_of(d)
        tcu.tcu_adapter_gemm_q8(a, K + pad, xs.to(DEV), b, N + pad, ws.to(DEV), x, K + pad,
                                *dev(d.A, d.B, d.alpha, d.ids), Y, N + pad, work, M, K, N, r, G)
        within(Y, y, e)
        assert untouched(yb, M, N, N + pad) and bool((work[-64:] == 255).all())
    y0 = torch.empty(M, N, dtype=BF16, device=DEV)
    d0 = Layer(M, K, N, r, 0, BF16, 1)
    tcu.tcu_adapter_gemm_q8(Xq.to(DEV), K, xs.to(DEV), Wq.to(DEV), N, ws.to(DEV), None, 0, None,
                            None, None, None, y0, N, work_of(d0), M, K, N, r, 0)
    within(y0, base, base.abs() * (4 * F32 + 2.0 ** -8))


@pytest.mark.parametrize("types", PAIRS)
@pytest.mark.parametrize("size", SIZES)
def test_adapter_input_grad(size, types):
    d = Layer(*size, types[0], sum(size))
    y, e = d.input_grad64()
    for pad in (0, 3):
        dY, Wt = pitched(d.dY, d.N + pad)[1], pitched(d.W.t().contiguous(), d.K + pad)[1]
        xb, dX = pitched(torch.zeros(d.M, d.K, dtype=types[1]), d.K + pad)
        work = work_of(d)
        tcu.tcu_adapter_input_grad(dY, d.N + pad, Wt, d.K + pad, *dev(d.A, d.B, d.alpha, d.ids),
                                   dX, d.K + pad, work, d.M, d.K, d.N, d.r, d.G)
        within(dX, y, e + y.abs() * ROUND[types[1]])
        assert untouched(xb, d.M, d.K, d.K + pad) and bool((work[-64:] == 255).all())


def grads(d, pad=0):
    X, dY = pitched(d.X, d.K + pad)[1], pitched(d.dY, d.N + pad)[1]
    dA = torch.full(d.A.shape, float("nan"), device=DEV)
    dB = torch.full(d.B.shape, float("nan"), device=DEV)
    work = work_of(d)
    tcu.tcu_adapter_grad(X, d.K + pad, dY, d.N + pad, *dev(d.A, d.B, d.alpha, d.ids), dA, dB, work,
                         d.M, d.K, d.N, d.r, d.G)
    assert bool((work[-64:] == 255).all())
    return dA, dB


GRAD_SIZES = SIZES + [(5000, 200, 136, 16, 3), (3000, 64, 72, 32, 50), (0, 40, 40, 8, 2)]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("size", GRAD_SIZES)
def test_adapter_grad(size, dtype):
    d = Layer(*size, dtype, sum(size))
    A64, B64, eA, eB = d.grads64()
    for pad in (0, 3):
        dA, dB = grads(d, pad)
        within(dA, A64, eA)
        within(dB, B64, eB)
    again = grads(d, 3)
    assert torch.equal(again[0], dA) and torch.equal(again[1], dB)


def test_adapter_grad_one_adapter_and_sorted_runs():
    for ids in (torch.zeros(2500), torch.arange(2500) // 700, torch.full((2500,), -1)):
        d = Layer(2500, 300, 260, 16, 4, BF16, 11, ids)
        A64, B64, eA, eB = d.grads64()
        dA, dB = grads(d)
        within(dA, A64, eA)
        within(dB, B64, eB)


def test_adapter_grad_rows_are_apart():
    """A row that is not finite reaches its own adapter's gradients only."""
    d = Layer(300, 72, 88, 16, 3, BF16, 2, torch.arange(300) % 3)
    clean = grads(d)
    d.X[7, 3] = float("nan")      # adapter 1
    d.dY[10, 5] = float("inf")    # adapter 1
    got = grads(d)
    for a, b in zip(got, clean):
        assert torch.equal(a[[0, 2]], b[[0, 2]])
        assert not bool(torch.isfinite(a[1]).all())


@pytest.mark.parametrize("M", [7, 150, 400])
def test_gradients_against_differences(M):
    """The forward call is linear in A, in B and in X: central differences of
    sum(Y dY) are exact but for rounding where the shifted operand is exact too."""
    d = Layer(M, 96, 80, 16, 2, BF16, M)
    g = gen(M)

    def eighths(shape):
        return (torch.randint(-8, 9, shape, generator=g).double() / 8).to(BF16)

    d.A, d.B, d.X = eighths(d.A.shape), eighths(d.B.shape), eighths(d.X.shape)
    dA, dB = grads(d)
    dX = torch.empty(M, 96, device=DEV)
    tcu.tcu_adapter_input_grad(d.dY.to(DEV), 80, d.W.t().contiguous().to(DEV), 96,
                               *dev(d.A, d.B, d.alpha, d.ids), dX, 96, work_of(d), M, 96, 80, 16, 2)

    def loss():
        y, e = forward(d, FL).cpu().double(), d.forward64()[1]
        return float((y * d.dY.double()).sum()), float((e * d.dY.double().abs()).sum())

    for name, grad in (("A", dA), ("B", dB), ("X", dX)):
        at, v = getattr(d, name), eighths(getattr(d, name).shape)
        out = []
        for sign in (1, -1):
            setattr(d, name, (at.double() + sign * v.double()).to(BF16))
            out.append(loss())
        setattr(d, name, at)
        slope, err = (out[0][0] - out[1][0]) / 2, (out[0][1] + out[1][1]) / 2
        got = float((grad.cpu().double() * v.double()).sum())
        assert abs(got - slope) <= 2 * err, (name, got, slope, err)


@pytest.mark.parametrize("M", [4, 300])
def test_adapter_wide_offsets(M):
    """Rows of X and Y more than 2^32 bytes from their bases."""
    ld = (1 << 32) // M + 8
    d = Layer(M, 200, 136, 16, 3, BF16, 5)
    xb = torch.zeros((M - 1) * ld + 200, dtype=BF16, device=DEV)
    yb = torch.zeros((M - 1) * ld + 136, dtype=BF16, device=DEV)
    X, Y = xb.as_strided((M, 200), (ld, 1)), yb.as_strided((M, 136), (ld, 1))
    X.copy_(d.X)
    tcu.tcu_adapter_gemm(X, ld, d.W.to(DEV), 136, *dev(d.A, d.B, d.alpha, d.ids), Y, ld,
                         work_of(d), M, 200, 136, 16, 3)
    y, e = d.forward64()
    within(Y, y, e + y.abs() * ROUND[BF16])


def test_adapter_more_pieces_than_a_launch():
    """2^26 rows of one adapter: 2^22 pieces of 16 rows and some."""
    M = (1 << 26) + 33
    d = Layer(64, 8, 8, 4, 2, BF16, 3, torch.ones(64))
    reps = M // 64 + 1
    X = d.X.to(DEV).repeat(reps, 1)[:M]
    ids = torch.ones(M, dtype=torch.int32, device=DEV)
    ids[:100] = 0
    Y = torch.empty(M, 8, dtype=BF16, device=DEV)
    work = torch.empty(tcu.tcu_adapter_work(M, 8, 8, 4, 2), dtype=torch.uint8, device=DEV)
    tcu.tcu_adapter_gemm(X, 8, d.W.to(DEV), 8, *dev(d.A, d.B, d.alpha), ids, Y, 8, work, M, 8, 8, 4,
                         2)
    y, e = d.forward64()
    within(Y[128:192], y, e + y.abs() * ROUND[BF16])
    tail = Y[128:][:(M - 128) // 64 * 64].view(-1, 64, 8)
    assert bool((tail == tail[0]).all())
    rest = (M - 128) % 64
    assert torch.equal(Y[M - rest:], tail[0][:rest])


def test_adapter_other_stream_and_graph():
    d = Layer(48, 512, 640, 16, 6, BF16, 3)
    X, W, A, B, al, ids, dY = dev(d.X, d.W, d.A, d.B, d.alpha, d.ids, d.dY)
    Wt = d.W.t().contiguous().to(DEV)
    Y, dX = torch.empty(48, 640, dtype=BF16, device=DEV), torch.empty(48, 512, dtype=BF16, device=DEV)
    dA, dB = torch.empty(A.shape, device=DEV), torch.empty(B.shape, device=DEV)
    work = work_of(d)

    def step():
        tcu.tcu_adapter_gemm(X, 512, W, 640, A, B, al, ids, Y, 640, work, 48, 512, 640, 16, 6)
        tcu.tcu_adapter_grad(X, 512, dY, 640, A, B, al, ids, dA, dB, work, 48, 512, 640, 16, 6)
        tcu.tcu_adapter_input_grad(dY, 640, Wt, 512, A, B, al, ids, dX, 512, work, 48, 512, 640,
                                   16, 6)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    first = [t.clone() for t in (Y, dX, dA, dB)]
    y, e = d.forward64()
    within(first[0], y, e + y.abs() * ROUND[BF16])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        for t in (Y, dX, dA, dB):
            t.fill_(-1)
        ids.copy_((d.ids + k) % 7 - 1 if k else d.ids)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (Y, dX, dA, dB)]
        step()
        for a, b in zip(got, (Y, dX, dA, dB)):
            assert torch.equal(a, b)
        if k == 0:
            assert all(torch.equal(a, b) for a, b in zip(got, first))

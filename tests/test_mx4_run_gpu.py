"""The products in 4 bits and the heads' norms as a layer uses them together -- the norm, the
projection of queries, keys and values in 4 bits, the heads' norms with rotation, and
back -- eager, on another stream, captured and replayed, with pointer checks on, and with
graphs that have scratch of their own."""
import ctypes
import threading

import numpy as np
import pytest
import torch

from heads_util import TURN, angles, bound, forward64, grad64
from layer_util import DEV, F32 as EPS, ROUND, gen, norm64, randn, within
from mx4_util import rounded64
from paper_1908_06649_amd import tcu

pytestmark = pytest.mark.gpu
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8


class Layer:
    """A layer's first half: h = x + res, its norm, queries, keys and values by a weight in 4
    bits, the heads' norms with rotation; the gradients of all of it."""

    def __init__(self, T, K, hq, hk, D, seed=0):
        g = gen(seed)
        self.T, self.K, self.hq, self.hk, self.D = T, K, hq, hk, D
        self.N = N = (hq + 2 * hk) * D
        self.host = dict(x=randn((T, K), BF16, g), res=randn((T, K), BF16, g),
                         w=randn((K,), BF16, g), W=randn((N, K), BF16, g, K ** -0.5),
                         wq=randn((D,), BF16, g), wk=randn((D,), BF16, g),
                         freq=(1e4 ** (-torch.arange(0, D, 2).double() / D)).float(),
                         pos=torch.randint(0, 9000, (T,), generator=g).to(I32),
                         dyq=randn((T, hq, D), BF16, g), dyk=randn((T, hk, D), BF16, g),
                         dv=randn((T, hk, D), BF16, g))
        self.d = {k: v.to(DEV) for k, v in self.host.items()}
        e = lambda *s, t=BF16: torch.empty(s, dtype=t, device=DEV)
        self.o = dict(h=e(T, K), y=e(T, K), qkv=e(T, hq + 2 * hk, D), yq=e(hq, T, D), yk=e(hk, T, D),
                      dqkv=e(T, hq + 2 * hk, D), dwq=e(D, t=F32), dwk=e(D, t=F32), dY=e(T, K),
                      dW=e(N, K, t=F32))
        self.work = e(max(tcu.tcu_mx4_work(T, K, N), tcu.tcu_mx4_work(T, N, K),
                          tcu.tcu_mx4_work(N, T, K), tcu.tcu_qk_norm_grad_work(T, hq, hk, D)), t=U8)
        # the weight in 4 bits both ways, kept; the others' room
        self.held = {}
        for name, r, c in (("W", N, K), ("Wt", K, N), ("Y", T, K), ("Yt", K, T), ("G", T, N),
                           ("Gt", N, T)):
            self.held[name] = (e(r, tcu.tcu_mx4_row_bytes(c), t=U8),
                               e(tcu.tcu_mx4_row_words(c), r, t=I32))
        self.quant(self.d["W"], "W", "Wt", N, K)

    def quant(self, x, along, across, rows, cols):
        (q, s), (qt, ts) = self.held[along], self.held[across]
        tcu.tcu_mx4_quant(x, cols, q, q.shape[1], s, rows, qt, qt.shape[1], ts, cols, rows, cols)

    def product(self, a, b, C, M, K, N, flags=0):
        (A, sa), (B, sb) = self.held[a], self.held[b]
        tcu.tcu_mx4_gemm(A, A.shape[1], sa, M, B, B.shape[1], sb, N, C, N, self.work, M, K, N, flags)

    def run(self):
        T, K, N, hq, hk, D, d, o = (self.T, self.K, self.N, self.hq, self.hk, self.D, self.d, self.o)
        tcu.tcu_rms_norm(d["x"], K, d["res"], K, d["w"], o["h"], K, o["y"], K, None, 0, None, T, K,
                         1e-5)
        W, s = self.held["W"]
        tcu.tcu_mx4_linear(o["y"], K, W, W.shape[1], s, N, o["qkv"].view(T, N), N, self.work, T, K, N)
        q, k = o["qkv"][:, :hq], o["qkv"][:, hq:hq + hk]
        yq, yk = o["yq"].transpose(0, 1), o["yk"].transpose(0, 1)
        tcu.tcu_qk_norm(q, k, d["wq"], d["wk"], d["freq"], d["pos"], yq, yk, T, hq, hk, D, D, 1e-6)
        # back: the values' gradient as it comes, the heads' through their norms
        G = o["dqkv"]
        G[:, hq + hk:].copy_(d["dv"])
        tcu.tcu_qk_norm_grad(d["dyq"], d["dyk"], q, k, d["wq"], d["wk"], d["freq"], d["pos"],
                             G[:, :hq], G[:, hq:hq + hk], o["dwq"], o["dwk"], self.work, T, hq, hk,
                             D, D, 1e-6)
        self.quant(G.view(T, N), "G", "Gt", T, N)
        self.quant(o["y"], "Y", "Yt", T, K)
        self.product("G", "Wt", o["dY"], T, N, K)
        self.product("Gt", "Yt", o["dW"], N, T, K)

    def snapshot(self):
        torch.cuda.synchronize()
        return {k: v.clone() for k, v in self.o.items()}

    def check(self):
        """Every stage against binary64 on the values that went into it."""
        T, K, N, hq, hk = self.T, self.K, self.N, self.hq, self.hk
        o = {k: v.cpu() for k, v in self.o.items()}
        x = self.host
        h64, y64 = norm64(x["x"], x["res"], x["w"], 1e-5)
        within(o["y"], y64, bound(y64, y64.abs() * (K + 8) * EPS, BF16))
        W4, Y4 = rounded64(x["W"]), rounded64(o["y"])
        want, mag = Y4 @ W4.t(), Y4.abs() @ W4.abs().t()
        within(o["qkv"].view(T, N), want, bound(want, (K + 8) * EPS * mag, BF16))
        angle = angles(x["pos"], x["freq"])
        q, k = o["qkv"][:, :hq], o["qkv"][:, hq:hq + hk]
        rel = (self.D + 20) * EPS + TURN
        for y, v, w in ((o["yq"], q, "wq"), (o["yk"], k, "wk")):
            want, mag = forward64(v, x[w], angle, self.D, False, 1e-6)
            within(y.transpose(0, 1), want, bound(want, mag * rel, BF16))
        for dx, dy, v, w, H in ((o["dqkv"][:, :hq], x["dyq"], q, "wq", hq),
                                (o["dqkv"][:, hq:hq + hk], x["dyk"], k, "wk", hk)):
            want, dw, mag, wm = grad64(dy, v, x[w], angle, self.D, False, 1e-6)
            within(dx, want, bound(want, mag * 2 * rel, BF16))
            within(o["d" + w], dw, wm * (rel + T * H * EPS))
        G = o["dqkv"].reshape(T, N)
        for got, a, b, n in ((o["dY"], rounded64(G), rounded64(x["W"].t()), N),
                             (o["dW"], rounded64(G.t()), rounded64(o["y"].t()), T)):
            want, mag = a @ b.t(), a.abs() @ b.abs().t()
            within(got, want, (n + 8) * EPS * mag + want.abs() * ROUND[got.dtype])


SHAPES = [(1, 256, 4, 2, 64), (3, 300, 2, 1, 50), (33, 512, 4, 1, 80), (150, 640, 4, 2, 128),
          (700, 1000, 6, 2, 64)]


@pytest.mark.parametrize("shape", SHAPES)
def test_together(shape):
    layer = Layer(*shape)
    layer.run()
    layer.check()


@pytest.mark.parametrize("shape", SHAPES[::2])
def test_captured_and_replayed(shape):
    """Replays with the program's own eager work between them give what eager calls give."""
    layer = Layer(*shape)
    graph = torch.cuda.CUDAGraph()
    layer.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        layer.run()
    for seed in range(3):
        g = gen(seed)
        for k in ("x", "dyq", "dyk"):
            layer.host[k] = randn(layer.host[k].shape, BF16, g)
            layer.d[k].copy_(layer.host[k])
        layer.run()
        want = layer.snapshot()
        for t in layer.o.values():
            t.fill_(float("nan"))
        layer.work.fill_(255)
        torch.cuda.synchronize()
        graph.replay()
        got = layer.snapshot()
        assert all(torch.equal(got[k], want[k]) for k in want)
    layer.check()


def test_two_graphs_with_scratch_of_their_own():
    """Two layers' graphs replayed on two streams at once."""
    layers = [Layer(40, 512, 4, 2, 64, 1), Layer(200, 384, 2, 2, 96, 2)]
    want, graphs, streams = [], [], [torch.cuda.Stream() for _ in layers]
    for layer in layers:
        layer.run()
        want.append(layer.snapshot())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            layer.run()
        graphs.append(graph)
    for layer in layers:
        for t in layer.o.values():
            t.fill_(float("nan"))
    torch.cuda.synchronize()
    for _ in range(5):
        for graph, stream in zip(graphs, streams):
            with torch.cuda.stream(stream):
                graph.replay()
    for layer, w in zip(layers, want):
        got = layer.snapshot()
        assert all(torch.equal(got[k], w[k]) for k in w)


def test_another_stream():
    layer = Layer(20, 256, 2, 2, 64)
    layer.run()
    want = layer.snapshot()
    for t in layer.o.values():
        t.fill_(float("nan"))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer.run()
    stream.synchronize()
    assert all(torch.equal(layer.o[k], want[k]) for k in want)


def test_two_host_threads():
    """Two threads, a layer and a stream each, at once."""
    layers = [Layer(30, 256, 2, 2, 64, 3), Layer(50, 384, 3, 1, 80, 4)]
    want = []
    for layer in layers:
        layer.run()
        want.append(layer.snapshot())
    failures = []

    def go(layer, w):
        try:
            stream = torch.cuda.Stream()
            with torch.cuda.stream(stream):
                for _ in range(20):
                    for t in layer.o.values():
                        t.fill_(float("nan"))
                    layer.run()
                    stream.synchronize()
                    assert all(torch.equal(layer.o[k], w[k]) for k in w)
        except BaseException as e:   # (asserted in the test's own thread)
            failures.append(e)

    threads = [threading.Thread(target=go, args=a) for a in zip(layers, want)]
    torch.cuda.synchronize()
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failures


@pytest.mark.parametrize("M,K,N", [(1, 4096, 512), (40, 2048, 300), (300, 3000, 200),
                                   (1100, 8192, 1024), (4096, 512, 4096), (100, 40000, 64)])
def test_the_same_on_every_call(M, K, N):
    """Also where ranges of the contracted index are summed apart."""
    g = torch.Generator(device=DEV).manual_seed(1)
    rows = lambda r: (torch.randint(0, 256, (r, tcu.tcu_mx4_row_bytes(K)), generator=g, device=DEV,
                                    dtype=U8),
                      torch.randint(0x70, 0x80, (tcu.tcu_mx4_row_words(K), r), generator=g,
                                    device=DEV, dtype=I32) * 0x01010101)
    (A, a), (B, b) = rows(M), rows(N)
    work = torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=U8, device=DEV)
    first = None
    for _ in range(4):
        C = torch.empty(M, N, device=DEV)
        tcu.tcu_mx4_gemm(A, A.shape[1], a, M, B, B.shape[1], b, N, C, N, work, M, K, N)
        first = C if first is None else first
        assert torch.equal(C, first)
    # scratch of this batch is enough for a smaller one
    m = max(1, M // 3)
    C = torch.empty(m, N, device=DEV)
    tcu.tcu_mx4_gemm(A[:m], A.shape[1], a[:, :m], M, B, B.shape[1], b, N, C, N, work, m, K, N)
    off = (C - first[:m]).abs().max() / first.abs().max()
    assert float(off) < (K + 8) * EPS


# ------------------------------------------------------------------ pointer checks
M, K, N, HQ, HK, D = 40, 200, 30, 4, 2, 64
HELD = {"mk": (((M, 128), U8), ((2, M), I32)), "nk": (((N, 128), U8), ((2, N), I32)),
        "km": (((K, 64), U8), ((1, K), I32))}
WORK = ((1 << 25,), U8)
CALLS = {
    "tcu_mx4_quant": (
        dict(x=((M, K), BF16), q=HELD["mk"][0], s=HELD["mk"][1], qt=HELD["km"][0],
             ts=HELD["km"][1]),
        lambda p: (p["x"], K, p["q"], 128, p["s"], M, p["qt"], 64, p["ts"], K, M, K, 2, None)),
    "tcu_mx4_dequant": (
        dict(q=HELD["mk"][0], s=HELD["mk"][1], y=((M, K), F32)),
        lambda p: (p["q"], 128, p["s"], M, p["y"], K, M, K, 0, None)),
    "tcu_mx4_gemm": (
        dict(A=HELD["mk"][0], a=HELD["mk"][1], B=HELD["nk"][0], b=HELD["nk"][1], C=((M, N), BF16),
             work=WORK),
        lambda p: (p["A"], 128, p["a"], M, p["B"], 128, p["b"], N, p["C"], N, p["work"], M, K, N, 0,
                   2, None)),
    "tcu_mx4_linear": (
        dict(X=((M, K), BF16), W=HELD["nk"][0], w=HELD["nk"][1], Y=((M, N), BF16), work=WORK),
        lambda p: (p["X"], K, p["W"], 128, p["w"], N, p["Y"], N, p["work"], M, K, N, 0, 2, 2, None)),
    "tcu_qk_norm": (
        dict(q=((M, HQ, D), BF16), k=((M, HK, D), BF16), wq=((D,), BF16), wk=((D,), BF16),
             f=((D // 2,), F32), pos=((M,), I32), yq=((M, HQ, D), BF16), yk=((M, HK, D), BF16)),
        lambda p: (p["q"], HQ * D, D, p["k"], HK * D, D, p["wq"], p["wk"], p["f"], p["pos"], p["yq"],
                   HQ * D, D, p["yk"], HK * D, D, M, HQ, HK, D, D, 1e-5, 0, 2, None)),
    "tcu_qk_norm_grad": (
        dict(dyq=((M, HQ, D), BF16), dyk=((M, HK, D), BF16), q=((M, HQ, D), BF16),
             k=((M, HK, D), BF16), wq=((D,), BF16), wk=((D,), BF16), f=((D // 2,), F32),
             pos=((M,), I32), dq=((M, HQ, D), BF16), dk=((M, HK, D), BF16), dwq=((D,), F32),
             dwk=((D,), F32), work=WORK),
        lambda p: (p["dyq"], HQ * D, D, p["dyk"], HK * D, D, p["q"], HQ * D, D, p["k"], HK * D, D,
                   p["wq"], p["wk"], p["f"], p["pos"], p["dq"], HQ * D, D, p["dk"], HK * D, D,
                   p["dwq"], p["dwk"], p["work"], M, HQ, HK, D, D, 1e-5, 1, 2, None)),
}


@pytest.mark.parametrize("name", CALLS)
def test_host_operands_are_refused(name, knobs):
    """Every operand in turn on the host: refused before any launch, nothing counted."""
    knobs(tcu.TCU_KNOB_CHECK_POINTERS, 1)
    L = tcu.lib()
    host = np.zeros(1 << 26, dtype=np.uint8)
    hp = host.ctypes.data
    assert hp % 16 == 0 and L.tcu_check_device_range(hp, 1024) == tcu.TCU_ERR_POINTER
    shapes, args = CALLS[name]
    tensors = {k: torch.ones(s, dtype=t, device=DEV) for k, (s, t) in shapes.items()}
    addresses = {k: t.data_ptr() for k, t in tensors.items()}
    tcu.tcu_reset_calls()
    for k in tensors:
        assert getattr(L, name)(*args({**addresses, k: hp})) == tcu.TCU_ERR_POINTER, k
    torch.cuda.synchronize()
    assert tcu.tcu_calls() == 0 and not host.any()
    assert all(bool((t == 1).all()) for t in tensors.values())
    assert getattr(L, name)(*args(addresses)) == tcu.TCU_OK
    torch.cuda.synchronize()
    if name in ("tcu_mx4_gemm", "tcu_mx4_linear"):
        s = tcu.tcu_get_unit()
        assert tcu.tcu_calls() == -(-K // s) * -(-N // s)


def test_calls_from_c_take_their_stream():
    """The stream is the last argument: the same by ctypes on a stream of its own."""
    shapes, args = CALLS["tcu_mx4_linear"]
    tensors = {k: torch.ones(s, dtype=t, device=DEV) for k, (s, t) in shapes.items()}
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    full = args({k: t.data_ptr() for k, t in tensors.items()})
    assert tcu.lib().tcu_mx4_linear(*full[:-1], ctypes.c_void_p(stream.cuda_stream)) == tcu.TCU_OK
    stream.synchronize()
    # X = 1.  W: of every code byte 0x01 the even value is 1/2; a scale word 1 is byte 1 of the
    # group's first block, 0 of the others.
    want = sum(min(32, K - 32 * b) / 4 * 2.0 ** ((1 if b % 4 == 0 else 0) - 127) for b in range(7))
    assert torch.allclose(tensors["Y"].double().cpu(), torch.tensor(want).double().expand(M, N),
                          rtol=2.0 ** -8, atol=0)

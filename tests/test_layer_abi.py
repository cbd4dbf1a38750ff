"""Refusals of the operators around a layer's products: every bad argument is named
before any HIP call (fake pointers that are never dereferenced)."""
import ctypes

import pytest
import torch

from paper_1908_06649_amd import tcu

P = [0x100000000 + (i << 36) for i in range(16)]
NULL, SHAPE, UNSUP, ALIGN, OVER = (tcu.TCU_ERR_NULL, tcu.TCU_ERR_SHAPE, tcu.TCU_ERR_UNSUPPORTED,
                                   tcu.TCU_ERR_ALIGN, tcu.TCU_ERR_OVERLAP)
NAN, INF = float("nan"), float("inf")

CALLS = {
    "tcu_rms_norm": dict(x=P[0], ldx=64, res=P[1], ldr=64, w=P[2], h=P[3], ldh=64, y=P[4], ldy=64,
                         q=P[5], ldq=64, qscale=P[6], rows=10, cols=64, eps=1e-5, elem=2,
                         stream=None),
    "tcu_rms_norm_grad": dict(dy=P[0], lddy=64, h=P[1], ldh=64, w=P[2], dh=P[3], lddh=64, dx=P[4],
                              lddx=64, dw=P[5], work=P[6], rows=10, cols=64, eps=1e-5, elem=1,
                              stream=None),
    "tcu_adapter_gemm": dict(X=P[0], ldx=64, W=P[1], ldw=96, A=P[2], B=P[3], alpha=P[4], ids=P[5],
                             Y=P[6], ldy=96, work=P[7], M=10, K=64, N=96, r=16, G=3, dtype=2,
                             stream=None),
    "tcu_adapter_gemm_q8": dict(Xq=P[8], ldxq=64, xscale=P[9], Wq=P[1], ldwq=96, wscale=P[10],
                                X=P[0], ldx=64, A=P[2], B=P[3], alpha=P[4], ids=P[5], Y=P[6],
                                ldy=96, work=P[7], M=10, K=64, N=96, r=16, G=3, stream=None),
    "tcu_adapter_grad": dict(X=P[0], ldx=64, dY=P[1], lddy=96, A=P[2], B=P[3], alpha=P[4],
                             ids=P[5], dA=P[6], dB=P[7], work=P[8], M=10, K=64, N=96, r=16, G=3,
                             elem=2, stream=None),
    "tcu_adapter_input_grad": dict(dY=P[0], lddy=96, Wt=P[1], ldwt=64, A=P[2], B=P[3], alpha=P[4],
                                   ids=P[5], dX=P[6], lddx=64, work=P[7], M=10, K=64, N=96, r=16,
                                   G=3, dtype=1, stream=None),
}
NORM, GRAD = "tcu_rms_norm", "tcu_rms_norm_grad"
FWD, Q8, AG, IG = ("tcu_adapter_gemm", "tcu_adapter_gemm_q8", "tcu_adapter_grad",
                   "tcu_adapter_input_grad")
BIG = 1 << 30

REFUSED = [
    (NORM, dict(x=0), NULL), (NORM, dict(w=0), NULL), (NORM, dict(qscale=0), NULL),
    (NORM, dict(q=0), NULL), (NORM, dict(rows=-1), SHAPE), (NORM, dict(cols=0), SHAPE),
    (NORM, dict(rows=BIG + 1), SHAPE), (NORM, dict(ldx=63), SHAPE), (NORM, dict(ldq=63), SHAPE),
    (NORM, dict(ldx=1 << 36), SHAPE), (NORM, dict(eps=-1.0), SHAPE), (NORM, dict(eps=NAN), SHAPE),
    (NORM, dict(eps=INF), SHAPE), (NORM, dict(elem=3), UNSUP), (NORM, dict(elem=-1), UNSUP),
    (NORM, dict(x=P[0] + 2), ALIGN), (NORM, dict(q=P[5] + 1), ALIGN),
    (NORM, dict(qscale=P[6] + 2), ALIGN), (NORM, dict(y=P[0]), OVER),
    (NORM, dict(h=P[0], ldh=72), OVER), (NORM, dict(h=P[0] + 16), OVER),
    (NORM, dict(y=P[3] + 9 * 128), OVER), (NORM, dict(qscale=P[2] + 124), OVER),
    (GRAD, dict(dy=0), NULL), (GRAD, dict(h=0), NULL), (GRAD, dict(dw=0), NULL),
    (GRAD, dict(dx=0), NULL), (GRAD, dict(work=0), NULL), (GRAD, dict(lddx=60), SHAPE),
    (GRAD, dict(cols=BIG + 1), SHAPE), (GRAD, dict(elem=7), UNSUP), (GRAD, dict(work=P[6] + 8), ALIGN),
    (GRAD, dict(dw=P[5] + 2), ALIGN), (GRAD, dict(dx=P[1]), OVER), (GRAD, dict(work=P[4]), OVER),
    (GRAD, dict(dw=P[6] + 16), OVER), (GRAD, dict(dx=P[3] + 128), OVER),
]
for f, left, right, out in ((FWD, "X", "W", "Y"), (Q8, "X", "Wq", "Y"), (IG, "dY", "Wt", "dX"),
                            (AG, "X", "dY", "dA")):
    REFUSED += [(f, {k: 0}, NULL) for k in (left, right, "A", "B", "alpha", "ids", out, "work")]
    REFUSED += [(f, {k: v}, SHAPE) for k, v in (("M", -1), ("K", -1), ("N", -5), ("M", BIG + 1),
                                                ("r", 0), ("r", 129), ("G", -1), ("G", 65537),
                                                ("K", (1 << 24) + 1), ("N", (1 << 24) + 1))]
    REFUSED += [(f, {k: CALLS[f][k] + 2}, ALIGN) for k in (left, "A", "B", out, "work", "ids")]
    REFUSED += [(f, {out: CALLS[f][left]}, OVER), (f, {out: CALLS[f]["A"]}, OVER),
                (f, dict(work=CALLS[f][right]), OVER), (f, {"work": CALLS[f][out]}, OVER)]
REFUSED += [
    (FWD, dict(ldx=63), SHAPE), (FWD, dict(ldy=95), SHAPE), (FWD, dict(dtype=3), UNSUP),
    (FWD, dict(dtype=-1), UNSUP), (FWD, dict(M=BIG, K=BIG, ldx=BIG), SHAPE),
    (Q8, dict(Xq=0), NULL), (Q8, dict(xscale=0), NULL), (Q8, dict(wscale=0), NULL),
    (Q8, dict(K=1 << 17, ldx=1 << 17, ldxq=1 << 17), SHAPE), (Q8, dict(ldwq=95), SHAPE),
    (Q8, dict(Xq=P[8] + 8), ALIGN), (Q8, dict(wscale=P[10] + 1), ALIGN),
    (Q8, dict(Y=P[9] - 16), OVER), (AG, dict(elem=0), UNSUP), (AG, dict(K=0), SHAPE),
    (AG, dict(N=0), SHAPE), (AG, dict(dB=0), NULL), (AG, dict(dB=P[6] + 64), OVER),
    (AG, dict(dA=P[6] + 4), ALIGN), (IG, dict(ldwt=63), SHAPE), (IG, dict(lddy=95), SHAPE),
    (IG, dict(dtype=3), UNSUP)]


@pytest.mark.parametrize("name,change,want", REFUSED)
def test_refused(name, change, want):
    lib = tcu.lib()
    lib.tcu_reset_calls()
    assert getattr(lib, name)(*{**CALLS[name], **change}.values()) == want
    assert lib.tcu_calls() == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="valid arguments with fake pointers")
@pytest.mark.parametrize("name", sorted(CALLS))
@pytest.mark.parametrize("change", [{}, "in place", "absent"])
def test_valid_arguments_reach_the_device_query(name, change):
    if change == "in place":
        change = {NORM: dict(h=P[0]), GRAD: dict(dx=P[3])}.get(name, {})
    elif change == "absent":
        change = {NORM: dict(res=0, q=0, qscale=0, h=0), GRAD: dict(dh=0)}.get(
            name, dict(G=0, A=0, B=0, alpha=0, ids=0))
        if name == AG:
            change = dict(M=0, X=0, dY=0, ids=0)
    assert getattr(tcu.lib(), name)(*{**CALLS[name], **change}.values()) == tcu.TCU_ERR_NO_DEVICE


def test_nothing_to_do():
    lib = tcu.lib()
    assert lib.tcu_rms_norm(*{**CALLS[NORM], "rows": 0, "x": 0}.values()) == tcu.TCU_OK
    for f in (FWD, Q8, IG):
        assert getattr(lib, f)(*{**CALLS[f], "M": 0}.values()) == tcu.TCU_OK
    assert lib.tcu_adapter_grad(*{**CALLS[AG], "G": 0}.values()) == tcu.TCU_OK


def test_work_sizes():
    lib = tcu.lib()
    assert lib.tcu_rms_norm_grad_work(-1, 4) == -1 and lib.tcu_rms_norm_grad_work(4, 0) == -1
    assert lib.tcu_adapter_work(-1, 4, 4, 4, 4) == -1 and lib.tcu_adapter_work(4, 4, 4, 129, 4) == -1
    assert lib.tcu_adapter_work(BIG, BIG, BIG, 16, 4) >= -1
    for size in ((1, 1, 1, 1, 0), (0, 64, 64, 16, 2), (5, 0, 64, 16, 2), (5, 64, 0, 16, 2),
                 (0, 0, 0, 1, 0), (64, 8192, 8192, 128, 65536), (5000, 4096, 4096, 16, 8)):
        assert 0 <= lib.tcu_adapter_work(*size) < 1 << 40
    assert lib.tcu_clip_grads_work() > 0


def clip(grads, outs, counts, elems, max_norm=1.0, result=P[14], work=P[15]):
    n = len(grads)
    return tcu.lib().tcu_clip_grads((ctypes.c_void_p * n)(*grads), (ctypes.c_void_p * n)(*outs),
                                    (ctypes.c_int64 * n)(*counts), (ctypes.c_int32 * n)(*elems), n,
                                    max_norm, result, work, None)


@pytest.mark.parametrize("args,want", [
    (([P[0]], [P[1]], [10], [3]), UNSUP), (([P[0]], [P[1]], [-1], [0]), SHAPE),
    (([P[0]], [P[1]], [1 << 40], [0]), SHAPE), (([0], [P[1]], [10], [0]), NULL),
    (([P[0]], [0], [10], [0]), NULL), (([P[0] + 2], [P[1]], [10], [0]), ALIGN),
    (([P[0]], [P[1] + 1], [10], [1]), ALIGN), (([P[0]], [P[0] + 4], [10], [0]), OVER),
    (([P[0], P[1]], [P[2], P[0] + 8], [10, 10], [0, 0]), OVER),
    (([P[0], P[1]], [P[2], P[2] + 36], [10, 10], [0, 0]), OVER),
    (([P[0], P[0]], [P[0], P[2]], [10, 10], [0, 0]), OVER),
    (([P[0]], [P[1]], [10], [0], -1.0), SHAPE), (([P[0]], [P[1]], [10], [0], NAN), SHAPE),
    (([P[0]], [P[1]], [10], [0], 1.0, 0), NULL), (([P[0]], [P[1]], [10], [0], 1.0, P[14], 0), NULL),
    (([P[0]], [P[1]], [10], [0], 1.0, P[14] + 2), ALIGN),
    (([P[0]], [P[1]], [10], [0], 1.0, P[14], P[15] + 4), ALIGN),
    (([P[0]], [P[14]], [10], [0]), OVER), (([P[15] + 8], [P[1]], [10], [0]), OVER)])
def test_clip_refused(args, want):
    assert clip(*args) == want


@pytest.mark.skipif(torch.cuda.is_available(), reason="valid arguments with fake pointers")
def test_clip_valid():
    ok = tcu.TCU_ERR_NO_DEVICE
    assert clip([P[0], 0], [P[0], 0], [10, 0], [0, 2]) == ok
    assert clip([P[0], P[0]], [P[1], P[2]], [10, 5], [0, 1]) == ok     # inputs may share
    assert clip([P[0] + 2], [P[1] + 2], [10], [1]) == ok
    assert clip([], [], [], []) == ok
    assert clip([P[0]], [P[0] + 40], [10], [0]) == ok


def test_python_refuses_host_and_mismatched_tensors():
    b = torch.bfloat16
    x, w = torch.zeros(4, 8, dtype=b), torch.zeros(8, dtype=b)
    with pytest.raises(ValueError):
        tcu.tcu_rms_norm(x, 8, None, 0, w, None, 0, x.clone(), 8, None, 0, None, 4, 8, 1e-5)
    with pytest.raises(ValueError):
        tcu.tcu_rms_norm(x, 8, x.float(), 8, w, None, 0, None, 0, None, 0, None, 4, 8, 1e-5)
    with pytest.raises(ValueError):
        tcu.tcu_rms_norm(x, 9, None, 0, w, None, 0, None, 0, None, 0, None, 4, 8, 1e-5)
    with pytest.raises(tcu.TcuError):
        tcu.tcu_rms_norm(x.double(), 8, None, 0, w, None, 0, None, 0, None, 0, None, 4, 8, 1e-5)
    with pytest.raises(tcu.TcuError):
        tcu.tcu_adapter_gemm(x.float(), 8, w, 8, None, None, None, None, x, 8, None, 4, 8, 8, 4, 0)

"""Refusals of the products in 4 bits and of the heads' norms: every bad argument is named
before any HIP call (fake pointers that are never dereferenced)."""
import pytest
import torch

from paper_1908_06649_amd import tcu

P = [0x100000000 + (i << 36) for i in range(16)]
NULL, SHAPE, UNSUP, ALIGN, OVER = (tcu.TCU_ERR_NULL, tcu.TCU_ERR_SHAPE, tcu.TCU_ERR_UNSUPPORTED,
                                   tcu.TCU_ERR_ALIGN, tcu.TCU_ERR_OVERLAP)
NAN, INF = float("nan"), float("inf")
BIG = 1 << 27

QUANT, BACK, GEMM, LIN = "tcu_mx4_quant", "tcu_mx4_dequant", "tcu_mx4_gemm", "tcu_mx4_linear"
QK, QKG = "tcu_qk_norm", "tcu_qk_norm_grad"
CALLS = {
    # 10 x 200 values: rows of 128 bytes and 2 words; 200 x 10: 64 bytes and 1 word
    QUANT: dict(x=P[0], ldx=200, q=P[1], ldq=128, scale=P[2], lds=10, qt=P[3], ldqt=64, tscale=P[4],
                ldts=200, rows=10, cols=200, elem=2, stream=None),
    BACK: dict(q=P[0], ldq=128, scale=P[1], lds=10, y=P[2], ldy=200, rows=10, cols=200, elem=0,
               stream=None),
    GEMM: dict(A=P[0], lda=128, ascale=P[1], ldas=10, B=P[2], ldb=128, bscale=P[3], ldbs=30, C=P[4],
               ldc=30, work=P[5], M=10, K=200, N=30, flags=0, elem=1, stream=None),
    LIN: dict(X=P[0], ldx=200, W=P[2], ldw=128, wscale=P[3], ldws=30, Y=P[4], ldy=30, work=P[5],
              M=10, K=200, N=30, flags=1, xelem=2, elem=0, stream=None),
    # 7 tokens of 4 and 2 heads of 64 in rows of 512
    QK: dict(q=P[0], ldq=512, hdq=64, k=P[0] + 512, ldk=512, hdk=64, wq=P[1], wk=P[2], freq=P[3],
             pos=P[4], yq=P[5], ldyq=256, hdyq=64, yk=P[6], ldyk=64, hdyk=448, tokens=7, hq=4, hk=2,
             dim=64, rot=64, eps=1e-5, flags=0, elem=2, stream=None),
    QKG: dict(dyq=P[7], lddyq=256, hddyq=64, dyk=P[8], lddyk=64, hddyk=448, q=P[0], ldq=512, hdq=64,
              k=P[0] + 512, ldk=512, hdk=64, wq=P[1], wk=P[2], freq=P[3], pos=P[4], dq=P[5],
              lddq=512, hddq=64, dk=P[5] + 512, lddk=512, hddk=64, dwq=P[9], dwk=P[10], work=P[11],
              tokens=7, hq=4, hk=2, dim=64, rot=32, eps=0.0, flags=1, elem=2, stream=None),
}

REFUSED = [
    (QUANT, dict(x=0), NULL), (QUANT, dict(q=0), NULL), (QUANT, dict(scale=0), NULL),
    (QUANT, dict(qt=0), NULL), (QUANT, dict(tscale=0), NULL), (QUANT, dict(rows=-1), SHAPE),
    (QUANT, dict(cols=-1), SHAPE), (QUANT, dict(rows=BIG + 1), SHAPE),
    (QUANT, dict(cols=BIG + 1), SHAPE), (QUANT, dict(ldx=199), SHAPE), (QUANT, dict(ldq=112), SHAPE),
    (QUANT, dict(lds=9), SHAPE), (QUANT, dict(ldqt=48), SHAPE), (QUANT, dict(ldts=199), SHAPE),
    (QUANT, dict(ldq=(1 << 26) + 16), SHAPE), (QUANT, dict(ldqt=(1 << 26) + 16), SHAPE),
    (QUANT, dict(ldq=136), ALIGN), (QUANT, dict(ldqt=72), ALIGN), (QUANT, dict(elem=3), UNSUP),
    (QUANT, dict(elem=-1), UNSUP), (QUANT, dict(x=P[0] + 2), ALIGN), (QUANT, dict(q=P[1] + 8), ALIGN),
    (QUANT, dict(scale=P[2] + 2), ALIGN), (QUANT, dict(qt=P[3] + 4), ALIGN),
    (QUANT, dict(tscale=P[4] + 1), ALIGN), (QUANT, dict(q=P[0]), OVER), (QUANT, dict(qt=P[1]), OVER),
    (QUANT, dict(tscale=P[2]), OVER), (QUANT, dict(scale=P[0] + 396), OVER),
    (BACK, dict(q=0), NULL), (BACK, dict(scale=0), NULL), (BACK, dict(y=0), NULL),
    (BACK, dict(ldy=199), SHAPE), (BACK, dict(ldq=127), SHAPE), (BACK, dict(lds=9), SHAPE),
    (BACK, dict(cols=BIG + 1), SHAPE), (BACK, dict(ldq=129), ALIGN), (BACK, dict(y=P[2] + 4), ALIGN),
    (BACK, dict(elem=5), UNSUP), (BACK, dict(y=P[0]), OVER), (BACK, dict(y=P[1] - 16), OVER),
    (QUANT, dict(rows=1, ldq=3), SHAPE), (GEMM, dict(M=1, lda=5), SHAPE),
    (GEMM, dict(flags=2), UNSUP), (GEMM, dict(elem=3), UNSUP), (GEMM, dict(lda=120), SHAPE),
    (GEMM, dict(ldas=9), SHAPE), (GEMM, dict(A=0), NULL), (GEMM, dict(ascale=0), NULL),
    (GEMM, dict(lda=130), ALIGN), (GEMM, dict(lda=(1 << 26) + 16), SHAPE),
    (GEMM, dict(A=P[0] + 8), ALIGN), (GEMM, dict(ascale=P[1] + 2), ALIGN),
    (GEMM, dict(C=P[1]), OVER), (GEMM, dict(work=P[0]), OVER),
    (LIN, dict(X=0), NULL), (LIN, dict(ldx=199), SHAPE), (LIN, dict(xelem=0), UNSUP),
    (LIN, dict(xelem=1, elem=2), UNSUP), (LIN, dict(elem=1), UNSUP), (LIN, dict(flags=-1), UNSUP),
    (LIN, dict(X=P[0] + 2), ALIGN), (LIN, dict(Y=P[0]), OVER),
]
for f, b, bs, c, ldb, ldbs, ldc in ((GEMM, "B", "bscale", "C", "ldb", "ldbs", "ldc"),
                                    (LIN, "W", "wscale", "Y", "ldw", "ldws", "ldy")):
    REFUSED += [(f, {k: 0}, NULL) for k in (b, bs, c, "work")]
    REFUSED += [(f, {k: v}, SHAPE) for k, v in (("M", -1), ("K", -1), ("N", -1), ("M", BIG + 1),
                                                ("K", BIG + 1), ("N", BIG + 1), (ldc, 29),
                                                (ldb, 112), (ldbs, 29))]
    REFUSED += [(f, {ldb: 136}, ALIGN), (f, {bs: P[3] + 2}, ALIGN), (f, {c: P[4] + 4}, ALIGN),
                (f, dict(work=P[5] + 8), ALIGN), (f, {c: P[2]}, OVER), (f, {c: P[3] + 16}, OVER),
                (f, {"work": P[4]}, OVER), (f, dict(M=BIG, N=BIG, **{ldc: BIG}), SHAPE)]
for f in (QK, QKG):
    REFUSED += [(f, {k: 0}, NULL) for k in ("q", "k", "wq", "wk", "freq", "pos")]
    REFUSED += [(f, {k: v}, SHAPE) for k, v in (
        ("tokens", -1), ("tokens", (1 << 30) + 1), ("hq", -1), ("hk", 65537), ("dim", 0),
        ("dim", 1025), ("rot", -2), ("rot", 66), ("rot", 31), ("eps", -1.0), ("eps", NAN),
        ("eps", INF), ("hdq", 63), ("ldq", 200), ("hdq", -64), ("ldk", -512), ("ldq", 1 << 62),
        ("hdk", 1 << 62), ("hdq", 512))]
    REFUSED += [(f, {k: v}, UNSUP) for k, v in (("elem", 3), ("elem", -1), ("flags", 2),
                                                ("flags", -1))]
    REFUSED += [(f, {k: CALLS[f][k] + 1}, ALIGN) for k in ("q", "k")]
    REFUSED += [(f, dict(wq=P[1] + 8), ALIGN), (f, dict(freq=P[3] + 2), ALIGN),
                (f, dict(pos=P[4] + 2), ALIGN)]
REFUSED += [
    (QK, dict(yq=0), NULL), (QK, dict(yk=0), NULL), (QK, dict(yq=P[5] + 1), ALIGN),
    (QK, dict(yq=P[0]), OVER), (QK, dict(yq=P[0], ldyq=512, hdyq=72), OVER),
    (QK, dict(yk=P[0] + 512, ldyk=512, hdyk=64, yq=P[0] + 128, ldyq=512), OVER),
    (QK, dict(yq=P[0] + 512, ldyq=512), OVER), (QK, dict(yk=P[5] + 500), OVER),
    (QK, dict(yk=P[1]), OVER), (QK, dict(yq=P[4] - 64), OVER), (QK, dict(yk=P[3]), OVER),
    (QK, dict(hdyk=447), SHAPE), (QK, dict(ldyq=255), SHAPE),
    (QKG, dict(dyq=0), NULL), (QKG, dict(dyk=0), NULL), (QKG, dict(dq=0), NULL),
    (QKG, dict(dwq=0), NULL), (QKG, dict(dwk=0), NULL), (QKG, dict(work=0), NULL),
    (QKG, dict(work=P[11] + 8), ALIGN), (QKG, dict(dwq=P[9] + 2), ALIGN),
    (QKG, dict(dq=P[7] + 2, lddq=256), OVER), (QKG, dict(dq=P[8]), OVER),
    (QKG, dict(dk=P[5]), OVER), (QKG, dict(dwq=P[10] + 252), OVER), (QKG, dict(work=P[0]), OVER),
    (QKG, dict(dwk=P[11] + 16), OVER), (QKG, dict(hddyk=440), SHAPE)]


@pytest.mark.parametrize("name,change,want", REFUSED)
def test_refused(name, change, want):
    lib = tcu.lib()
    lib.tcu_reset_calls()
    assert getattr(lib, name)(*{**CALLS[name], **change}.values()) == want
    assert lib.tcu_calls() == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="valid arguments with fake pointers")
@pytest.mark.parametrize("name,change", [(n, {}) for n in CALLS] + [
    (QUANT, dict(q=0, scale=0)), (QUANT, dict(qt=0, tscale=0)),
    (QUANT, dict(rows=1, ldq=131)), (GEMM, dict(K=0, A=0, ascale=0, B=0, bscale=0)),
    (LIN, dict(K=0, X=0, W=0, wscale=0, flags=0)), (LIN, dict(xelem=1, elem=1)),
    (GEMM, dict(ldas=1 << 30)), (GEMM, dict(M=1, lda=129)),
    (QK, dict(yq=P[0], ldyq=512)), (QK, dict(yq=P[0], ldyq=512, yk=P[0] + 512, ldyk=512, hdyk=64)),
    (QK, dict(hk=0, k=0, yk=0, wk=0)), (QK, dict(hq=0, q=0, yq=0, wq=0)),
    (QK, dict(rot=0, freq=0, pos=0)), (QK, dict(q=P[0] + 2, k=P[0] + 514, yq=P[5] + 6)),
    (QK, dict(tokens=1, ldq=0, ldk=-5, ldyq=1)), (QK, dict(hq=1, hdq=0, hdyq=-1)),
    (QKG, dict(dq=P[7], lddq=256)), (QKG, dict(dk=P[0] + 512)),
    (QKG, dict(dq=P[0], dk=P[0] + 512)), (QKG, dict(hk=0, k=0, dyk=0, dk=0, wk=0, dwk=0)),
    (QKG, dict(tokens=0, q=0, k=0, dyq=0, dyk=0, dq=0, dk=0, pos=0, wq=0, wk=0, freq=0))])
def test_valid_arguments_reach_the_device_query(name, change):
    assert getattr(tcu.lib(), name)(*{**CALLS[name], **change}.values()) == tcu.TCU_ERR_NO_DEVICE


@pytest.mark.parametrize("name,change", [
    (QUANT, dict(rows=0)), (QUANT, dict(cols=0)), (QUANT, dict(q=0, scale=0, qt=0, tscale=0)),
    (BACK, dict(rows=0)), (BACK, dict(cols=0, q=0, scale=0, y=0)), (GEMM, dict(M=0)),
    (GEMM, dict(N=0)), (GEMM, dict(K=0, flags=1)), (LIN, dict(M=0, X=0)), (LIN, dict(K=0)),
    (QK, dict(tokens=0)), (QK, dict(hq=0, hk=0)), (QKG, dict(hq=0, hk=0))])
def test_nothing_to_do(name, change):
    assert getattr(tcu.lib(), name)(*{**CALLS[name], **change}.values()) == tcu.TCU_OK


def test_work_sizes():
    lib = tcu.lib()
    assert lib.tcu_mx4_work(-1, 4, 4) == lib.tcu_mx4_work(4, BIG + 1, 4) == -1
    assert lib.tcu_mx4_work(BIG, BIG, 4) == -1      # X in 4 bits is out of range
    assert lib.tcu_qk_norm_grad_work(-1, 1, 1, 64) == lib.tcu_qk_norm_grad_work(1, 1, 1, 1025) == -1
    last = 0
    for M in (0, 1, 5, 64, 65, 1000, 8192, 100000):     # enough for fewer rows
        now = lib.tcu_mx4_work(M, 4096, 4096)
        assert last <= now < 1 << 40
        last = now
    assert lib.tcu_qk_norm_grad_work(0, 8, 2, 128) == lib.tcu_qk_norm_grad_work(1 << 20, 8, 2, 128)
    assert tcu.tcu_mx4_row_bytes(129) == 128 and tcu.tcu_mx4_row_words(129) == 2
    assert tcu.tcu_mx4_row_bytes(0) == 0 and tcu.tcu_mx4_row_words(128) == 1


def test_python_refuses_host_and_mismatched_tensors():
    b = torch.bfloat16
    x, q = torch.zeros(4, 8, dtype=b), torch.zeros(4, 64, dtype=torch.uint8)
    s = torch.zeros(1, 4, dtype=torch.int32)
    for bad in ((x, 8, q, 64, s, 4), (x, 8, q.int(), 64, s, 4), (x, 8, q[:, :32], 64, s, 4),
                (x, 8, q, 64, s.t(), 4)):
        with pytest.raises(ValueError):
            tcu.tcu_mx4_quant(*bad, None, 0, None, 0, 4, 8)
    with pytest.raises(tcu.TcuError):
        tcu.tcu_mx4_quant(x.double(), 8, q, 64, s, 4, None, 0, None, 0, 4, 8)
    h = torch.zeros(4, 2, 8, dtype=b)
    w, f, p = torch.zeros(8, dtype=b), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    for q, k, pos in ((h, h, p), (h.float(), h, p), (h, h[:, :1], p), (h, h, p.long()),
                      (h[0], h, p), (h.transpose(1, 2), h, p)):
        with pytest.raises(ValueError):
            tcu.tcu_qk_norm(q, k, w, w, f, pos, h, h, 4, 2, 2, 8, 8, 1e-5)

"""The operators of an adapted layer that the library is timed on: what feeds a
projection, what rides on it and what takes its gradients, from single tokens
to the largest batches.

A case is a dict of plain values; ``kind`` names what one pass computes:

    norm         tcu_rms_norm              rows, cols, dtype, res (a residual is added)
    norm_grad    tcu_rms_norm_grad         rows, cols, dtype, res (the residual stream's
                                           gradient is added)
    adapter      tcu_adapter_gemm          M, K, N, r, G, dtype, order, pad
    serve8       tcu_rms_norm with 8-bit   M, K, N, r, G, order
                 output, then
                 tcu_adapter_gemm_q8
    adapter_grad tcu_adapter_grad and      M, K, N, r, G, dtype, order
                 tcu_adapter_input_grad
    clip         tcu_clip_grads            tensors, size (mean elements), dtype

M rows are tokens; K and N the layer's inputs and outputs; r the adapters'
rank and G how many are held.  ``order`` is how the rows' adapters lie: "runs"
(prompts or sequences one after the other, each with its adapter, a few with
none) or "mixed" (single tokens of many requests).  ``own`` chooses between the
library's calls and the same operators in elementary torch operations.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-5
MAX_NORM = 1.0
# dtype name -> (input type, output type) of the projections
DTYPES = {"f16": (torch.float16, torch.float32),
          "bf16": (torch.bfloat16, torch.float32),
          "bf16out": (torch.bfloat16, torch.bfloat16)}
# dtype name -> element type of the norms and of the clipped gradients
ELEMS = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # The norm before a projection while 16 requests each generate a token.
        dict(name="norm_bf16_16x4096", kind="norm", rows=16, cols=4096, dtype="bf16", res=True),
        # The same over a batch of prompts: memory bandwidth.
        dict(name="norm_bf16_8192x8192", kind="norm", rows=8192, cols=8192, dtype="bf16",
             res=True),
        # Its gradient in training, rows that start at 8-byte addresses.
        dict(name="norm_grad_bf16_6007x4100", kind="norm_grad", rows=6007, cols=4100,
             dtype="bf16", res=True),
        # One token of each of 8 requests, every one with an adapter of its own.
        dict(name="adapter_bf16_8x4096x4096_r16", kind="adapter", M=8, K=4096, N=4096, r=16, G=8,
             dtype="bf16out", order="mixed", pad=0),
        # Sizes as data has them: odd dimensions, a rank below the unit's, rows at
        # any 2-byte address.
        dict(name="adapter_f16_1000x1003x2005_r8", kind="adapter", M=1000, K=1003, N=2005, r=8,
             G=3, dtype="f16", order="runs", pad=0),
        # Prompts of several requests that arrive together.
        dict(name="adapter_bf16_2000x4096x4096_r16", kind="adapter", M=2000, K=4096, N=4096,
             r=16, G=12, dtype="bf16out", order="runs", pad=0),
        # The largest projection, four adapters trained or served at once.
        dict(name="adapter_bf16_8192x8192x8192_r32", kind="adapter", M=8192, K=8192, N=8192,
             r=32, G=4, dtype="bf16out", order="runs", pad=0),
        # An 8-bit layer generating tokens for 48 requests with 16 adapters.
        dict(name="serve8_48x8192x8192_r16", kind="serve8", M=48, K=8192, N=8192, r=16, G=16,
             order="mixed"),
        # The same layer reading prompts.
        dict(name="serve8_4096x4096x8192_r16", kind="serve8", M=4096, K=4096, N=8192, r=16, G=8,
             order="runs"),
        # The gradients of one adapted layer, four adapters in one batch.
        dict(name="adapter_grad_bf16_8192x4096x4096_r16", kind="adapter_grad", M=8192, K=4096,
             N=4096, r=16, G=4, dtype="bf16out", order="runs"),
        # The adapters' gradients of a small model, clipped by their common norm.
        dict(name="clip_f32_48x65536", kind="clip", tensors=48, size=65536, dtype="f32"),
        # The gradients of whole weights.
        dict(name="clip_bf16_32x16777216", kind="clip", tensors=32, size=1 << 24, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _any_or_round(rng, v, unit):
    """v as it is, or as a multiple of `unit`: programs pass both."""
    return max(unit, v // unit * unit) if rng.random() < 0.6 else v


def draw(rng):
    kind = rng.choice(["norm", "norm_grad", "adapter", "adapter", "serve8", "adapter_grad",
                       "clip"])
    if kind in ("norm", "norm_grad"):
        cols = _any_or_round(rng, _log_int(rng, 64, 16384), 64)
        rows = _log_int(rng, 1, min(65536, (1 << 26) // cols))
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(list(ELEMS)),
                    res=rng.random() < 0.7)
    if kind == "clip":
        tensors = rng.randint(1, 56)
        size = _log_int(rng, 64, (1 << 28) // tensors)
        return dict(kind=kind, tensors=tensors, size=size, dtype=rng.choice(list(ELEMS)))
    K = _any_or_round(rng, _log_int(rng, 64, 8192), 64)
    N = _any_or_round(rng, _log_int(rng, 64, 8192), 64)
    r = rng.choice([4, 8, 16, 16, 32, 32, 64])
    G = _log_int(rng, 1, 32)
    # below the largest listed product
    most = max(1, (1 << 38) // (K * N))
    if kind == "adapter_grad":
        M = min(most, _log_int(rng, 1, 8192))
        return dict(kind=kind, M=M, K=K, N=N, r=r, G=G, dtype=rng.choice(list(DTYPES)),
                    order="runs")
    M = _log_int(rng, 1, 128) if rng.random() < 0.5 else min(most, _log_int(rng, 128, 8192))
    order = "mixed" if M <= 128 else rng.choice(["runs", "runs", "mixed"])
    if kind == "serve8":
        return dict(kind=kind, M=M, K=K, N=N, r=r, G=G, order=order)
    return dict(kind=kind, M=M, K=K, N=N, r=r, G=G, dtype=rng.choice(list(DTYPES)), order=order,
                pad=rng.choice([0, 0, 64, rng.randint(1, 63)]))


# ------------------------------------------------------------------ inputs
def _gen(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed)
    return g


def _randn(shape, dtype, g, scale=1.0):
    return torch.randn(shape, generator=g, device=DEVICE).mul_(scale).to(dtype)


def _padded(t, pad):
    """t as a view of rows `pad` elements longer."""
    if not pad:
        return t
    v = torch.zeros((t.shape[0], t.shape[1] + pad), dtype=t.dtype, device=DEVICE)[:, :t.shape[1]]
    return v.copy_(t)


def _ids(M, G, order, g):
    """The adapter of every row; about one row or run in eight has none (-1)."""
    def pick(n):
        i = torch.randint(0, G, (n,), generator=g, device=DEVICE)
        none = torch.rand(n, generator=g, device=DEVICE) < 0.125
        return torch.where(none, torch.full_like(i, -1), i).to(torch.int32)
    if order == "mixed":
        return pick(M)
    runs = min(M, 3 * G)
    ends = torch.randint(0, M, (runs - 1,), generator=g, device=DEVICE).sort().values
    return pick(runs)[torch.searchsorted(ends, torch.arange(M, device=DEVICE), right=True)]


def _adapters(st, dtype, g):
    M, K, N, r, G = (st[k] for k in ("M", "K", "N", "r", "G"))
    st.update(A=_randn((G, r, K), dtype, g, K ** -0.5), B=_randn((G, N, r), dtype, g, 0.5 * r ** -0.5),
              alpha=torch.rand(G, generator=g, device=DEVICE) + 0.5, ids=_ids(M, G, st["order"], g))


def prepare(case, seed):
    kind = case["kind"]
    g = _gen(seed)
    st = dict(case)
    if kind in ("norm", "norm_grad"):
        dt, shape = ELEMS[case["dtype"]], (case["rows"], case["cols"])
        st.update(x=_randn(shape, dt, g), w=(1 + 0.1 * torch.randn(shape[1], generator=g, device=DEVICE)).to(dt),
                  res=_randn(shape, dt, g, 2.0) if case["res"] else None)
        if kind == "norm":
            st.update(h=torch.empty_like(st["x"]), y=torch.empty_like(st["x"]))
        else:
            st.update(h=_randn(shape, dt, g, 1.5), dx=torch.empty_like(st["x"]),
                      dw=torch.empty(shape[1], device=DEVICE))
        return st
    if kind == "clip":
        dt, n, size = ELEMS[case["dtype"]], case["tensors"], case["size"]
        # sizes around the mean, as a model's tensors have them
        sizes = [max(1, size * (i % 5 + 1) // 3) for i in range(n)]
        st.update(g=[_randn((m,), dt, g, 0.01) for m in sizes])
        st.update(out=[torch.empty_like(t) for t in st["g"]], norm=torch.empty(2, device=DEVICE))
        return st
    M, K, N = case["M"], case["K"], case["N"]
    if kind == "serve8":
        bf16 = torch.bfloat16
        st.update(x=_randn((M, K), bf16, g), res=_randn((M, K), bf16, g, 2.0),
                  w=(1 + 0.1 * torch.randn(K, generator=g, device=DEVICE)).to(bf16))
        st.update(Wq=torch.randint(-127, 128, (K, N), generator=g, dtype=torch.int8, device=DEVICE),
                  wscale=(torch.rand(N, generator=g, device=DEVICE) + 0.5) * (K ** -0.5 / 73))
        _adapters(st, bf16, g)
        st.update(h=torch.empty_like(st["x"]), y=torch.empty_like(st["x"]),
                  q=torch.empty((M, K), dtype=torch.int8, device=DEVICE),
                  qscale=torch.empty(M, device=DEVICE),
                  Y=torch.empty((M, N), dtype=bf16, device=DEVICE))
        return st
    it, ot = DTYPES[case["dtype"]]
    pad = case.get("pad", 0)
    st.update(X=_padded(_randn((M, K), it, g), pad))
    _adapters(st, it, g)
    if kind == "adapter":
        st.update(W=_padded(_randn((K, N), it, g, K ** -0.5), pad),
                  Y=_padded(torch.zeros((M, N), dtype=ot, device=DEVICE), pad))
    else:
        st.update(Wt=_randn((N, K), it, g, K ** -0.5), dY=_randn((M, N), it, g, 0.1),
                  dX=torch.empty((M, K), dtype=ot, device=DEVICE),
                  dA=torch.empty(st["A"].shape, device=DEVICE),
                  dB=torch.empty(st["B"].shape, device=DEVICE))
    return st


# --------------------------------------------- the operators in elementary operations
def _plain_norm(x, res, w):
    """(x + res, its norm) in binary32."""
    h = x.float() if res is None else x.float() + res.float()
    return h, h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * w.float()


def _select(st):
    """M x G: alpha[g] where the row's adapter is g, else 0."""
    return (st["ids"][:, None] == torch.arange(st["G"], device=DEVICE)) * st["alpha"]


def _wide(A):
    """G x r x K -> (G r) x K in binary32."""
    return A.float().flatten(0, 1)


def _low_rank(X, A, Bt, st):
    """alpha[g] (X A_g^T) B_g^T of every row's adapter: all adapters' products side by
    side, the other adapters' cleared between them.  Bt: (G r) x N."""
    T = (X.float() @ _wide(A).t()).view(st["M"], st["G"], st["r"]) * _select(st)[:, :, None]
    return T.flatten(1) @ Bt


def _plain(st):
    kind = st["kind"]
    if kind == "norm":
        h, y = _plain_norm(st["x"], st["res"], st["w"])
        return {"h": h.to(st["x"].dtype), "y": y.to(st["x"].dtype)}
    if kind == "norm_grad":
        h, dy = st["h"].float(), st["x"].float()
        rstd = torch.rsqrt((h * h).mean(1, keepdim=True) + EPS)
        n, g = h * rstd, dy * st["w"].float()
        dx = rstd * (g - n * (g * n).mean(1, keepdim=True))
        if st["res"] is not None:
            dx = dx + st["res"].float()
        return {"dx": dx.to(st["x"].dtype), "dw": (dy * n).sum(0)}
    if kind == "clip":
        norm = torch.stack([(t.float() * t.float()).sum() for t in st["g"]]).sum().sqrt()
        coef = (MAX_NORM / (norm + 1e-6)).clamp(max=1.0)
        return {"norm": norm, "g": [(t.float() * coef).to(t.dtype) for t in st["g"]]}
    Bt = st["B"].float().transpose(1, 2).flatten(0, 1)     # (G r) x N
    if kind == "adapter":
        Y = st["X"].float() @ st["W"].float() + _low_rank(st["X"], st["A"], Bt, st)
        return Y.to(st["Y"].dtype)
    if kind == "serve8":
        h, y = _plain_norm(st["x"], st["res"], st["w"])
        amax = y.abs().amax(1, keepdim=True)
        q = (y * (127.0 / amax)).round().clamp(-127, 127)
        Y = (q @ st["Wq"].float()) * (amax / 127.0) * st["wscale"]
        Y = Y + _low_rank(y.to(torch.bfloat16), st["A"], Bt, st)
        return {"h": h.to(st["x"].dtype), "Y": Y.to(st["Y"].dtype)}
    M, G, r = st["M"], st["G"], st["r"]
    X, dY, sel = st["X"].float(), st["dY"].float(), _select(st)[:, :, None]
    T = ((X @ _wide(st["A"]).t()).view(M, G, r) * sel).flatten(1)
    dT = ((dY @ Bt.t()).view(M, G, r) * sel).flatten(1)
    dX = dY @ st["Wt"].float() + dT @ _wide(st["A"])
    return {"dX": dX.to(st["dX"].dtype), "dA": (dT.t() @ X).view(st["A"].shape),
            "dB": (T.t() @ dY).view(G, r, -1).transpose(1, 2).contiguous()}


# ------------------------------------------------------------ the library's calls
def _work(st, tcu):
    """The calls' scratch, kept with the state as a program keeps it."""
    if "work" not in st:
        kind = st["kind"]
        if kind == "norm_grad":
            n = tcu.tcu_rms_norm_grad_work(st["rows"], st["cols"])
        elif kind == "clip":
            n = tcu.tcu_clip_grads_work()
        else:
            n = tcu.tcu_adapter_work(st["M"], st["K"], st["N"], st["r"], st["G"])
        st["work"] = torch.empty(n, dtype=torch.uint8, device=DEVICE)
    return st["work"]


def _own(st):
    from paper_1908_06649_amd import tcu
    kind = st["kind"]
    if kind == "norm":
        rows, cols = st["rows"], st["cols"]
        tcu.tcu_rms_norm(st["x"], cols, st["res"], cols, st["w"], st["h"], cols, st["y"], cols,
                         None, 0, None, rows, cols, EPS)
        return {"h": st["h"], "y": st["y"]}
    if kind == "norm_grad":
        rows, cols = st["rows"], st["cols"]
        tcu.tcu_rms_norm_grad(st["x"], cols, st["h"], cols, st["w"], st["res"], cols, st["dx"],
                              cols, st["dw"], _work(st, tcu), rows, cols, EPS)
        return {"dx": st["dx"], "dw": st["dw"]}
    if kind == "clip":
        tcu.tcu_clip_grads(st["g"], st["out"], MAX_NORM, st["norm"], _work(st, tcu))
        return {"norm": st["norm"][0], "g": st["out"]}
    M, K, N, r, G = (st[k] for k in ("M", "K", "N", "r", "G"))
    if kind == "adapter":
        pad = st["pad"]
        tcu.tcu_adapter_gemm(st["X"], K + pad, st["W"], N + pad, st["A"], st["B"], st["alpha"],
                             st["ids"], st["Y"], N + pad, _work(st, tcu), M, K, N, r, G)
        return st["Y"]
    if kind == "serve8":
        tcu.tcu_rms_norm(st["x"], K, st["res"], K, st["w"], st["h"], K, st["y"], K, st["q"], K,
                         st["qscale"], M, K, EPS)
        tcu.tcu_adapter_gemm_q8(st["q"], K, st["qscale"], st["Wq"], N, st["wscale"], st["y"], K,
                                st["A"], st["B"], st["alpha"], st["ids"], st["Y"], N,
                                _work(st, tcu), M, K, N, r, G)
        return {"h": st["h"], "Y": st["Y"]}
    tcu.tcu_adapter_grad(st["X"], K, st["dY"], N, st["A"], st["B"], st["alpha"], st["ids"],
                         st["dA"], st["dB"], _work(st, tcu), M, K, N, r, G)
    tcu.tcu_adapter_input_grad(st["dY"], N, st["Wt"], K, st["A"], st["B"], st["alpha"], st["ids"],
                               st["dX"], K, _work(st, tcu), M, K, N, r, G)
    return {"dX": st["dX"], "dA": st["dA"], "dB": st["dB"]}


def run(st):
    return _own(st) if own else _plain(st)


# ------------------------------------------------- what a pass cannot avoid
def work(case):
    kind = case["kind"]
    if kind in ("norm", "norm_grad"):
        es, n = ELEMS[case["dtype"]].itemsize, case["rows"] * case["cols"]
        if kind == "norm":      # x, the residual and w in; h and y out
            return {"bytes": es * (n * (4 if case["res"] else 3) + case["cols"]), "flops": 6.0 * n}
        return {"bytes": es * (n * (4 if case["res"] else 3) + case["cols"]) + 4 * case["cols"],
                "flops": 12.0 * n}
    if kind == "clip":
        n = sum(max(1, case["size"] * (i % 5 + 1) // 3) for i in range(case["tensors"]))
        return {"bytes": 2 * ELEMS[case["dtype"]].itemsize * n, "flops": 3.0 * n}
    M, K, N, r, G = (case[k] for k in ("M", "K", "N", "r", "G"))
    low = 2.0 * M * r * (K + N)
    factors = min(M, G) * r * (K + N) * 2
    if kind == "serve8":        # x, residual, weights in; h and Y out
        return {"bytes": 3 * 2 * M * K + K * N + 4 * N + factors + 2 * M * N + 4 * M,
                "flops": 2.0 * M * K * N + low}
    it, ot = DTYPES[case["dtype"]]
    if kind == "adapter":
        return {"bytes": it.itemsize * (M * K + K * N) + factors + ot.itemsize * M * N + 4 * M,
                "flops": 2.0 * M * K * N + low}
    return {"bytes": it.itemsize * (M * K + M * N + K * N) + factors + ot.itemsize * M * K
                     + 4 * G * r * (K + N) + 4 * M,
            "flops": 2.0 * M * K * N + 2.5 * low}


# --------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    d = {k: v.double() for k, v in st.items() if torch.is_tensor(v) and v.is_floating_point()}
    if kind == "clip":
        norm = math.sqrt(sum(float(t.double().pow(2).sum()) for t in st["g"]))
        c = min(1.0, MAX_NORM / (norm + 1e-6))
        return {"norm": torch.tensor(norm, dtype=torch.float64, device=DEVICE),
                "g": [c * t.double() for t in st["g"]]}
    if kind == "norm_grad":
        h, dy, w, cols = d["h"], d["x"], d["w"], case["cols"]
        s = (h.pow(2).sum(1) / cols + EPS).sqrt()
        c = torch.linalg.vecdot(dy * w, h) / (cols * s.pow(3))
        dx = dy * w / s[:, None] - h * c[:, None]
        return {"dx": dx + d["res"] if "res" in d else dx, "dw": (dy * (h / s[:, None])).sum(0)}
    if kind in ("norm", "serve8"):
        h = d["x"] + d["res"] if "res" in d else d["x"]
        y = d["w"] * h / (h.pow(2).sum(1) / h.shape[1] + EPS).sqrt()[:, None]
        if kind == "norm":
            return {"h": h, "y": y}
        amax = y.abs().max(1).values
        q = torch.round(127 * y / amax[:, None])
        Y = (q @ st["Wq"].double()) * torch.outer(amax / 127, d["wscale"])
        X = y.to(torch.bfloat16).double()
    else:
        X = d["X"]
        Y = X @ d["W"] if kind == "adapter" else d["dY"] @ d["Wt"]
    dA, dB = torch.zeros_like(d["A"]), torch.zeros_like(d["B"])
    for g, a in enumerate(d["alpha"].tolist()):
        rows = (st["ids"] == g).nonzero()[:, 0]
        A, B = d["A"][g], d["B"][g]
        if kind == "adapter_grad":
            x, dy = X[rows], d["dY"][rows]
            dT = a * (dy @ B)
            Y[rows] += dT @ A
            dA[g], dB[g] = dT.t() @ x, dy.t() @ (a * (x @ A.t()))
        else:
            Y[rows] += a * ((X[rows] @ A.t()) @ B.t())
    if kind == "adapter_grad":
        return {"dX": Y, "dA": dA, "dB": dB}
    return {"h": h, "Y": Y} if kind == "serve8" else Y

"""The operators of a projection in 4 bits and of what follows it in an attention
layer that the library is timed on, from single tokens to the largest batches.

A case is a dict of plain values; ``kind`` names what one pass computes:

    mx_weight   tcu_mx4_quant both ways,      rows, cols, dtype
                tcu_mx4_dequant of each
    mx_linear   tcu_mx4_linear                M, K, N, dtype, pad
    mx_train    tcu_mx4_quant of X, W and dY  M, K, N, dtype
                both ways, then tcu_mx4_gemm
                for Y, dX and dW
    heads       tcu_qk_norm                   tokens, hq, hk, dim, rot, adjacent, dtype, order
    heads_grad  tcu_qk_norm_grad              the same

M rows are tokens; K and N a layer's inputs and outputs; hq and hk the heads of
queries and keys, dim their elements, rot how many of them are rotated, in pairs
that are adjacent or half of rot apart.  Queries and keys are views of packed rows
that hold the values too; the rotated ones lie token by token ("tokens") or head by
head ("heads").  ``own`` chooses between the library's calls and the same operators
in elementary torch operations.
"""
import math

import torch

own = False

DEVICE = "cuda"
EPS = 1e-6
BASE = 10000.0
# dtype name -> (input type, output type) of the projections
DTYPES = {"f16": (torch.float16, torch.float32), "bf16": (torch.bfloat16, torch.float32),
          "f16out": (torch.float16, torch.float16), "bf16out": (torch.bfloat16, torch.bfloat16)}
ELEMS = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# the magnitudes that a 4-bit code's low three bits stand for
MAGNITUDES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # Queries and keys of one generated token.
        dict(name="heads_bf16_1x32x8x128", kind="heads", tokens=1, hq=32, hk=8, dim=128, rot=128,
             adjacent=False, dtype="bf16", order="tokens"),
        # Prompts with odd lengths; heads of no power of two, half of each rotated, pairs adjacent.
        dict(name="heads_f16_1003x15x5x80", kind="heads", tokens=1003, hq=15, hk=5, dim=80, rot=40,
             adjacent=True, dtype="f16", order="heads"),
        # A large batch of prompts: memory bandwidth.
        dict(name="heads_bf16_16384x64x8x128", kind="heads", tokens=16384, hq=64, hk=8, dim=128,
             rot=128, adjacent=False, dtype="bf16", order="heads"),
        # The gradient of a short batch in binary32.
        dict(name="heads_grad_f32_517x7x1x64", kind="heads_grad", tokens=517, hq=7, hk=1, dim=64,
             rot=64, adjacent=False, dtype="f32", order="tokens"),
        # The gradient in training.
        dict(name="heads_grad_bf16_8192x32x8x128", kind="heads_grad", tokens=8192, hq=32, hk=8,
             dim=128, rot=128, adjacent=False, dtype="bf16", order="heads"),
        # A small odd weight brought to 4 bits, both ways it is contracted in training.
        dict(name="mx_weight_f16_1003x2005", kind="mx_weight", rows=1003, cols=2005, dtype="f16"),
        # A large one.
        dict(name="mx_weight_bf16_8192x8192", kind="mx_weight", rows=8192, cols=8192, dtype="bf16"),
        # One token through a layer: latency and the weight's bytes.
        dict(name="mx_linear_bf16_1x4096x4096", kind="mx_linear", M=1, K=4096, N=4096,
             dtype="bf16out", pad=0),
        # A token of each of 16 requests.
        dict(name="mx_linear_bf16_16x8192x8192", kind="mx_linear", M=16, K=8192, N=8192,
             dtype="bf16out", pad=0),
        # Sizes as data has them, rows at any 2-byte address.
        dict(name="mx_linear_f16_1000x1003x2005", kind="mx_linear", M=1000, K=1003, N=2005,
             dtype="f16", pad=0),
        # The largest projection of prompts.
        dict(name="mx_linear_bf16_8192x8192x8192", kind="mx_linear", M=8192, K=8192, N=8192,
             dtype="bf16out", pad=0),
        # Forward and both gradients of a layer trained in 4 bits.
        dict(name="mx_train_bf16_8192x4096x4096", kind="mx_train", M=8192, K=4096, N=4096,
             dtype="bf16out"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _any_or_round(rng, v, unit):
    """v as it is, or as a multiple of `unit`: programs pass both."""
    return max(unit, v // unit * unit) if rng.random() < 0.6 else v


def draw(rng):
    kind = rng.choice(["heads", "heads", "heads_grad", "mx_weight", "mx_linear", "mx_linear",
                       "mx_train"])
    if kind.startswith("heads"):
        dim = rng.choice([32, 64, 64, 80, 96, 100, 128, 128, 128, 192, 256])
        hk = rng.choice([1, 2, 4, 5, 8, 16])
        hq = hk * rng.choice([1, 1, 2, 3, 4, 8])
        tokens = _log_int(rng, 1, min(32768, (1 << 27) // ((hq + hk) * dim)))
        return dict(kind=kind, tokens=tokens, hq=hq, hk=hk, dim=dim,
                    rot=rng.choice([dim, dim, dim, dim // 4 * 2]), adjacent=rng.random() < 0.4,
                    dtype=rng.choice(["bf16", "bf16", "f16", "f32"]),
                    order=rng.choice(["tokens", "heads"]))
    if kind == "mx_weight":
        rows = _any_or_round(rng, _log_int(rng, 32, 16384), 32)
        cols = _any_or_round(rng, _log_int(rng, 32, min(16384, (1 << 26) // rows)), 32)
        return dict(kind=kind, rows=rows, cols=cols, dtype=rng.choice(list(ELEMS)))
    K = _any_or_round(rng, _log_int(rng, 64, 8192), 64)
    N = _any_or_round(rng, _log_int(rng, 64, 8192), 64)
    if kind == "mx_train":
        M = _any_or_round(rng, _log_int(rng, 32, 8192), 32)
        M = min(M, max(32, (1 << 37) // (K * N)))
        return dict(kind=kind, M=M, K=K, N=N, dtype=rng.choice(list(DTYPES)))
    M = _log_int(rng, 1, 128) if rng.random() < 0.5 else _log_int(rng, 128, 8192)
    return dict(kind=kind, M=M, K=K, N=N, dtype=rng.choice(list(DTYPES)),
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


def _activations(shape, dtype, g):
    """Rows of different size, and a few columns much larger than the others."""
    x = torch.randn(shape, generator=g, device=DEVICE)
    x *= torch.exp(0.5 * torch.randn((shape[0], 1), generator=g, device=DEVICE))
    x *= torch.where(torch.rand(shape[1], generator=g, device=DEVICE) < 0.01, 12.0, 1.0)
    return x.to(dtype)


def _groups(n):
    return (n + 127) // 128


def _pack(W):
    """W's rows in 4 bits as a program holds them: codes (two to a byte, whole groups of
    128) and scale words (group by group, a word of four scales for every row)."""
    rows, cols = W.shape
    G = _groups(cols)
    v = torch.zeros((rows, G * 128), device=DEVICE)
    v[:, :cols] = W.float()
    e = _block_exponent(v.view(rows, G * 4, 32))
    v = _rounded(v).view(rows, G * 4, 32) * torch.exp2(-e)
    code = torch.bucketize(v.abs(), torch.tensor(MAGNITUDES, device=DEVICE)).to(torch.uint8)
    code += torch.where(v < 0, 8, 0).to(torch.uint8)
    code = code.view(rows, G * 64, 2)
    scale = (e + 127).to(torch.uint8).view(rows, G * 4)
    return ((code[..., 0] | (code[..., 1] << 4)).contiguous(),
            scale.view(torch.int32).t().contiguous())


def prepare(case, seed):
    kind = case["kind"]
    g = _gen(seed)
    st = dict(case)
    if kind.startswith("heads"):
        dt, T, dim = ELEMS[case["dtype"]], case["tokens"], case["dim"]
        hq, hk, rot = case["hq"], case["hk"], case["rot"]
        qkv = _randn((T, hq + 2 * hk, dim), dt, g, 2.0)
        st.update(q=qkv[:, :hq], k=qkv[:, hq:hq + hk])
        for n in ("wq", "wk"):
            st[n] = (1 + 0.1 * torch.randn(dim, generator=g, device=DEVICE)).to(dt)
        i = torch.arange(0, rot, 2, dtype=torch.float64, device=DEVICE)
        st["freq"] = (BASE ** (-i / rot)).float()
        # sequences of different lengths one after the other, some continued at far positions
        n = min(T, 5)
        starts = torch.randint(0, T, (n,), generator=g, device=DEVICE).sort().values
        starts[0] = 0
        at = torch.arange(T, device=DEVICE)
        seq = torch.searchsorted(starts, at, right=True) - 1
        first = torch.randint(0, 120000, (n,), generator=g, device=DEVICE) * \
            torch.randint(0, 2, (n,), generator=g, device=DEVICE)
        st["pos"] = (at - starts[seq] + first[seq]).to(torch.int32)
        like = {n: torch.empty((h, T, dim) if case["order"] == "heads" else (T, h, dim), dtype=dt,
                               device=DEVICE) for n, h in (("yq", hq), ("yk", hk))}
        if case["order"] == "heads":
            like = {n: t.transpose(0, 1) for n, t in like.items()}
        if kind == "heads":
            st.update(like)
            return st
        for n, t in like.items():
            st["d" + n] = t.copy_(torch.randn(t.shape, generator=g, device=DEVICE))
        d = torch.zeros_like(qkv)
        st.update(dq=d[:, :hq], dk=d[:, hq:hq + hk], dwq=torch.empty(dim, device=DEVICE),
                  dwk=torch.empty(dim, device=DEVICE))
        return st
    if kind == "mx_weight":
        dt, rows, cols = ELEMS[case["dtype"]], case["rows"], case["cols"]
        st.update(x=_randn((rows, cols), dt, g, cols ** -0.5),
                  y=torch.empty((rows, cols), dtype=dt, device=DEVICE),
                  yt=torch.empty((cols, rows), dtype=dt, device=DEVICE))
        return st
    M, K, N = case["M"], case["K"], case["N"]
    it, ot = DTYPES[case["dtype"]]
    if kind == "mx_linear":
        Wq, wscale = _pack(_randn((N, K), it, g, K ** -0.5))
        st.update(X=_padded(_activations((M, K), it, g), case["pad"]), Wq=Wq, wscale=wscale,
                  Y=torch.empty((M, N), dtype=ot, device=DEVICE))
        return st
    st.update(X=_activations((M, K), it, g), W=_randn((N, K), it, g, K ** -0.5),
              dY=_randn((M, N), it, g, 0.01), Y=torch.empty((M, N), dtype=ot, device=DEVICE),
              dX=torch.empty((M, K), dtype=ot, device=DEVICE),
              dW=torch.empty((N, K), device=DEVICE))
    return st


# --------------------------------------------- the operators in elementary operations
def _block_exponent(v):
    """The exponent of the scale of every block (the last dimension) of v."""
    amax = v.abs().amax(-1, keepdim=True)
    return torch.where(amax > 0, torch.frexp(amax).exponent - 3.0, -127.0).clamp(min=-127.0)


def _rounded(x):
    """The values in binary32 that x's rows stand for in 4 bits, in blocks of 32."""
    rows, cols = x.shape
    n = (cols + 31) // 32 * 32
    v = torch.nn.functional.pad(x.float(), (0, n - cols)).view(rows, n // 32, 32)
    e = _block_exponent(v)
    v = v * torch.exp2(-e)
    # steps of a half below 2, of one to 4, of two above
    step = torch.exp2((torch.frexp(v).exponent - 2.0).clamp(-1.0, 1.0))
    v = (torch.round(v / step) * step).clamp(-6.0, 6.0) * torch.exp2(e)
    return v.view(rows, n)[:, :cols]


def _decoded(q, words, cols):
    """The values in binary32 of codes and scale words."""
    table = torch.tensor(MAGNITUDES + tuple(-m for m in MAGNITUDES), device=DEVICE)
    v = table[torch.stack((q & 15, q >> 4), 2).int()].view(q.shape[0], -1, 32)
    e = (words.t()[:, :, None] >> torch.tensor([0, 8, 16, 24], device=DEVICE)) & 255
    e = e.flatten(1).float() - 127.0
    return (v * torch.exp2(e)[:, :, None]).flatten(1)[:, :cols]


def _tables(st):
    """cos and sin of every token's angles in binary32, from binary64."""
    a = st["pos"].double()[:, None] * st["freq"].double()
    return a.cos().float()[:, None], a.sin().float()[:, None]


def _pairs(x, st):
    """The rotated pairs' first and second elements, and the rest."""
    rot = st["rot"]
    if st["adjacent"]:
        return x[..., 0:rot:2], x[..., 1:rot:2], x[..., rot:]
    return x[..., :rot // 2], x[..., rot // 2:rot], x[..., rot:]


def _join(a, b, rest, st):
    ab = torch.stack((a, b), -1).flatten(-2) if st["adjacent"] else torch.cat((a, b), -1)
    return torch.cat((ab, rest), -1)


def _plain_heads(x, w, cs, st):
    x = x.float()
    n = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * w.float()
    a, b, rest = _pairs(n, st)
    return _join(a * cs[0] - b * cs[1], a * cs[1] + b * cs[0], rest, st)


def _plain_heads_grad(dy, x, w, cs, st):
    x = x.float()
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * rstd
    a, b, rest = _pairs(dy.float(), st)
    dv = _join(a * cs[0] + b * cs[1], b * cs[0] - a * cs[1], rest, st)
    g = dv * w.float()
    return rstd * (g - n * (g * n).mean(-1, keepdim=True)), (dv * n).sum((0, 1))


def _plain(st):
    kind = st["kind"]
    if kind == "heads":
        cs = _tables(st)
        return {n: _plain_heads(st[x], st[w], cs, st).to(st[n].dtype)
                for n, x, w in (("yq", "q", "wq"), ("yk", "k", "wk"))}
    if kind == "heads_grad":
        cs = _tables(st)
        dq, dwq = _plain_heads_grad(st["dyq"], st["q"], st["wq"], cs, st)
        dk, dwk = _plain_heads_grad(st["dyk"], st["k"], st["wk"], cs, st)
        return {"dq": dq.to(st["dq"].dtype), "dk": dk.to(st["dk"].dtype), "dwq": dwq, "dwk": dwk}
    if kind == "mx_weight":
        return {"y": _rounded(st["x"]).to(st["y"].dtype),
                "yt": _rounded(st["x"].t()).to(st["y"].dtype)}
    if kind == "mx_linear":
        W = _decoded(st["Wq"], st["wscale"], st["K"])
        return (_rounded(st["X"]) @ W.t()).to(st["Y"].dtype)
    X, W, dY = st["X"], st["W"], st["dY"]
    return {"Y": (_rounded(X) @ _rounded(W).t()).to(st["Y"].dtype),
            "dX": (_rounded(dY) @ _rounded(W.t()).t()).to(st["dX"].dtype),
            "dW": _rounded(dY.t()) @ _rounded(X.t()).t()}


# ------------------------------------------------------------ the library's calls
def _codes(st, tcu, name, rows, cols):
    """Room for a matrix in 4 bits, kept with the state as a program keeps it."""
    if name not in st:
        st[name] = (torch.empty((rows, tcu.tcu_mx4_row_bytes(cols)), dtype=torch.uint8,
                                device=DEVICE),
                    torch.empty((tcu.tcu_mx4_row_words(cols), rows), dtype=torch.int32,
                                device=DEVICE))
    return st[name]


def _quant(st, tcu, name, rows, cols):
    """st[name] in 4 bits along its rows and along its columns."""
    q, s = _codes(st, tcu, name + "4", rows, cols)
    qt, ts = _codes(st, tcu, name + "t4", cols, rows)
    tcu.tcu_mx4_quant(st[name], cols, q, q.shape[1], s, rows, qt, qt.shape[1], ts, cols, rows,
                      cols)
    return q, s, qt, ts


def _product(tcu, st, A, a, B, b, C, M, K, N):
    """C (M x N) = A B^T of matrices in 4 bits."""
    n = tcu.tcu_mx4_work(M, K, N)
    if "work" not in st or st["work"].numel() < n:
        st["work"] = torch.empty(n, dtype=torch.uint8, device=DEVICE)
    tcu.tcu_mx4_gemm(A, A.shape[1], a, M, B, B.shape[1], b, N, C, N, st["work"], M, K, N, 0)


def _own(st):
    from paper_1908_06649_amd import tcu
    kind = st["kind"]
    if kind.startswith("heads"):
        T, hq, hk, dim, rot = (st[k] for k in ("tokens", "hq", "hk", "dim", "rot"))
        flags = tcu.TCU_ROPE_ADJACENT if st["adjacent"] else 0
        if kind == "heads":
            tcu.tcu_qk_norm(st["q"], st["k"], st["wq"], st["wk"], st["freq"], st["pos"], st["yq"],
                            st["yk"], T, hq, hk, dim, rot, EPS, flags)
            return {"yq": st["yq"], "yk": st["yk"]}
        if "work" not in st:
            st["work"] = torch.empty(tcu.tcu_qk_norm_grad_work(T, hq, hk, dim), dtype=torch.uint8,
                                     device=DEVICE)
        tcu.tcu_qk_norm_grad(st["dyq"], st["dyk"], st["q"], st["k"], st["wq"], st["wk"],
                             st["freq"], st["pos"], st["dq"], st["dk"], st["dwq"], st["dwk"],
                             st["work"], T, hq, hk, dim, rot, EPS, flags)
        return {n: st[n] for n in ("dq", "dk", "dwq", "dwk")}
    if kind == "mx_weight":
        rows, cols = st["rows"], st["cols"]
        q, s, qt, ts = _quant(st, tcu, "x", rows, cols)
        tcu.tcu_mx4_dequant(q, q.shape[1], s, rows, st["y"], cols, rows, cols)
        tcu.tcu_mx4_dequant(qt, qt.shape[1], ts, cols, st["yt"], rows, cols, rows)
        return {"y": st["y"], "yt": st["yt"]}
    M, K, N = (st[k] for k in ("M", "K", "N"))
    if kind == "mx_linear":
        if "work" not in st:
            st["work"] = torch.empty(tcu.tcu_mx4_work(M, K, N), dtype=torch.uint8, device=DEVICE)
        tcu.tcu_mx4_linear(st["X"], K + st["pad"], st["Wq"], st["Wq"].shape[1], st["wscale"], N,
                           st["Y"], N, st["work"], M, K, N, 0)
        return st["Y"]
    X, x, Xt, xt = _quant(st, tcu, "X", M, K)
    W, w, Wt, wt = _quant(st, tcu, "W", N, K)
    D, d, Dt, dt = _quant(st, tcu, "dY", M, N)
    _product(tcu, st, X, x, W, w, st["Y"], M, K, N)
    _product(tcu, st, D, d, Wt, wt, st["dX"], M, N, K)
    _product(tcu, st, Dt, dt, Xt, xt, st["dW"], N, M, K)
    return {"Y": st["Y"], "dX": st["dX"], "dW": st["dW"]}


def run(st):
    return _own(st) if own else _plain(st)


# ------------------------------------------------- what a pass cannot avoid
def work(case):
    kind = case["kind"]
    if kind.startswith("heads"):
        n = case["tokens"] * (case["hq"] + case["hk"]) * case["dim"]
        es, small = ELEMS[case["dtype"]].itemsize, 4 * case["tokens"] + 2 * case["rot"]
        if kind == "heads":     # x in, y out, both weights
            return {"bytes": es * (2 * n + 2 * case["dim"]) + small, "flops": 8.0 * n}
        return {"bytes": es * (3 * n + 2 * case["dim"]) + 8 * case["dim"] + small,
                "flops": 16.0 * n}
    if kind == "mx_weight":     # x in; both 4-bit forms and the values they stand for out
        n = case["rows"] * case["cols"]
        return {"bytes": 3 * ELEMS[case["dtype"]].itemsize * n + 2 * (n // 2 + n // 32),
                "flops": 8.0 * n}
    M, K, N = (case[k] for k in ("M", "K", "N"))
    it, ot = DTYPES[case["dtype"]]
    if kind == "mx_linear":
        return {"bytes": it.itemsize * M * K + N * K // 2 + N * K // 32 + ot.itemsize * M * N,
                "flops": 2.0 * M * K * N}
    return {"bytes": it.itemsize * (M * K + N * K + M * N) + ot.itemsize * M * (K + N) + 4 * N * K,
            "flops": 6.0 * M * K * N}


# --------------------------------------------------------- the same in 64 bits
def _four_bits64(x):
    """x's values in 4 bits along its rows, found by comparison with all magnitudes' borders."""
    rows, cols = x.shape
    out = torch.zeros((rows, -(-cols // 32) * 32), dtype=torch.float64, device=DEVICE)
    out[:, :cols] = x.double()
    out = out.view(rows, -1, 32)
    amax = out.abs().amax(2, keepdim=True)
    # exact: log2 of a power of two is, and no other input is so near one
    power = torch.floor(torch.log2(amax.clamp(min=2.0 ** -125)))
    scale = torch.exp2((power - 2).clamp(min=-127))
    v = out / scale
    m = v.abs()
    mag = torch.zeros_like(m)
    # a half-way value goes to the magnitude whose code is even
    for i in range(1, 8):
        mid = (MAGNITUDES[i - 1] + MAGNITUDES[i]) / 2
        mag = torch.where((m >= mid) if i % 2 == 0 else (m > mid), MAGNITUDES[i], mag)
    return (torch.copysign(mag, v) * scale).flatten(1)[:, :cols]


def _held64(q, words, cols):
    rows = q.shape[0]
    mags = torch.tensor(MAGNITUDES, dtype=torch.float64, device=DEVICE)
    out = torch.empty((rows, q.shape[1] * 2), dtype=torch.float64, device=DEVICE)
    for half, shift in ((0, 0), (1, 4)):
        c = (q >> shift).long() & 15
        out[:, half::2] = torch.where(c > 7, -1.0, 1.0) * mags[c & 7]
    for byte in range(4):
        s = (words >> (8 * byte)) & 255
        out.view(rows, -1, 4, 32)[:, :, byte] *= torch.exp2(s.t().double() - 127)[:, :, None]
    return out[:, :cols]


def _turned64(x, angle, st):
    """x's rotated elements as complex numbers, turned by the angle."""
    rot = st["rot"]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]
    out = x.clone()
    if st["adjacent"]:
        z = torch.complex(x[..., 0:rot:2], x[..., 1:rot:2]) * turn
        out[..., 0:rot:2], out[..., 1:rot:2] = z.real, z.imag
    else:
        z = torch.complex(x[..., :rot // 2], x[..., rot // 2:rot]) * turn
        out[..., :rot // 2], out[..., rot // 2:rot] = z.real, z.imag
    return out


def exact(case, seed):
    kind = case["kind"]
    st = prepare(case, seed)
    if kind.startswith("heads"):
        angle = torch.outer(st["pos"].double(), st["freq"].double())
        out = {}
        for x, w in (("q", "wq"), ("k", "wk")):
            h, weight = st[x].double(), st[w].double()
            s = (h.pow(2).sum(-1, keepdim=True) / case["dim"] + EPS).sqrt()
            if kind == "heads":
                out["y" + x] = _turned64(weight * h / s, angle, st)
            else:
                dv = _turned64(st["dy" + x].double(), -angle, st)
                c = (dv * weight * h).sum(-1, keepdim=True) / (case["dim"] * s.pow(3))
                out["d" + x] = dv * weight / s - h * c
                out["dw" + x] = (dv * h / s).flatten(0, 1).sum(0)
        names = ("yq", "yk") if kind == "heads" else ("dq", "dk", "dwq", "dwk")
        return {n: out[n] for n in names}
    if kind == "mx_weight":
        return {"y": _four_bits64(st["x"]), "yt": _four_bits64(st["x"].t())}
    if kind == "mx_linear":
        return _four_bits64(st["X"]) @ _held64(st["Wq"], st["wscale"], case["K"]).t()
    X, W, dY = st["X"], st["W"], st["dY"]
    return {"Y": _four_bits64(X) @ _four_bits64(W).t(),
            "dX": _four_bits64(dY) @ _four_bits64(W.t()).t(),
            "dW": _four_bits64(dY.t()) @ _four_bits64(X.t()).t()}

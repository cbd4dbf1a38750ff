"""Plain implementations in binary64 of the operators around a layer's products,
and seeded inputs for their tests."""
import torch

DEV = "cuda"
# unit roundoff of a stored type; binary32 results are bounded by their sums alone
ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 0.0}
F32 = 2.0 ** -24


def gen(seed):
    return torch.Generator().manual_seed(seed)


def randn(shape, dtype, g, scale=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float64) * scale).to(dtype)


def pitched(t, ld, fill=float("nan")):
    """A device copy of a 2-D tensor with row pitch ld, the rest of the rows filled."""
    rows, cols = t.shape
    buf = torch.empty(max(rows, 1) * ld + 64, dtype=t.dtype, device=DEV)
    buf.fill_(fill if t.is_floating_point() else 113)
    v = buf[:max(rows, 1) * ld].view(max(rows, 1), ld)[:rows, :cols]
    v.copy_(t)
    return buf, v


def untouched(buf, rows, cols, ld, fill=float("nan")):
    """Whether everything of a pitched buffer outside its rows is as filled."""
    keep = torch.ones(buf.numel(), dtype=torch.bool, device=buf.device)
    keep[:max(rows, 1) * ld].view(max(rows, 1), ld)[:rows, :cols] = False
    rest = buf[keep]
    return bool(torch.isnan(rest).all()) if buf.is_floating_point() else bool((rest == 113).all())


def within(got, want, bound):
    """Every element within its bound; places that are not finite agree."""
    got = got.detach().cpu().double()
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "NaN in other places"
    odd = ~fine & ~torch.isnan(want)
    assert torch.equal(got[odd], want[odd]), "infinities differ"
    excess = ((got - want).abs() - bound)[fine]
    assert excess.numel() == 0 or float(excess.max()) <= 0, \
        f"off by {float((got - want).abs()[fine].max())}, over the bound by {float(excess.max())}"


# ------------------------------------------------------------------ norm
def norm64(x, res, w, eps):
    h = x.double() if res is None else x.double() + res.double()
    return h, h / (h.pow(2).mean(1, keepdim=True) + eps).sqrt() * w.double()


def norm_grad64(dy, h, w, dh, eps):
    h, dy = h.double(), dy.double()
    rstd = (h.pow(2).mean(1, keepdim=True) + eps).rsqrt()
    g = dy * w.double()
    dx = rstd * (g - h * rstd.pow(2) * (g * h).mean(1, keepdim=True))
    mag = rstd * (g.abs() + h.abs() * rstd.pow(2) * (g * h).abs().mean(1, keepdim=True))
    if dh is not None:
        dx, mag = dx + dh.double(), mag + dh.double().abs()
    return dx, (dy * h * rstd).sum(0), mag, (dy * h * rstd).abs().sum(0)


# -------------------------------------------------------------- adapters
class Layer:
    """Seeded operands of an adapted projection on the host."""

    def __init__(self, M, K, N, r, G, dtype, seed, ids=None):
        g = gen(seed)
        self.M, self.K, self.N, self.r, self.G = M, K, N, r, G
        self.X = randn((M, K), dtype, g)
        self.W = randn((K, N), dtype, g, max(K, 1) ** -0.5)
        self.A = randn((G, r, K), dtype, g, max(K, 1) ** -0.5)
        self.B = randn((G, N, r), dtype, g, r ** -0.5)
        self.alpha = torch.rand(G, generator=g) + 0.5
        self.dY = randn((M, N), dtype, g)
        if ids is None:
            ids = torch.randint(-1, G + 1, (M,), generator=g) if G else torch.zeros(M)
        self.ids = ids.to(torch.int32)

    def rows(self, g):
        return (self.ids == g).nonzero()[:, 0]

    def adapters64(self, X=None):
        """(low-rank part, the sum of its terms' magnitudes)."""
        X = self.X if X is None else X
        y = torch.zeros(self.M, self.N, dtype=torch.float64)
        mag = torch.zeros_like(y)
        for g in range(self.G):
            at, a = self.rows(g), float(self.alpha[g])
            A, B, x = self.A[g].double(), self.B[g].double(), X[at].double()
            y[at] = a * ((x @ A.t()) @ B.t())
            mag[at] = a * ((x.abs() @ A.abs().t()) @ B.abs().t())
        return y, mag

    def forward64(self):
        """(Y, bound of a binary32 evaluation before the last rounding)."""
        x, w = self.X.double(), self.W.double()
        low, mag = self.adapters64()
        # sums of K (and r) binary32 terms; T enters with at least 16 bits
        return x @ w + low, (self.K + 8) * F32 * (x.abs() @ w.abs()) + \
            ((self.K + self.r + 8) * F32 + 2.0 ** -16) * mag

    def input_grad64(self):
        dy, w = self.dY.double(), self.W.double().t()
        y, mag = dy @ w, dy.abs() @ w.abs() * (self.N + 8) * F32
        for g in range(self.G):
            at, a = self.rows(g), float(self.alpha[g])
            A, B = self.A[g].double(), self.B[g].double()
            y[at] += a * ((dy[at] @ B) @ A)
            mag[at] += a * ((dy[at].abs() @ B.abs()) @ A.abs()) * \
                ((self.N + self.r + 8) * F32 + 2.0 ** -16)
        return y, mag

    def grads64(self):
        """dA, dB and their bounds."""
        dA = torch.zeros(self.G, self.r, self.K, dtype=torch.float64)
        dB = torch.zeros(self.G, self.N, self.r, dtype=torch.float64)
        eA, eB = torch.zeros_like(dA), torch.zeros_like(dB)
        for g in range(self.G):
            at, a = self.rows(g), float(self.alpha[g])
            A, B = self.A[g].double(), self.B[g].double()
            x, dy = self.X[at].double(), self.dY[at].double()
            dA[g] = a * (dy @ B).t() @ x
            dB[g] = a * dy.t() @ (x @ A.t())
            n = len(at) + 8
            eA[g] = a * (dy.abs() @ B.abs()).t() @ x.abs() * (self.N + n) * F32
            eB[g] = a * dy.abs().t() @ (x.abs() @ A.abs().t()) * (self.K + n) * F32
        return dA, dB, eA, eB

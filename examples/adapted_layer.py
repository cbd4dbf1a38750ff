"""A projection with low-rank adapters, trained and served with the library's calls.

Training: several adapters at once, each on its own sequences of one batch, beside a
frozen weight: the norm with the residual's addition, the projection with every
row's adapter, the gradients of the adapters, of the input and of the norm, clipping
by their common norm, and a plain gradient step.  The targets come from other
adapters, so the loss falls as these are found.

Serving: single tokens of many requests, each with its adapter, on the weight in 8
bits: the norm writes the 8-bit operand and its scales beside the bfloat16 rows that
the adapters read.

    python examples/adapted_layer.py [--steps 60]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1908_06649_amd import tcu  # noqa: E402

EPS = 1e-5
BF16 = torch.bfloat16


class Layer:
    """Frozen weight, norm weight and G adapters of rank r, with the buffers of
    batches of up to `rows` rows."""

    def __init__(self, K, N, r, G, rows, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)

        def randn(*shape, scale=1.0):
            return torch.randn(shape, generator=g, device=device) * scale

        self.K, self.N, self.r, self.G, self.device = K, N, r, G, device
        self.W = randn(K, N, scale=K ** -0.5).to(BF16)
        self.Wt = self.W.t().contiguous()            # for the input's gradient
        self.wscale = self.W.float().abs().amax(0) / 127
        self.Wq = (self.W.float() / self.wscale).round().to(torch.int8)
        self.norm = torch.ones(K, device=device)
        self.A = randn(G, r, K, scale=K ** -0.5)     # binary32 masters of the factors
        self.B = torch.zeros(G, N, r, device=device)
        self.alpha = torch.full((G,), 2.0, device=device)
        work = max(tcu.tcu_adapter_work(rows, K, N, r, G), tcu.tcu_rms_norm_grad_work(rows, K),
                   tcu.tcu_clip_grads_work())
        self.work = torch.empty(work, dtype=torch.uint8, device=device)

    def forward(self, x, res, ids):
        """(h, y, Y): the residual stream, its norm, the projection."""
        M, K, N, dev = x.shape[0], self.K, self.N, self.device
        h, y = torch.empty_like(x), torch.empty_like(x)
        tcu.tcu_rms_norm(x, K, res, K, self.norm.to(BF16), h, K, y, K, None, 0, None, M, K, EPS)
        Y = torch.empty(M, N, dtype=BF16, device=dev)
        tcu.tcu_adapter_gemm(y, K, self.W, N, self.A.to(BF16), self.B.to(BF16), self.alpha, ids, Y,
                             N, self.work, M, K, N, self.r, self.G)
        return h, y, Y

    def backward(self, h, y, dY, dh, ids):
        """Gradients (dA, dB, dnorm) and the gradient of x and of the residual."""
        M, K, N, r, G = y.shape[0], self.K, self.N, self.r, self.G
        A, B = self.A.to(BF16), self.B.to(BF16)
        dA, dB = torch.empty_like(self.A), torch.empty_like(self.B)
        tcu.tcu_adapter_grad(y, K, dY, N, A, B, self.alpha, ids, dA, dB, self.work, M, K, N, r, G)
        dy, dx = torch.empty_like(y), torch.empty_like(y)
        tcu.tcu_adapter_input_grad(dY, N, self.Wt, K, A, B, self.alpha, ids, dy, K, self.work, M, K,
                                   N, r, G)
        dnorm = torch.empty_like(self.norm)
        tcu.tcu_rms_norm_grad(dy, K, h, K, self.norm.to(BF16), dh, K, dx, K, dnorm, self.work, M, K,
                              EPS)
        return [dA, dB, dnorm], dx

    def step(self, grads, lr, max_norm):
        """Clip in place, then a gradient step; returns the norm before clipping."""
        result = torch.empty(2, device=self.device)
        tcu.tcu_clip_grads(grads, grads, max_norm, result, self.work)
        for p, g in zip((self.A, self.B, self.norm), grads):
            p.sub_(g, alpha=lr)
        return result[0]

    def decode(self, x, res, ids):
        """(h, Y) of single tokens on the 8-bit weight."""
        M, K, N, dev = x.shape[0], self.K, self.N, self.device
        h, y = torch.empty_like(x), torch.empty_like(x)
        q = torch.empty(M, K, dtype=torch.int8, device=dev)
        scale = torch.empty(M, device=dev)
        tcu.tcu_rms_norm(x, K, res, K, self.norm.to(BF16), h, K, y, K, q, K, scale, M, K, EPS)
        Y = torch.empty(M, N, dtype=BF16, device=dev)
        tcu.tcu_adapter_gemm_q8(q, K, scale, self.Wq, N, self.wscale, y, K, self.A.to(BF16),
                                self.B.to(BF16), self.alpha, ids, Y, N, self.work, M, K, N, self.r,
                                self.G)
        return h, Y


def train(layer, steps, M=512, lr=0.5, max_norm=1.0, seed=1):
    """Losses of `steps` steps on one batch of M rows in runs, one per adapter."""
    dev, K, N, r, G = layer.device, layer.K, layer.N, layer.r, layer.G
    g = torch.Generator(device=dev).manual_seed(seed)
    x = torch.randn(M, K, generator=g, device=dev).to(BF16)
    res = torch.randn(M, K, generator=g, device=dev).to(BF16)
    ids = (torch.arange(M, device=dev) * G // M).to(torch.int32)
    goal = Layer(K, N, r, G, M, seed=seed + 1, device=dev)
    goal.W, goal.B = layer.W, torch.randn(G, N, r, generator=g, device=dev) * r ** -0.5 * 0.5
    target = goal.forward(x, res, ids)[2].float()
    losses = []
    for _ in range(steps):
        h, y, Y = layer.forward(x, res, ids)
        diff = Y.float() - target
        losses.append(float((diff * diff).mean()))
        # the mean over the rows of the squared distance, a row's sum over N
        grads, _ = layer.backward(h, y, (diff / M).to(BF16), torch.zeros_like(h), ids)
        layer.step(grads, lr, max_norm)
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=60)
    a = ap.parse_args()
    layer = Layer(K=1024, N=768, r=16, G=4, rows=512)
    losses = train(layer, a.steps)
    print(f"training: loss {losses[0]:.4f} -> {losses[-1]:.4f} in {a.steps} steps")
    tokens = 24
    x, res = (torch.randn(tokens, layer.K, device="cuda").to(BF16) for _ in range(2))
    ids = torch.arange(tokens, device="cuda", dtype=torch.int32) % (layer.G + 1) - 1
    exact, q8 = layer.forward(x, res, ids)[2].float(), layer.decode(x, res, ids)[1].float()
    print(f"serving: {tokens} tokens, 8-bit weight against bfloat16: "
          f"{float((q8 - exact).norm() / exact.norm()):.4f} apart")


if __name__ == "__main__":
    main()

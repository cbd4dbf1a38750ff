"""The binding's operand checks of the operators around a layer's products, on
stand-in tensors (no device): an operand on the host or on another device is
refused, wherever it stands, before the library is called."""
import pytest
import torch

from paper_1908_06649_amd import tcu
from test_binding_checks import Fake

M, K, N, R, G = 5, 24, 40, 8, 3
BF16, F32, I32, I8 = torch.bfloat16, torch.float32, torch.int32, torch.int8


class Library:
    """The entry points by name: work sizes as they are, calls recorded."""

    def __init__(self, real):
        self.real, self.calls = real, []

    def __getattr__(self, name):
        if name.endswith("_work"):
            return getattr(self.real, name)
        return lambda *args: self.calls.append((name, args)) or tcu.TCU_OK


@pytest.fixture
def library(monkeypatch):
    fake = Library(tcu.lib())
    monkeypatch.setattr(tcu, "_lib", fake)
    monkeypatch.setattr(tcu, "_GET_DEVICE", lambda: 0)
    monkeypatch.setattr(tcu, "_RAW_STREAM", lambda dev: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return fake


def mats(*shapes):
    return [torch.zeros(s, dtype=t) for s, t in shapes]


FACTORS = (((G, R, K), BF16), ((G, N, R), BF16), ((G,), F32), ((M,), I32))
WORK = ((1 << 20,), torch.uint8)

# name -> (operands, call of them)
CALLS = {
    "tcu_rms_norm": (
        mats(((M, K), BF16), ((M, K), BF16), ((K,), BF16), ((M, K), BF16), ((M, K), BF16),
             ((M, K), I8), ((M,), F32)),
        lambda x, res, w, h, y, q, s: tcu.tcu_rms_norm(x, K, res, K, w, h, K, y, K, q, K, s, M, K,
                                                       1e-5)),
    "tcu_rms_norm_grad": (
        mats(((M, K), BF16), ((M, K), BF16), ((K,), BF16), ((M, K), BF16), ((M, K), BF16),
             ((K,), F32), WORK),
        lambda dy, h, w, dh, dx, dw, work: tcu.tcu_rms_norm_grad(dy, K, h, K, w, dh, K, dx, K, dw,
                                                                 work, M, K, 1e-5)),
    "tcu_adapter_gemm": (
        mats(((M, K), BF16), ((K, N), BF16), *FACTORS, ((M, N), F32), WORK),
        lambda X, W, A, B, al, ids, Y, work: tcu.tcu_adapter_gemm(X, K, W, N, A, B, al, ids, Y, N,
                                                                  work, M, K, N, R, G)),
    "tcu_adapter_gemm_q8": (
        mats(((M, K), I8), ((M,), F32), ((K, N), I8), ((N,), F32), ((M, K), BF16), *FACTORS,
             ((M, N), BF16), WORK),
        lambda Xq, xs, Wq, ws, X, A, B, al, ids, Y, work: tcu.tcu_adapter_gemm_q8(
            Xq, K, xs, Wq, N, ws, X, K, A, B, al, ids, Y, N, work, M, K, N, R, G)),
    "tcu_adapter_grad": (
        mats(((M, K), BF16), ((M, N), BF16), *FACTORS, ((G, R, K), F32), ((G, N, R), F32), WORK),
        lambda X, dY, A, B, al, ids, dA, dB, work: tcu.tcu_adapter_grad(
            X, K, dY, N, A, B, al, ids, dA, dB, work, M, K, N, R, G)),
    "tcu_adapter_input_grad": (
        mats(((M, N), BF16), ((N, K), BF16), *FACTORS, ((M, K), BF16), WORK),
        lambda dY, Wt, A, B, al, ids, dX, work: tcu.tcu_adapter_input_grad(
            dY, N, Wt, K, A, B, al, ids, dX, K, work, M, K, N, R, G)),
}


def outcome(name, devices):
    operands, call = CALLS[name]
    return call(*[Fake(t, d, 4096 * (i + 1)) for i, (t, d) in enumerate(zip(operands, devices))])


NAMES = list(CALLS)


@pytest.mark.parametrize("name", NAMES)
def test_operands_on_the_device_reach_the_library(library, name):
    count = len(CALLS[name][0])
    outcome(name, [0] * count)
    (called, args), = library.calls
    assert called == name and set(range(4096, 4096 * (count + 1), 4096)) <= set(args)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("other", [-1, 1])
def test_operands_elsewhere_are_refused(library, name, other):
    count = len(CALLS[name][0])
    for first in range(count):
        for last in range(first + 1, count + 1):
            devices = [other if first <= i < last else 0 for i in range(count)]
            with pytest.raises(ValueError):
                outcome(name, devices)
    assert library.calls == []

"""The binding's operand checks of the products in 4 bits and of the heads' norms, on
stand-in tensors (no device): an operand on the host or on another device is refused,
wherever it stands, before the library is called."""
import pytest
import torch

from paper_1908_06649_amd import tcu
from test_binding_checks import Fake
from test_layer_binding import Library as Recorder

M, K, N, T, HQ, HK, D = 5, 200, 30, 6, 3, 2, 32
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
WORK = ((1 << 20,), U8)


class Library(Recorder):
    def __getattr__(self, name):
        if name == "tcu_strerror":
            return self.real.tcu_strerror
        return super().__getattr__(name)


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


def held(rows, cols):
    g = (cols + 127) // 128
    return ((rows, 64 * g), U8), ((g, rows), I32)


HEADS = (((T, HQ, D), BF16), ((T, HK, D), BF16))
VECTORS = (((D,), BF16), ((D,), BF16), ((D // 2,), F32), ((T,), I32))

# name -> (operands, call of them)
CALLS = {
    "tcu_mx4_quant": (
        mats(((M, K), BF16), *held(M, K), *held(K, M)),
        lambda x, q, s, qt, ts: tcu.tcu_mx4_quant(x, K, q, 128, s, M, qt, 64, ts, K, M, K)),
    "tcu_mx4_dequant": (
        mats(*held(M, K), ((M, K), F32)),
        lambda q, s, y: tcu.tcu_mx4_dequant(q, 128, s, M, y, K, M, K)),
    "tcu_mx4_gemm": (
        mats(*held(M, K), *held(N, K), ((M, N), BF16), WORK),
        lambda A, a, B, b, C, work: tcu.tcu_mx4_gemm(A, 128, a, M, B, 128, b, N, C, N, work, M, K,
                                                     N)),
    "tcu_mx4_linear": (
        mats(((M, K), BF16), *held(N, K), ((M, N), F32), WORK),
        lambda X, W, w, Y, work: tcu.tcu_mx4_linear(X, K, W, 128, w, N, Y, N, work, M, K, N)),
    "tcu_qk_norm": (
        mats(*HEADS, *VECTORS, *HEADS),
        lambda q, k, wq, wk, f, p, yq, yk: tcu.tcu_qk_norm(q, k, wq, wk, f, p, yq, yk, T, HQ, HK, D,
                                                           D, 1e-5)),
    "tcu_qk_norm_grad": (
        mats(*HEADS, *HEADS, *VECTORS, *HEADS, ((D,), F32), ((D,), F32), WORK),
        lambda *t: tcu.tcu_qk_norm_grad(*t, T, HQ, HK, D, D, 1e-5)),
}


def outcome(name, devices, change=lambda operands: operands):
    operands, call = CALLS[name]
    return call(*[Fake(t, d, 4096 * (i + 1))
                  for i, (t, d) in enumerate(zip(change(list(operands)), devices))])


@pytest.mark.parametrize("name", CALLS)
def test_operands_on_the_device_reach_the_library(library, name):
    count = len(CALLS[name][0])
    outcome(name, [0] * count)
    (called, args), = library.calls
    assert called == name and set(range(4096, 4096 * (count + 1), 4096)) <= set(args)


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("other", [-1, 1])
def test_operands_elsewhere_are_refused(library, name, other):
    count = len(CALLS[name][0])
    for first in range(count):
        for last in range(first + 1, count + 1):
            devices = [other if first <= i < last else 0 for i in range(count)]
            with pytest.raises(ValueError):
                outcome(name, devices)
    assert library.calls == []


@pytest.mark.parametrize("name", CALLS)
def test_other_types_and_sizes_are_refused(library, name):
    count = len(CALLS[name][0])
    for i in range(count):
        for change in (lambda t: t.to(torch.float64), lambda t: t[..., :-1], lambda t: t[None],
                       lambda t: t.new_zeros(t.shape + (2,))[..., 0]):
            def swap(operands):
                operands[i] = change(operands[i])
                return operands
            if operands_ok(name, i, swap):
                continue
            with pytest.raises((ValueError, tcu.TcuError)):
                outcome(name, [0] * count, swap)
    assert library.calls == []


def operands_ok(name, i, swap):
    """Larger scratch of any type, and an output of another type, are fine."""
    t = swap(list(CALLS[name][0]))[i]
    old = CALLS[name][0][i]
    if old.shape == WORK[0] and old.dtype == WORK[1]:
        return True
    # (vectors of any shape with their elements)
    return old.dim() == 1 and t.dtype == old.dtype and t.numel() == old.numel() and \
        t.is_contiguous()


@pytest.mark.parametrize("name", ["tcu_qk_norm", "tcu_qk_norm_grad"])
def test_the_general_checks_pass_the_same_arguments(library, name, monkeypatch):
    """Without a rotation, which the flat condition does not take."""
    operands, call = CALLS[name]
    count = len(operands)
    outcome(name, [0] * count)
    flat = library.calls.pop()
    monkeypatch.setattr(tcu, "_current_device", lambda: 0)
    real = tcu._heads
    seen = []
    monkeypatch.setattr(tcu, "_heads", lambda *a: seen.append(1) or real(*a))
    fakes = [Fake(t, 0, 4096 * (i + 1)) for i, t in enumerate(operands)]
    rot0 = {"tcu_qk_norm": lambda q, k, wq, wk, f, p, yq, yk: tcu.tcu_qk_norm(
                q, k, wq, wk, None, None, yq, yk, T, HQ, HK, D, 0, 1e-5),
            "tcu_qk_norm_grad": lambda dyq, dyk, q, k, wq, wk, f, p, dq, dk, a, b, w:
                tcu.tcu_qk_norm_grad(dyq, dyk, q, k, wq, wk, None, None, dq, dk, a, b, w, T, HQ, HK,
                                     D, 0, 1e-5)}[name]
    rot0(*fakes)
    (_, args), = library.calls
    assert seen and flat[0] == name
    # the same but for freq, pos and rot
    different = [i for i, (x, y) in enumerate(zip(flat[1], args)) if x != y]
    assert len(args) == len(flat[1]) and len(different) == 3


@pytest.mark.parametrize("name", CALLS)
def test_absent_operands_are_the_librarys_to_refuse(library, name):
    """An operand that is None arrives as a null pointer; scratch that is needed and None, and an
    operand whose type the call takes for its own, are refused before."""
    operands, call = CALLS[name]
    for i in range(len(operands)):
        t = [Fake(t, 0, 4096 * (j + 1)) for j, t in enumerate(operands)]
        t[i] = None
        try:
            call(*t)
        except (ValueError, AttributeError):
            assert operands[i].shape == WORK[0] or operands[i].dtype in (BF16, F32)
            assert library.calls == []
            continue
        called, args = library.calls.pop()
        assert called == name and 4096 * (i + 1) not in args and None in args


@pytest.mark.parametrize("name,i", [("tcu_mx4_quant", 2), ("tcu_mx4_quant", 4),
                                    ("tcu_mx4_dequant", 0), ("tcu_mx4_linear", 1),
                                    ("tcu_mx4_linear", 2), ("tcu_mx4_gemm", 0), ("tcu_mx4_gemm", 3),
                                    ("tcu_qk_norm", 2), ("tcu_qk_norm", 4),
                                    ("tcu_qk_norm", 5), ("tcu_qk_norm", 7),
                                    ("tcu_qk_norm_grad", 1), ("tcu_qk_norm_grad", 9),
                                    ("tcu_qk_norm_grad", 11)])
def test_a_missing_operand_is_an_error_of_the_library(library, name, i):
    """Scales without codes, weights, tables or outputs that are missing arrive as null."""
    operands, call = CALLS[name]
    t = [Fake(t, 0, 4096 * (j + 1)) for j, t in enumerate(operands)]
    t[i] = None
    call(*t)
    (called, args), = library.calls
    assert called == name and None in args

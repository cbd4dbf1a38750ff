"""Sizes out of range are a shape error of the binding, with scratch and without it (stand-in
tensors, no device)."""
import pytest
import torch

from paper_1908_06649_amd import tcu
from test_binding_checks import Fake
from test_mx4_binding import library  # noqa: F401 (a fixture)

M = tcu.TCU_MAX_MX4_DIM + 1
T = 1 << 31
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def empty(*shape, t=BF16):
    return Fake(torch.empty(shape, dtype=t))


CALLS = {
    "tcu_mx4_gemm": lambda w: tcu.tcu_mx4_gemm(None, 0, None, 0, None, 0, None, 0, empty(M, 0), 0,
                                               w, M, 0, 0),
    "tcu_mx4_linear": lambda w: tcu.tcu_mx4_linear(empty(M, 0), 0, None, 0, None, 0, empty(M, 0), 0,
                                                   w, M, 0, 0),
    "tcu_qk_norm_grad": lambda w: tcu.tcu_qk_norm_grad(
        *[empty(0, 1, 2000) for _ in range(4)], empty(2000), empty(2000), None, empty(0, t=I32),
        empty(0, 1, 2000), empty(0, 1, 2000), empty(2000, t=F32), empty(2000, t=F32), w, 0, 1, 1,
        2000, 0, 1e-6),
    "tcu_rms_norm_grad": lambda w: tcu.tcu_rms_norm_grad(
        empty(0, T), T, empty(0, T), T, None, None, 0, empty(0, T), T, None, w, 0, T, 1e-6),
    "tcu_adapter_grad": lambda w: tcu.tcu_adapter_grad(
        empty(T, 0), 0, empty(T, 0), 0, None, None, None, None, None, None, w, T, 0, 0, 16, 1),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("work", [False, True])
def test_out_of_range(library, name, work):
    with pytest.raises(tcu.TcuError) as e:
        CALLS[name](empty(64, t=torch.uint8) if work else None)
    assert e.value.status == tcu.TCU_ERR_SHAPE and name in str(e.value)


def test_missing_work_is_named(library):
    with pytest.raises(ValueError, match="work needs"):
        tcu.tcu_mx4_gemm(None, 0, None, 0, None, 0, None, 0, empty(4, 8), 8, None, 4, 128, 8)

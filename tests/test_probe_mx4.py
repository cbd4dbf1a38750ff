"""The matrix-core ceiling probe in 4 bits (bench.py --mfma-probe): its type is known, and it
runs to completion on a small grid."""
import pytest
import torch    # (its HIP runtime is the process's: before the probes' library)

from paper_1908_06649_amd import tcu
from test_probe_lib import FAKE, P  # noqa: F401 (a fixture)

MX4 = 100


def test_types(P):
    for dt in (tcu.TCU_F16_F32, 99, 101, -1):
        assert P.tcu_probe_mfma(dt, FAKE, FAKE, 1, 1, None) == -1
    assert P.tcu_probe_mfma(MX4, FAKE, None, 1, 1, None) == -1
    assert P.tcu_probe_mfma(MX4, FAKE, FAKE, 1, 0, None) == -1


@pytest.mark.gpu
def test_runs(P):
    """Codes of 1 and scales of 1: every sum is 128 a round."""
    blocks, iters = 2, 3
    ops = torch.full((blocks * 512 * 12 * 4,), 0x22222222, dtype=torch.int32, device="cuda")
    out = torch.zeros(blocks * 512, dtype=torch.int32, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert P.tcu_probe_mfma(MX4, ops.data_ptr(), out.data_ptr(), iters, blocks, stream) == 0
    bits = int(torch.tensor(128.0 * iters).view(torch.int32))
    want = 0
    for _ in range(32 * 4):
        want = (want * 31 + bits) & 0xffffffff
    assert bool(((out.long() & 0xffffffff) == want).all())

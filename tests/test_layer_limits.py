"""The operators around a layer's products at the ends of their documented sizes, in
a process of their own on the recording runtime (tests/recording.py)."""
import random
import shutil

import pytest

from paper_1908_06649_amd import tcu

import recording as rec

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
P = rec.ptr
ROWS = 1 << 30      # TCU_MAX_RECT_DIM
DIM = 1 << 24       # TCU_MAX_ADAPTED_DIM


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return rec.build(tmp_path_factory.mktemp("recording"))


# every size within its own limit; the row operands of the first four pass 2^40 bytes, the
# last one's work does (T of both sides: 2 x 2^30 x 128 binary32 values)
SIZES = [(ROWS, 1 << 18, 1 << 18, 16, 4), (ROWS, DIM, DIM, 16, 0), (ROWS, DIM, 1, 16, 4),
         (ROWS, 1, DIM, 128, 65536), (ROWS, 512, 512, 128, 4)]
WITHIN = [(ROWS, 1, 1, 1, 1), (1, DIM, DIM, 16, 4), (1, DIM, DIM, 1, 0), (65535, DIM, DIM, 16, 1)]


def test_work_of_extreme_sizes(so):
    answers = rec.run(so, [dict(fn="tcu_adapter_work", args=list(s)) for s in SIZES + WITHIN])
    got = [a["rc"] for a in answers]
    assert got[:len(SIZES)] == [-1] * len(SIZES)
    for size, n in zip(WITHIN, got[len(SIZES):]):
        M, K, N, r, G = size
        # T of both sides and the rows' order at least
        assert M * r * 8 + M * 4 <= n < 1 << 40, size


@pytest.mark.parametrize("size", SIZES)
def test_calls_of_extreme_sizes_are_refused(so, size):
    M, K, N, r, G = size
    tail = [M, K, N, r, G]
    jobs = [
        dict(fn="tcu_adapter_gemm", args=[P(0), K, P(1), N, P(2), P(3), P(4), P(5), P(6), N, P(7),
                                          *tail, 2, None]),
        dict(fn="tcu_adapter_gemm_q8", args=[P(0), K, P(4), P(1), N, P(4), P(2), K, P(3), P(3),
                                             P(4), P(5), P(6), N, P(7), *tail, None]),
        dict(fn="tcu_adapter_grad", args=[P(0), K, P(1), N, P(2), P(2), P(4), P(5), P(6), P(3),
                                          P(7), *tail, 2, None]),
        dict(fn="tcu_adapter_input_grad", args=[P(0), N, P(1), K, P(2), P(3), P(4), P(5), P(6), K,
                                                P(7), *tail, 2, None])]
    for answer in rec.run(so, jobs):
        assert answer["rc"] == tcu.TCU_ERR_SHAPE and answer["launches"] == []


@pytest.mark.parametrize("rows", [0, 1, 600])
@pytest.mark.parametrize("cols", [(1 << 27) - 32, 1 << 27, (1 << 27) + 1, 1 << 30])
def test_norm_gradient_of_long_rows(so, rows, cols):
    """Work items of a launch count in 32 bits."""
    if rows * cols >= 1 << 38:     # (their bytes would pass 2^40)
        rows = 200
    args = [P(0), cols, P(1), cols, P(2), P(3), cols, P(4), cols, P(5), P(6), rows, cols, 1e-5, 2,
            None]
    answer = rec.run(so, [dict(fn="tcu_rms_norm_grad", args=args)])[0]
    assert answer["rc"] == tcu.TCU_OK
    assert len(answer["launches"]) == (2 if rows else 1)
    assert all(0 < la["blocks"] * la["threads"] < 1 << 32 for la in answer["launches"])


def test_work_of_more_rows_is_enough_for_fewer(so):
    """A program keeps the scratch of its largest batch."""
    rng = random.Random(3)
    jobs = []
    for _ in range(3000):
        K, N = (int(2 ** rng.uniform(0, 17)) for _ in range(2))
        rest = [K, N, rng.choice([1, 4, 8, 16, 20, 32, 64, 128]), int(2 ** rng.uniform(0, 8)) - 1]
        M = int(2 ** rng.uniform(0, 14))
        jobs += [dict(fn="tcu_adapter_work", args=[m, *rest]) for m in (rng.randint(0, M), M)]
    for M in range(1, 512):
        jobs += [dict(fn="tcu_adapter_work", args=[m, 4096, 4096, 16, 4]) for m in (M, 512)]
    got = [a["rc"] for a in rec.run(so, jobs)]
    for fewer, more, job in zip(got[::2], got[1::2], jobs[1::2]):
        assert 0 <= fewer <= more, job

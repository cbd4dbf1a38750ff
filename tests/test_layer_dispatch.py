"""The launches that the operators of a layer are made of (tests/recording.py), on a
device of 256 compute units."""
import shutil

import pytest

from paper_1908_06649_amd import tcu

import recording as rec

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
P = rec.ptr


@pytest.fixture(scope="module")
def so(tmp_path_factory):
    return rec.build(tmp_path_factory.mktemp("recording"))


def forward(M, K, N, r, G, dtype=2, **kw):
    return dict(fn="tcu_adapter_gemm", args=[P(0), K, P(1), N, P(2), P(3), P(4), P(5), P(6), N,
                                             P(7), M, K, N, r, G, dtype, None], **kw)


def q8(M, K, N, r, G, **kw):
    return dict(fn="tcu_adapter_gemm_q8",
                args=[P(0), K, P(4), P(1), N, P(4), P(2), K, P(3), P(3), P(4), P(5), P(6), N, P(7),
                      M, K, N, r, G, None], **kw)


def grad(M, K, N, r, G, **kw):
    return dict(fn="tcu_adapter_grad", args=[P(0), K, P(1), N, P(2), P(2), P(4), P(5), P(6), P(3),
                                             P(7), M, K, N, r, G, 2, None], **kw)


def kinds(answer):
    assert answer["rc"] == tcu.TCU_OK, answer["rc"]
    out = []
    for la in answer["launches"]:
        name = la["name"].split("_GLOBAL__N_1")[1].lstrip("0123456789")
        out.append("tail" if name.startswith("tail") else name.split("_kernel")[0])
    return out


@pytest.mark.parametrize("job,want", [
    # single tokens; the narrow product apart where its values are many
    (forward(1, 4096, 4096, 16, 8), ["few", "join"]),
    (forward(64, 8192, 8192, 16, 8), ["few", "join"]),
    (forward(64, 8192, 1024, 128, 8), ["narrow", "few", "join"]),
    (q8(48, 8192, 8192, 16, 16), ["few", "join"]),
    # up to 256 rows where the product has few tiles
    (forward(128, 4096, 4096, 16, 16), ["few", "join"]),
    (forward(256, 8192, 256, 16, 4), ["few", "join"]),
    (forward(256, 8192, 8192, 16, 4), ["narrow", "tail"]),
    (forward(257, 8192, 256, 16, 4), ["narrow", "tail"]),
    # prompts, the rank padded where it is no multiple of 8
    (forward(2000, 4096, 4096, 16, 12), ["narrow", "tail"]),
    (forward(2000, 4096, 4096, 20, 12), ["pad_ranks", "narrow", "tail"]),
    (forward(8192, 8192, 8192, 32, 4), ["narrow", "tail"]),
    (q8(4096, 4096, 8192, 16, 8), ["narrow", "tail"]),
    # too many rows or adapters to be looked through by every workgroup
    (forward(8193, 1024, 1024, 16, 4), ["group", "narrow", "tail"]),
    (forward(1000, 1024, 1024, 16, 600), ["group", "narrow", "tail"]),
    # no adapters
    (forward(2000, 4096, 4096, 16, 0), ["tail"])])
def test_launches(so, job, want):
    assert kinds(rec.run(so, [job])[0]) == want


def test_gradients(so):
    a, b = rec.run(so, [grad(8192, 4096, 4096, 16, 4), grad(0, 64, 64, 16, 4)])
    assert kinds(a) == ["prepare", "narrow", "factor", "finish"]
    assert kinds(b) == ["prepare", "finish"]


def test_more_pieces_than_a_launch(so):
    """Work items of a launch count in 32 bits."""
    answer = rec.run(so, [forward(1 << 28, 8, 8, 16, 1)])[0]
    assert answer["rc"] == tcu.TCU_OK
    narrow = [la for la in answer["launches"] if "narrow" in la["name"]]
    assert sum(la["blocks"] for la in narrow) == (1 << 28) // 16
    assert all(la["blocks"] * la["threads"] < 1 << 32 for la in answer["launches"])


@pytest.mark.parametrize("fail", [0, 1, 2])
def test_a_failed_launch_is_reported(so, fail):
    answer = rec.run(so, [forward(8193, 1024, 1024, 16, 4, fail=fail)])[0]
    assert answer["rc"] == tcu.TCU_ERR_HIP and len(answer["launches"]) == fail + 1

"""tcu_qk_norm and tcu_qk_norm_grad on packed rows of each head's query, key and value, token by
token and head by head, in place and not: the bits of contiguous operands, the values left as
they were."""
import pytest
import torch

from heads_util import Case
from layer_util import DEV
from paper_1908_06649_amd import tcu
from test_heads_gpu import backward, forward

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def packed(kind, a, b, more):
    """(buffer, views of a, b and the values beside them) of tokens x heads x dim operands."""
    T, H, D = a.shape
    if kind == "tokens":
        buf = torch.full((T, H * 3 * D + more), 7.0, dtype=a.dtype, device=DEV)
        v = buf[:, :H * 3 * D].view(T, H, 3, D) if not more else \
            buf.as_strided((T, H, 3, D), (H * 3 * D + more, 3 * D, D, 1))
    else:
        buf = torch.full((H, T * 3 * D + more), 7.0, dtype=a.dtype, device=DEV)
        v = buf.as_strided((T, H, 3, D), (3 * D, T * 3 * D + more, D, 1))
    v[:, :, 0], v[:, :, 1] = a.to(DEV), b.to(DEV)
    return buf, v[:, :, 0], v[:, :, 1], v[:, :, 2]


def rest_is_kept(buf, a, b):
    left = buf.clone()
    for v in (a, b):
        left.as_strided(v.shape, v.stride(), v.storage_offset()).fill_(7.0)
    return bool((left == 7).all())


@pytest.mark.parametrize("kind", ["tokens", "heads"])
@pytest.mark.parametrize("more", [0, 5])
@pytest.mark.parametrize("size", [(7, 4, 4, 64, 64), (1, 3, 3, 128, 128), (9, 2, 2, 80, 40),
                                  (5, 3, 3, 33, 20), (2100, 2, 2, 64, 64)])
@pytest.mark.parametrize("dtype,adjacent", [(BF16, False), (F32, True)])
def test_heads_side_by_side(kind, more, size, dtype, adjacent):
    c = Case(*size, dtype)
    T, H, _, D, rot = size
    flags = tcu.TCU_ROPE_ADJACENT if adjacent else 0
    want = forward(c, adjacent, 1e-6)
    grads = backward(c, adjacent, 1e-6)
    zero = torch.zeros_like(c.q)
    for in_place in (True, False):
        buf, q, k, _ = packed(kind, c.q, c.k, more)
        out, yq, yk = (buf, q, k) if in_place else packed(kind, zero, zero, more)[:3]
        tcu.tcu_qk_norm(q, k, *c.vectors(), yq, yk, T, H, H, D, rot, 1e-6, flags)
        assert torch.equal(yq, want[0]) and torch.equal(yk, want[1])
        assert rest_is_kept(out, yq, yk) and rest_is_kept(buf, q, k)
    work = torch.empty(tcu.tcu_qk_norm_grad_work(T, H, H, D), dtype=torch.uint8, device=DEV)
    for over in ("x", "dy", None):
        buf, q, k, _ = packed(kind, c.q, c.k, more)
        gbuf, dyq, dyk, _ = packed(kind, c.dyq, c.dyk, more)
        out, dq, dk = {"x": (buf, q, k), "dy": (gbuf, dyq, dyk)}.get(over) or \
            packed(kind, zero, zero, more)[:3]
        dw = torch.empty(2, D, device=DEV)
        tcu.tcu_qk_norm_grad(dyq, dyk, q, k, *c.vectors(), dq, dk, dw[0], dw[1], work, T, H, H, D,
                             rot, 1e-6, flags)
        assert torch.equal(dq, grads[0]) and torch.equal(dk, grads[1])
        assert torch.equal(dw, grads[2])
        assert rest_is_kept(out, dq, dk)

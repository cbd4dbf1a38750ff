"""Python binding of the C ABI in include/tcu.h (argument marshalling only).

Functions carry the C names.  Matrices are torch tensors on the current HIP
device; torch supplies device memory and the stream, nothing else -- every
step of the computation runs in the library's HIP kernels.  There is no
fallback: if ``libtcu.so`` is missing or fails to load, every call raises.

    tcu_mm_tall(A, n, s, B, C)   C (n x s) = A (n x s) @ B (s x s)     (native call)
    tcu_gemm(A, B, C, N)         C (N x N) = A @ B, unit size tcu_get_unit()
    tcu_transitive_closure(X, n, ld)   X <- transitive closure, in place (Theorem 5)
    tcu_dft(x, y, work, n, batch)   y[b] = DFT(x[b]), complex64        (Theorem 7)
    tcu_poly_eval(coef, n, points, p, out)
                                 out[i] = sum_h coef[h] * points[i]**h    (Theorem 11)
    tcu_gemm_rect(A, lda, B, ldb, C, ldc, M, K, N, flags)
                                 C (M x N) = [C +] A (M x K) @ B (K x N); A, B and C
                                 may be row-strided 2-D views (row pitch = ld)

and the operators around a layer's products:

    tcu_rms_norm(x, ldx, res, ldr, w, h, ldh, y, ldy, q, ldq, qscale, rows, cols, eps)
                                 h = x + res, y = its RMS norm, q = y in 8 bits
    tcu_rms_norm_grad(dy, lddy, h, ldh, w, dh, lddh, dx, lddx, dw, work, rows, cols, eps)
    tcu_adapter_gemm(X, ldx, W, ldw, A, B, alpha, ids, Y, ldy, work, M, K, N, r, G)
                                 Y[m] = X[m] W + alpha[g] (X[m] A[g]^T) B[g]^T, g = ids[m]
    tcu_adapter_gemm_q8(Xq, ldxq, xscale, Wq, ldwq, wscale, X, ldx, A, B, alpha, ids, Y, ldy,
                        work, M, K, N, r, G)
                                 the same with an int8 base and scales
    tcu_adapter_grad(X, ldx, dY, lddy, A, B, alpha, ids, dA, dB, work, M, K, N, r, G)
    tcu_adapter_input_grad(dY, lddy, Wt, ldwt, A, B, alpha, ids, dX, lddx, work, M, K, N, r, G)
    tcu_clip_grads(grads, outs, max_norm, result, work)
                                 outs = grads * min(1, max_norm / (norm + 1e-6))

products in 4 bits (codes and power-of-two scales of blocks of 32, include/tcu.h) and
what queries and keys go through after their projection:

    tcu_mx4_quant(x, ldx, q, ldq, scale, lds, qt, ldqt, tscale, ldts, rows, cols)
                                 x in 4 bits along its rows and along its columns
    tcu_mx4_dequant(q, ldq, scale, lds, y, ldy, rows, cols)
    tcu_mx4_gemm(A, lda, ascale, ldas, B, ldb, bscale, ldbs, C, ldc, work, M, K, N, flags)
                                 C (M x N) = [C +] A (M x K) @ B (N x K)^T
    tcu_mx4_linear(X, ldx, W, ldw, wscale, ldws, Y, ldy, work, M, K, N, flags)
                                 the same with a 16-bit left operand
    tcu_qk_norm(q, k, wq, wk, freq, pos, yq, yk, tokens, hq, hk, dim, rot, eps, flags)
                                 every head's RMS norm, its pairs turned by the position
    tcu_qk_norm_grad(dyq, dyk, q, k, wq, wk, freq, pos, dq, dk, dwq, dwk, work, tokens, hq, hk,
                     dim, rot, eps, flags)

The element types are taken from the tensors: (float16 -> float32),
(bfloat16 -> float32), (bfloat16 -> bfloat16) or (int8 -> int32).  Calls are
issued on torch's current stream and are asynchronous.
"""
from __future__ import annotations

import array
import ctypes
import os

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libtcu.so")

TCU_OK = 0
TCU_ERR_NULL = -1
TCU_ERR_SHAPE = -2
TCU_ERR_UNSUPPORTED = -3
TCU_ERR_ALIGN = -4
TCU_ERR_OVERLAP = -5
TCU_ERR_HIP = -6
TCU_ERR_NO_DEVICE = -7
TCU_ERR_POINTER = -8
TCU_ERR_SCRATCH = -9

TCU_F16_F32 = 0
TCU_BF16_F32 = 1
TCU_BF16_BF16 = 2
TCU_I8_I32 = 3

TCU_ACCUMULATE = 1

# Test overrides and the pointer-check switch (tcu_set_knob)
TCU_KNOB_GEMM_KERNEL = 0
TCU_KNOB_PP_GRID = 1
TCU_KNOB_SPLIT_K = 2
TCU_KNOB_TAIL_SPLIT = 3
TCU_KNOB_CHECK_POINTERS = 4
TCU_KNOB_DFT_PAIRS = 5
TCU_PATH_AUTO = 0
TCU_PATH_FULL_TILE = 1
TCU_PATH_GENERAL = 2
TCU_PATH_RING = 3
TCU_MAX_RECT_DIM = 1 << 30

# Every symbol include/tcu.h declares: name -> (restype, argtypes)
_i64, _int, _vp = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p
SIGNATURES = {
    "tcu_set_unit": (_int, [_int]),
    "tcu_get_unit": (_int, []),
    "tcu_set_dtype": (_int, [_int]),
    "tcu_get_dtype": (_int, []),
    "tcu_set_stream": (_int, [_vp]),
    "tcu_get_stream": (_vp, []),
    "tcu_mm_tall": (_int, [_vp, _i64, _int, _vp, _vp]),
    "tcu_gemm": (_int, [_vp, _vp, _vp, _i64]),
    "tcu_mm_tall_ex": (_int, [_vp, _i64, _int, _vp, _vp, _int, _vp]),
    "tcu_gemm_ex": (_int, [_vp, _vp, _vp, _i64, _int, _int, _vp]),
    "tcu_gemm_rect": (_int, [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _i64, _int]),
    "tcu_gemm_rect_ex": (_int, [_vp, _i64, _vp, _i64, _vp, _i64, _i64, _i64, _i64, _int,
                                _int, _int, _vp]),
    "tcu_poly_eval": (_int, [_vp, _i64, _vp, _i64, _vp]),
    "tcu_poly_eval_ex": (_int, [_vp, _i64, _vp, _i64, _vp, _int, _int, _vp]),
    "tcu_transitive_closure": (_int, [_vp, _i64, _i64]),
    "tcu_transitive_closure_ex": (_int, [_vp, _i64, _i64, _int, _vp]),
    "tcu_dft": (_int, [_vp, _vp, _vp, _i64, _i64]),
    "tcu_dft_ex": (_int, [_vp, _vp, _vp, _i64, _i64, _int, _vp]),
    "tcu_dft_noalloc": (_int, [_vp, _vp, _i64, _i64, _int, _vp]),
    "tcu_rms_norm": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _i64, _vp, _i64,
                            _i64, ctypes.c_float, _int, _vp]),
    "tcu_rms_norm_grad": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _i64, _vp, _i64, _vp, _vp, _i64,
                                 _i64, ctypes.c_float, _int, _vp]),
    "tcu_rms_norm_grad_work": (_i64, [_i64, _i64]),
    "tcu_adapter_gemm": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp, _i64,
                                _i64, _i64, _i64, _i64, _int, _vp]),
    "tcu_adapter_gemm_q8": (_int, [_vp, _i64, _vp, _vp, _i64, _vp, _vp, _i64, _vp, _vp, _vp, _vp,
                                   _vp, _i64, _vp, _i64, _i64, _i64, _i64, _i64, _vp]),
    "tcu_adapter_grad": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _vp, _vp, _i64,
                                _i64, _i64, _i64, _i64, _int, _vp]),
    "tcu_adapter_input_grad": (_int, [_vp, _i64, _vp, _i64, _vp, _vp, _vp, _vp, _vp, _i64, _vp,
                                      _i64, _i64, _i64, _i64, _i64, _int, _vp]),
    "tcu_adapter_work": (_i64, [_i64, _i64, _i64, _i64, _i64]),
    "tcu_clip_grads": (_int, [_vp, _vp, _vp, _vp, _i64, ctypes.c_float, _vp, _vp, _vp]),
    "tcu_clip_grads_work": (_i64, []),
    "tcu_mx4_quant": (_int, [_vp, _i64] * 5 + [_i64, _i64, _int, _vp]),
    "tcu_mx4_dequant": (_int, [_vp, _i64] * 3 + [_i64, _i64, _int, _vp]),
    "tcu_mx4_gemm": (_int, [_vp, _i64] * 5 + [_vp, _i64, _i64, _i64, _int, _int, _vp]),
    "tcu_mx4_linear": (_int, [_vp, _i64] * 4 + [_vp, _i64, _i64, _i64, _int, _int, _int, _vp]),
    "tcu_mx4_work": (_i64, [_i64, _i64, _i64]),
    "tcu_qk_norm": (_int, [_vp, _i64, _i64] * 2 + [_vp] * 4 + [_vp, _i64, _i64] * 2 +
                    [_i64] * 5 + [ctypes.c_float, _int, _int, _vp]),
    "tcu_qk_norm_grad": (_int, [_vp, _i64, _i64] * 4 + [_vp] * 4 + [_vp, _i64, _i64] * 2 +
                         [_vp] * 3 + [_i64] * 5 + [ctypes.c_float, _int, _int, _vp]),
    "tcu_qk_norm_grad_work": (_i64, [_i64, _i64, _i64, _i64]),
    "tcu_calls": (_i64, []),
    "tcu_square_calls": (_i64, []),
    "tcu_work": (_i64, []),
    "tcu_reset_calls": (None, []),
    "tcu_strerror": (ctypes.c_char_p, [_int]),
    "tcu_check_device_range": (_int, [_vp, _i64]),
    "tcu_set_knob": (_int, [_int, _int]),
    "tcu_get_knob": (_int, [_int]),
}

_lib = None


class TcuError(RuntimeError):
    def __init__(self, status: int, where: str):
        self.status = status
        super().__init__(f"{where}: {tcu_strerror(status)} (status {status})")


def lib() -> ctypes.CDLL:
    """The loaded C library (raises if it was not built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build the HIP library first "
                "(python -c 'import __graft_entry__ as g; g.build()')")
        handle = ctypes.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _lib = handle
    return _lib


def _check(rc: int, where: str) -> None:
    if rc != TCU_OK:
        raise TcuError(rc, where)


_DTYPES = {}        # (input, output) torch dtypes -> code; the polynomials take no int8
_POLY_DTYPES = {}


def _dtype_tables():
    import torch
    floats = {(torch.float16, torch.float32): TCU_F16_F32,
              (torch.bfloat16, torch.float32): TCU_BF16_F32,
              (torch.bfloat16, torch.bfloat16): TCU_BF16_BF16}
    # one update each: another thread sees a table empty or whole
    _POLY_DTYPES.update(floats)
    _DTYPES.update({**floats, (torch.int8, torch.int32): TCU_I8_I32})


def _dtype_code(a_dtype, c_dtype, table=_DTYPES) -> int:
    if not table:
        _dtype_tables()
    code = table.get((a_dtype, c_dtype))
    if code is None:
        raise TcuError(TCU_ERR_UNSUPPORTED, f"dtype pair ({a_dtype}, {c_dtype})")
    return code


def _check_current_device(where: str, dev: int) -> None:
    """The library launches on the current HIP device: the tensors must be
    there (select it with torch.cuda.device(...))."""
    import torch
    cur = torch.cuda.current_device()
    if dev != cur:
        raise ValueError(f"{where}: tensors are on cuda:{dev}, the current device is cuda:{cur}")


_GET_DEVICE = None


def _current_device() -> int:
    """torch.cuda.current_device() without its per-call initialisation check
    (the callers hold device tensors, so the runtime is initialised)."""
    global _GET_DEVICE
    if _GET_DEVICE is None:
        import torch
        _GET_DEVICE = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _GET_DEVICE()


# The small calls are bound by the host: about 4 us of launch, and in Python
# the checks of the operands.  The common case -- everything as it should be
# -- is therefore one flat condition per shape of call; any other operands
# take the general checks below, which raise.  A native call on 4096 rows: 6.0
# us with the general checks alone, 5.2 with the flat ones.

def _marshal3(where, A, B, C, na, nb, nc):
    """_marshal of three tensors."""
    dev = A.get_device()
    if (dev >= 0 and B.get_device() == dev and C.get_device() == dev and A.is_contiguous()
            and B.is_contiguous() and C.is_contiguous() and A.numel() == na and B.numel() == nb
            and C.numel() == nc and A.is_cuda and _current_device() == dev):
        return dev, A.data_ptr(), B.data_ptr(), C.data_ptr()
    dev, (pa, pb, pc) = _marshal(where, (A, B, C), (na, nb, nc))
    return dev, pa, pb, pc


def _marshal_views3(where, A, lda, B, ldb, C, ldc, M, K, N):
    """_marshal_views of a product's operands."""
    dev = A.get_device()
    if (dev >= 0 and B.get_device() == dev and C.get_device() == dev and A.shape == (M, K)
            and B.shape == (K, N) and C.shape == (M, N) and A.stride() == (lda, 1)
            and B.stride() == (ldb, 1) and C.stride() == (ldc, 1) and A.is_cuda
            and _current_device() == dev):
        return dev, A.data_ptr(), B.data_ptr(), C.data_ptr()
    dev, (pa, pb, pc) = _marshal_views(where, ((A, M, K, lda), (B, K, N, ldb), (C, M, N, ldc)))
    return dev, pa, pb, pc


def _marshal(where: str, tensors, numels):
    """Check that tensors are contiguous, on one HIP device (the current one),
    and sized as the call will read/write them; return the device index and
    their device pointers."""
    dev = tensors[0].get_device() if tensors[0].is_cuda else -1
    ptrs = []
    for t, want in zip(tensors, numels):
        if not t.is_cuda or t.get_device() != dev:
            raise ValueError(f"{where}: all matrices must be on the same HIP device")
        if not t.is_contiguous():
            raise ValueError(f"{where}: matrices must be contiguous (row-major)")
        if t.numel() != want:
            raise ValueError(f"{where}: expected {want} elements, got {t.numel()}")
        ptrs.append(t.data_ptr())
    _check_current_device(where, dev)
    return dev, ptrs


_RAW_STREAM = None


def _stream_ptr(dev: int) -> int:
    """The current torch stream of device dev, as a hipStream_t value."""
    global _RAW_STREAM
    if _RAW_STREAM is None:
        import torch
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _RAW_STREAM = raw if raw is not None else (
            lambda d: torch.cuda.current_stream(d).cuda_stream)
    return _RAW_STREAM(dev)


# ------------------------------------------------------------ configuration
def tcu_set_unit(s: int) -> None:
    _check(lib().tcu_set_unit(int(s)), "tcu_set_unit")


def tcu_get_unit() -> int:
    return int(lib().tcu_get_unit())


def tcu_set_dtype(dtype: int) -> None:
    _check(lib().tcu_set_dtype(int(dtype)), "tcu_set_dtype")


def tcu_get_dtype() -> int:
    return int(lib().tcu_get_dtype())


def tcu_set_stream(stream_ptr: int | None) -> None:
    _check(lib().tcu_set_stream(stream_ptr), "tcu_set_stream")


def tcu_get_stream() -> int | None:
    return lib().tcu_get_stream()


# ------------------------------------------------------------------- calls
def tcu_mm_tall(A, n: int, s: int, B, C) -> None:
    """Native call: C (n x s) = A (n x s) @ B (s x s); s must equal the unit size."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal3("tcu_mm_tall", A, B, C, n * s, s * s, n * s)
    L = _lib or lib()
    _check(L.tcu_set_dtype(dt), "tcu_mm_tall")
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_mm_tall")
    _check(L.tcu_mm_tall(pa, int(n), int(s), pb, pc), "tcu_mm_tall")


def tcu_gemm(A, B, C, N: int) -> None:
    """Blocked product of Theorem 2: C (N x N) = A @ B with unit size tcu_get_unit()."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal3("tcu_gemm", A, B, C, N * N, N * N, N * N)
    L = _lib or lib()
    _check(L.tcu_set_dtype(dt), "tcu_gemm")
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_gemm")
    _check(L.tcu_gemm(pa, pb, pc, int(N)), "tcu_gemm")


def tcu_mm_tall_ex(A, n: int, s: int, B, C, stream_ptr: int | None = None) -> None:
    """Stateless native call (unit size, dtype and stream as arguments)."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal3("tcu_mm_tall_ex", A, B, C, n * s, s * s, n * s)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check((_lib or lib()).tcu_mm_tall_ex(pa, int(n), int(s), pb, pc, dt, st), "tcu_mm_tall_ex")


def tcu_gemm_ex(A, B, C, N: int, s: int, stream_ptr: int | None = None) -> None:
    """Stateless blocked product (unit size, dtype and stream as arguments)."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal3("tcu_gemm_ex", A, B, C, N * N, N * N, N * N)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check((_lib or lib()).tcu_gemm_ex(pa, pb, pc, int(N), int(s), dt, st), "tcu_gemm_ex")


def _marshal_views(where: str, views):
    """(tensor, rows, cols, ld) per operand: check that each is a 2-D view of
    that shape with unit column stride and row pitch ld on one HIP device
    (the current one); return the device index and the view base pointers."""
    dev = views[0][0].get_device() if views[0][0].is_cuda else -1
    ptrs = []
    for t, rows, cols, ld in views:
        if not t.is_cuda or t.get_device() != dev:
            raise ValueError(f"{where}: all matrices must be on the same HIP device")
        if t.dim() != 2 or tuple(t.shape) != (rows, cols):
            raise ValueError(f"{where}: expected a {rows} x {cols} view, got {tuple(t.shape)}")
        if cols > 1 and t.stride(1) != 1:
            raise ValueError(f"{where}: rows must be contiguous (column stride 1)")
        if rows > 1 and t.stride(0) != ld:
            raise ValueError(f"{where}: row pitch {t.stride(0)} does not match ld={ld}")
        ptrs.append(t.data_ptr())
    _check_current_device(where, dev)
    return dev, ptrs


def tcu_gemm_rect(A, lda: int, B, ldb: int, C, ldc: int, M: int, K: int, N: int,
                  flags: int = 0) -> None:
    """C (M x N) = A (M x K) @ B (K x N), or C += A @ B with flags=TCU_ACCUMULATE
    (Corollary 1 / the D functions' update); unit size tcu_get_unit()."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal_views3("tcu_gemm_rect", A, lda, B, ldb, C, ldc, M, K, N)
    L = _lib or lib()
    _check(L.tcu_set_dtype(dt), "tcu_gemm_rect")
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_gemm_rect")
    _check(L.tcu_gemm_rect(pa, int(lda), pb, int(ldb), pc, int(ldc), int(M), int(K), int(N),
                           int(flags)), "tcu_gemm_rect")


def tcu_gemm_rect_ex(A, lda: int, B, ldb: int, C, ldc: int, M: int, K: int, N: int, flags: int,
                     s: int, stream_ptr: int | None = None) -> None:
    """Stateless rectangular / accumulating product (unit size, dtype, stream as arguments)."""
    dt = _dtype_code(A.dtype, C.dtype)
    dev, pa, pb, pc = _marshal_views3("tcu_gemm_rect_ex", A, lda, B, ldb, C, ldc, M, K, N)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check((_lib or lib()).tcu_gemm_rect_ex(pa, int(lda), pb, int(ldb), pc, int(ldc), int(M),
                                            int(K), int(N), int(flags), int(s), dt, st),
           "tcu_gemm_rect_ex")


def tcu_poly_eval(coef, n: int, points, p: int, out) -> None:
    """Theorem 11: out[i] = sum_{h<n} coef[h] * points[i]**h, unit size tcu_get_unit()."""
    dt = _dtype_code(points.dtype, out.dtype, _POLY_DTYPES)
    if coef.dtype != points.dtype:
        raise ValueError("tcu_poly_eval: coefficients and points must share one input type")
    dev, ppts, pcoef, pout = _marshal3("tcu_poly_eval", points, coef, out, p, n, p)
    L = _lib or lib()
    _check(L.tcu_set_dtype(dt), "tcu_poly_eval")
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_poly_eval")
    _check(L.tcu_poly_eval(pcoef or None, int(n), ppts or None, int(p), pout or None),
           "tcu_poly_eval")


def tcu_poly_eval_ex(coef, n: int, points, p: int, out, s: int,
                     stream_ptr: int | None = None) -> None:
    """Stateless batch polynomial evaluation (unit size, dtype, stream as arguments)."""
    dt = _dtype_code(points.dtype, out.dtype, _POLY_DTYPES)
    if coef.dtype != points.dtype:
        raise ValueError("tcu_poly_eval_ex: coefficients and points must share one input type")
    dev, ppts, pcoef, pout = _marshal3("tcu_poly_eval_ex", points, coef, out, p, n, p)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check((_lib or lib()).tcu_poly_eval_ex(pcoef or None, int(n), ppts or None, int(p),
                                            pout or None, int(s), dt, st), "tcu_poly_eval_ex")


def tcu_transitive_closure(X, n: int, ld: int) -> None:
    """Theorem 5, in place: X (an n x n int8 view with row pitch ld) becomes
    the transitive closure of the graph it is the adjacency matrix of."""
    import torch
    if X.dtype not in (torch.int8, torch.uint8):
        raise ValueError("tcu_transitive_closure: X must be int8 or uint8")
    dev, (px,) = _marshal_views("tcu_transitive_closure", ((X, n, n, ld),))
    L = lib()
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_transitive_closure")
    _check(L.tcu_transitive_closure(px or None, int(n), int(ld)), "tcu_transitive_closure")


def tcu_transitive_closure_ex(X, n: int, ld: int, s: int, stream_ptr: int | None = None) -> None:
    """Stateless transitive closure (unit size and stream as arguments)."""
    import torch
    if X.dtype not in (torch.int8, torch.uint8):
        raise ValueError("tcu_transitive_closure_ex: X must be int8 or uint8")
    dev, (px,) = _marshal_views("tcu_transitive_closure_ex", ((X, n, n, ld),))
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check(lib().tcu_transitive_closure_ex(px or None, int(n), int(ld), int(s), st),
           "tcu_transitive_closure_ex")


_COMPLEX64 = None


def _dft_args(where, x, y, work, n, batch):
    global _COMPLEX64
    if _COMPLEX64 is None:
        import torch
        _COMPLEX64 = torch.complex64
    if x.dtype != _COMPLEX64 or y.dtype != _COMPLEX64:
        raise ValueError(f"{where}: {'x' if x.dtype != _COMPLEX64 else 'y'} must be complex64")
    total = n * batch
    if work is None:
        dev, (px, py) = _marshal(where, (x, y), (total, total))
        return dev, px or None, py or None, None
    dev, px, py, pw = _marshal3(where, x, y, work, total, total, total)
    if work.dtype != _COMPLEX64:
        raise ValueError(f"{where}: work must be complex64")
    return dev, px or None, py or None, pw or None


def tcu_dft(x, y, work, n: int, batch: int) -> None:
    """Theorem 7: y[b] = DFT(x[b]) for b < batch (complex64 tensors of
    batch * n elements); work is scratch of the same size (None if n <= s)."""
    dev, px, py, pw = _dft_args("tcu_dft", x, y, work, n, batch)
    L = lib()
    _check(L.tcu_set_stream(_stream_ptr(dev)), "tcu_dft")
    _check(L.tcu_dft(px, py, pw, int(n), int(batch)), "tcu_dft")


def tcu_dft_ex(x, y, work, n: int, batch: int, s: int, stream_ptr: int | None = None) -> None:
    """Stateless DFT (unit size and stream as arguments)."""
    dev, px, py, pw = _dft_args("tcu_dft_ex", x, y, work, n, batch)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check(lib().tcu_dft_ex(px, py, pw, int(n), int(batch), int(s), st), "tcu_dft_ex")


TCU_DFT_NOALLOC_MAX_BYTES = 64 << 20


def tcu_dft_noalloc(x, y, n: int, batch: int, s: int, stream_ptr: int | None = None) -> None:
    """The DFT with the levels' second buffer in the library's fixed device
    scratch (no allocation; batch * n * 8 <= TCU_DFT_NOALLOC_MAX_BYTES when
    n > s); calls overlapping in time on one device race on that scratch."""
    dev, px, py, _ = _dft_args("tcu_dft_noalloc", x, y, None, n, batch)
    st = _stream_ptr(dev) if stream_ptr is None else stream_ptr
    _check(lib().tcu_dft_noalloc(px, py, int(n), int(batch), int(s), st), "tcu_dft_noalloc")


# ------------------------------------------------ operators around a layer's products
TCU_ELEM_F32 = 0
TCU_ELEM_F16 = 1
TCU_ELEM_BF16 = 2
TCU_MAX_ADAPTERS = 1 << 16
TCU_MAX_RANK = 128

_ELEMS = {}
_BF16 = _F32 = _I32 = _I8 = _U8 = None
_NO_DEVICE = -2     # before the first tensor


def _elem_code(where: str, dtype) -> int:
    global _BF16, _F32, _I32, _I8, _U8
    if not _ELEMS:
        import torch
        _U8 = torch.uint8
        _BF16, _F32, _I32, _I8 = torch.bfloat16, torch.float32, torch.int32, torch.int8
        _ELEMS.update({torch.float32: TCU_ELEM_F32, torch.float16: TCU_ELEM_F16,
                       torch.bfloat16: TCU_ELEM_BF16})
    code = _ELEMS.get(dtype)
    if code is None:
        raise TcuError(TCU_ERR_UNSUPPORTED, f"{where}: element type {dtype}")
    return code


def _addresses(where: str, views, vectors, work, nbytes: int):
    """Checks of an operator's tensors: views (tensor, dtype, rows, cols, ld) are 2-D
    with unit column stride and row pitch ld, vectors (tensor, dtype, elements) are
    contiguous, all on the current HIP device, and work holds nbytes.  A tensor
    may be None where the call allows it.  Returns the device index and the
    addresses (None for absent tensors), work's last."""
    dev, ptrs = _NO_DEVICE, []
    for t, dtype, rows, cols, ld in views:
        if t is None:
            ptrs.append(None)
            continue
        d = t.get_device()
        if d != dev:
            dev = _first_device(where, dev, d)
        if t.dtype != dtype or t.shape != (rows, cols) or t.stride() != (ld, 1):
            _check_view(where, t, dtype, rows, cols, ld)
        ptrs.append(t.data_ptr() or None)
    for t, dtype, n in vectors:
        if t is None:
            ptrs.append(None)
            continue
        d = t.get_device()
        if d != dev:
            dev = _first_device(where, dev, d)
        if t.dtype != dtype:
            raise ValueError(f"{where}: expected {dtype}, got {t.dtype}")
        if t.numel() != n or not t.is_contiguous():
            raise ValueError(f"{where}: expected {n} contiguous elements, got {tuple(t.shape)}")
        ptrs.append(t.data_ptr() or None)
    if nbytes < 0:
        raise TcuError(TCU_ERR_SHAPE, where)
    if work is not None:
        if work.get_device() != dev or not work.is_contiguous() or \
                work.numel() * work.element_size() < nbytes:
            raise ValueError(f"{where}: work needs {nbytes} contiguous bytes on the same device")
        ptrs.append(work.data_ptr() or None)
    elif nbytes:
        raise ValueError(f"{where}: work needs {nbytes} contiguous bytes on the same device")
    if dev < 0:
        raise ValueError(f"{where}: all tensors must be on the same HIP device")
    if dev != _current_device():
        _check_current_device(where, dev)
    return dev, ptrs


def _first_device(where, dev, d):
    """d, the first tensor's device; a host tensor's is -1, also of the first."""
    if dev != _NO_DEVICE or d < 0:
        raise ValueError(f"{where}: all tensors must be on the same HIP device")
    return d


def _check_view(where, t, dtype, rows, cols, ld):
    """The general checks of a view (a pitch counts only between rows)."""
    if t.dtype != dtype:
        raise ValueError(f"{where}: expected {dtype}, got {t.dtype}")
    if t.shape != (rows, cols):
        raise ValueError(f"{where}: expected a {rows} x {cols} view, got {tuple(t.shape)}")
    st = t.stride()
    if rows and cols and ((st[1] != 1 and cols > 1) or (st[0] != ld and rows > 1)):
        raise ValueError(f"{where}: strides {st} do not match rows of pitch {ld}")


def _stream_of(dev: int, stream_ptr):
    return _stream_ptr(dev) if stream_ptr is None else stream_ptr


def tcu_rms_norm(x, ldx: int, res, ldr: int, w, h, ldh: int, y, ldy: int, q, ldq: int, qscale,
                 rows: int, cols: int, eps: float, stream_ptr: int | None = None) -> None:
    """h = x + res, y = h / sqrt(mean(h^2) + eps) * w and y in 8 bits (q int8, qscale
    float32 per row); res, h, y and (q, qscale) may be None."""
    t = x.dtype
    elem = _elem_code("tcu_rms_norm", t)
    dev, (px, pr, ph, py, pq, pw, ps) = _addresses(
        "tcu_rms_norm", ((x, t, rows, cols, ldx), (res, t, rows, cols, ldr),
                         (h, t, rows, cols, ldh), (y, t, rows, cols, ldy),
                         (q, _I8, rows, cols, ldq)),
        ((w, t, cols), (qscale, _F32, rows)), None, 0)
    _check((_lib or lib()).tcu_rms_norm(px, ldx, pr, ldr, pw, ph, ldh, py, ldy, pq, ldq, ps, rows,
                                        cols, eps, elem, _stream_of(dev, stream_ptr)),
           "tcu_rms_norm")


def tcu_rms_norm_grad_work(rows: int, cols: int) -> int:
    """Bytes of tcu_rms_norm_grad's work (-1: a size out of range)."""
    return (_lib or lib()).tcu_rms_norm_grad_work(rows, cols)


def tcu_rms_norm_grad(dy, lddy: int, h, ldh: int, w, dh, lddh: int, dx, lddx: int, dw, work,
                      rows: int, cols: int, eps: float, stream_ptr: int | None = None) -> None:
    """The norm's gradients: dx (dh, if any, added) and dw (float32), from h."""
    where, t = "tcu_rms_norm_grad", dy.dtype
    elem = _elem_code(where, t)
    L = _lib or lib()
    dev, (pdy, ph, pdh, pdx, pw, pdw, pwork) = _addresses(
        where, ((dy, t, rows, cols, lddy), (h, t, rows, cols, ldh), (dh, t, rows, cols, lddh),
                (dx, t, rows, cols, lddx)),
        ((w, t, cols), (dw, _F32, cols)), work, L.tcu_rms_norm_grad_work(rows, cols))
    _check(L.tcu_rms_norm_grad(pdy, lddy, ph, ldh, pw, pdh, lddh, pdx, lddx, pdw, pwork, rows,
                               cols, eps, elem, _stream_of(dev, stream_ptr)), where)


def tcu_adapter_work(M: int, K: int, N: int, r: int, G: int) -> int:
    """Bytes of work of the adapter calls (-1: a size out of range)."""
    return (_lib or lib()).tcu_adapter_work(M, K, N, r, G)


def _adapters(A, B, alpha, ids, t, M, K, N, r, G):
    """The adapters' operands as vectors."""
    return ((A, t, G * r * K), (B, t, G * N * r), (alpha, _F32, G), (ids, _I32, M))


def tcu_adapter_gemm(X, ldx: int, W, ldw: int, A, B, alpha, ids, Y, ldy: int, work, M: int, K: int,
                     N: int, r: int, G: int, stream_ptr: int | None = None) -> None:
    """Y[m] = X[m] @ W + alpha[g] * (X[m] @ A[g].T) @ B[g].T with g = ids[m] (no adapter
    outside [0, G)); A: G x r x K, B: G x N x r, alpha float32, ids int32."""
    where, t = "tcu_adapter_gemm", X.dtype
    dt = _dtype_code(t, Y.dtype, _POLY_DTYPES)
    _elem_code(where, t)
    L = _lib or lib()
    dev, (px, pw, py, pa, pb, pal, pid, pwork) = _addresses(
        where, ((X, t, M, K, ldx), (W, t, K, N, ldw), (Y, Y.dtype, M, N, ldy)),
        _adapters(A, B, alpha, ids, t, M, K, N, r, G), work, L.tcu_adapter_work(M, K, N, r, G))
    _check(L.tcu_adapter_gemm(px, ldx, pw, ldw, pa, pb, pal, pid, py, ldy, pwork, M, K, N, r, G,
                              dt, _stream_of(dev, stream_ptr)), where)


def tcu_adapter_gemm_q8(Xq, ldxq: int, xscale, Wq, ldwq: int, wscale, X, ldx: int, A, B, alpha,
                        ids, Y, ldy: int, work, M: int, K: int, N: int, r: int, G: int,
                        stream_ptr: int | None = None) -> None:
    """tcu_adapter_gemm with an 8-bit base: (Xq @ Wq) * xscale[:, None] * wscale; X, A,
    B and Y bfloat16."""
    where = "tcu_adapter_gemm_q8"
    _elem_code(where, Y.dtype)
    t = _BF16
    L = _lib or lib()
    dev, (pxq, pwq, px, py, pa, pb, pal, pid, pxs, pws, pwork) = _addresses(
        where, ((Xq, _I8, M, K, ldxq), (Wq, _I8, K, N, ldwq), (X, t, M, K, ldx),
                (Y, t, M, N, ldy)),
        _adapters(A, B, alpha, ids, t, M, K, N, r, G) + ((xscale, _F32, M), (wscale, _F32, N)),
        work, L.tcu_adapter_work(M, K, N, r, G))
    _check(L.tcu_adapter_gemm_q8(pxq, ldxq, pxs, pwq, ldwq, pws, px, ldx, pa, pb, pal, pid, py,
                                 ldy, pwork, M, K, N, r, G, _stream_of(dev, stream_ptr)), where)


def tcu_adapter_grad(X, ldx: int, dY, lddy: int, A, B, alpha, ids, dA, dB, work, M: int, K: int,
                     N: int, r: int, G: int, stream_ptr: int | None = None) -> None:
    """The adapters' gradients dA (G x r x K) and dB (G x N x r), float32."""
    where, t = "tcu_adapter_grad", X.dtype
    elem = _elem_code(where, t)
    L = _lib or lib()
    dev, (px, pdy, pa, pb, pal, pid, pda, pdb, pwork) = _addresses(
        where, ((X, t, M, K, ldx), (dY, t, M, N, lddy)),
        _adapters(A, B, alpha, ids, t, M, K, N, r, G) +
        ((dA, _F32, G * r * K), (dB, _F32, G * N * r)), work, L.tcu_adapter_work(M, K, N, r, G))
    _check(L.tcu_adapter_grad(px, ldx, pdy, lddy, pa, pb, pal, pid, pda, pdb, pwork, M, K, N, r, G,
                              elem, _stream_of(dev, stream_ptr)), where)


def tcu_adapter_input_grad(dY, lddy: int, Wt, ldwt: int, A, B, alpha, ids, dX, lddx: int, work,
                           M: int, K: int, N: int, r: int, G: int,
                           stream_ptr: int | None = None) -> None:
    """dX[m] = dY[m] @ Wt + alpha[g] * (dY[m] @ B[g]) @ A[g]; Wt: N x K."""
    where, t = "tcu_adapter_input_grad", dY.dtype
    dt = _dtype_code(t, dX.dtype, _POLY_DTYPES)
    _elem_code(where, t)
    L = _lib or lib()
    dev, (pdy, pw, pdx, pa, pb, pal, pid, pwork) = _addresses(
        where, ((dY, t, M, N, lddy), (Wt, t, N, K, ldwt), (dX, dX.dtype, M, K, lddx)),
        _adapters(A, B, alpha, ids, t, M, K, N, r, G), work, L.tcu_adapter_work(M, K, N, r, G))
    _check(L.tcu_adapter_input_grad(pdy, lddy, pw, ldwt, pa, pb, pal, pid, pdx, lddx, pwork, M, K,
                                    N, r, G, dt, _stream_of(dev, stream_ptr)), where)


def tcu_clip_grads_work() -> int:
    """Bytes of tcu_clip_grads' work."""
    return (_lib or lib()).tcu_clip_grads_work()


def tcu_clip_grads(grads, outs, max_norm: float, result, work,
                   stream_ptr: int | None = None) -> None:
    """outs[t] = grads[t] * min(1, max_norm / (norm + 1e-6)) with the norm over all tensors;
    result (2 float32): the norm and the factor.  Contiguous tensors of any shape,
    float32, float16 or bfloat16 each; outs[t] may be grads[t]."""
    where = "tcu_clip_grads"
    n = len(grads)
    if len(outs) != n:
        raise ValueError(f"{where}: {n} gradients and {len(outs)} outputs")
    _elem_code(where, result.dtype)
    L = _lib or lib()
    dev, (pres, pwork) = _addresses(where, (), ((result, _F32, 2),), work, L.tcu_clip_grads_work())
    # Each check in one pass over all tensors, and the tables as arrays (of lists: filled
    # in one go): with 48 tensors 19 us of the host's time, 31 a tensor at a time.
    import torch
    T = torch.Tensor
    types, counts = [g.dtype for g in grads], array.array("q", list(map(T.numel, grads)))
    try:
        if n and types.count(types[0]) == n:
            elems = array.array("i", (_ELEMS[types[0]],)) * n
        else:
            elems = array.array("i", [_ELEMS[t] for t in types])
    except KeyError as e:
        raise TcuError(TCU_ERR_UNSUPPORTED, f"{where}: element type {e.args[0]}") from None
    lists = (grads,)
    if outs is not grads:
        lists = (grads, outs)
        if [o.dtype for o in outs] != types or array.array("q", list(map(T.numel, outs))) != counts:
            raise ValueError(f"{where}: an output differs from its gradient in type or size")
    tables = []
    for ts in lists:
        if n and set(map(T.get_device, ts)) != {dev}:
            raise ValueError(f"{where}: all tensors must be on the same HIP device")
        if not all(map(T.is_contiguous, ts)):
            raise ValueError(f"{where}: tensors must be contiguous")
        tables.append(array.array("Q", list(map(T.data_ptr, ts))))
    _check(L.tcu_clip_grads(tables[0].buffer_info()[0], tables[-1].buffer_info()[0],
                            counts.buffer_info()[0], elems.buffer_info()[0], n, max_norm, pres,
                            pwork, _stream_of(dev, stream_ptr)), where)


# ------------------------------------------------------------- products in 4 bits
TCU_MAX_MX4_PITCH = 1 << 26
TCU_MAX_MX4_DIM = 1 << 27


def tcu_mx4_row_words(cols: int) -> int:
    """Scale words of a row of cols values in 4 bits (TCU_MX4_ROW_WORDS)."""
    return (cols + 127) // 128


def tcu_mx4_row_bytes(cols: int) -> int:
    """Bytes of codes of a row of cols values in 4 bits (TCU_MX4_ROW_BYTES)."""
    return 64 * tcu_mx4_row_words(cols)


def _mx4(q, ldq, scale, lds, rows, cols):
    """The views of a matrix in 4 bits: codes uint8, scales int32."""
    words = (cols + 127) // 128
    return (q, _U8, rows, 64 * words, ldq), (scale, _I32, words, rows, lds)


def tcu_mx4_quant(x, ldx: int, q, ldq: int, scale, lds: int, qt, ldqt: int, tscale, ldts: int,
                  rows: int, cols: int, stream_ptr: int | None = None) -> None:
    """x (rows x cols) in 4 bits along its rows (q: uint8, rows x tcu_mx4_row_bytes(cols);
    scale: int32, tcu_mx4_row_words(cols) x rows) and along its columns (qt, tscale: of
    x^T); either pair may be None."""
    where, t = "tcu_mx4_quant", x.dtype
    elem = _elem_code(where, t)
    if q is not None and scale is not None and qt is not None and tscale is not None:
        # everything as it should be: one flat condition (quantisation and back twice, 1003 x
        # 2005: 18.2 -> 16.7 us; a layer of one row: 6.8 -> 6.1)
        dev, g, h = x.get_device(), (cols + 127) // 128, (rows + 127) // 128
        if dev >= 0 and x.shape == (rows, cols) and x.stride() == (ldx, 1) and \
                q.shape == (rows, 64 * g) and q.stride() == (ldq, 1) and \
                scale.shape == (g, rows) and scale.stride() == (lds, 1) and \
                qt.shape == (cols, 64 * h) and qt.stride() == (ldqt, 1) and \
                tscale.shape == (h, cols) and tscale.stride() == (ldts, 1) and \
                q.dtype == qt.dtype == _U8 and scale.dtype == tscale.dtype == _I32 and \
                dev == q.get_device() == scale.get_device() == qt.get_device() == \
                tscale.get_device() == _current_device():
            _check((_lib or lib()).tcu_mx4_quant(
                x.data_ptr(), ldx, q.data_ptr(), ldq, scale.data_ptr(), lds, qt.data_ptr(), ldqt,
                tscale.data_ptr(), ldts, rows, cols, elem, _stream_of(dev, stream_ptr)), where)
            return
    dev, (px, pq, ps, pqt, pts) = _addresses(
        where, ((x, t, rows, cols, ldx),) + _mx4(q, ldq, scale, lds, rows, cols) +
        _mx4(qt, ldqt, tscale, ldts, cols, rows), (), None, 0)
    _check((_lib or lib()).tcu_mx4_quant(px, ldx, pq, ldq, ps, lds, pqt, ldqt, pts, ldts, rows,
                                         cols, elem, _stream_of(dev, stream_ptr)), where)


def tcu_mx4_dequant(q, ldq: int, scale, lds: int, y, ldy: int, rows: int, cols: int,
                    stream_ptr: int | None = None) -> None:
    """y (rows x cols) = the values that (q, scale) stands for."""
    where, t = "tcu_mx4_dequant", y.dtype
    elem = _elem_code(where, t)
    # as in tcu_mx4_quant
    dev, g = y.get_device(), (cols + 127) // 128
    if q is not None and scale is not None and dev >= 0 and y.shape == (rows, cols) and \
            y.stride() == (ldy, 1) and q.shape == (rows, 64 * g) and q.stride() == (ldq, 1) and \
            scale.shape == (g, rows) and scale.stride() == (lds, 1) and q.dtype == _U8 and \
            scale.dtype == _I32 and \
            dev == q.get_device() == scale.get_device() == _current_device():
        _check((_lib or lib()).tcu_mx4_dequant(q.data_ptr(), ldq, scale.data_ptr(), lds,
                                               y.data_ptr(), ldy, rows, cols, elem,
                                               _stream_of(dev, stream_ptr)), where)
        return
    dev, (py, pq, ps) = _addresses(
        where, ((y, t, rows, cols, ldy),) + _mx4(q, ldq, scale, lds, rows, cols), (), None, 0)
    _check((_lib or lib()).tcu_mx4_dequant(pq, ldq, ps, lds, py, ldy, rows, cols, elem,
                                           _stream_of(dev, stream_ptr)), where)


def tcu_mx4_work(M: int, K: int, N: int) -> int:
    """Bytes of work of tcu_mx4_gemm and tcu_mx4_linear (-1: a size out of range)."""
    return (_lib or lib()).tcu_mx4_work(M, K, N)


def tcu_mx4_gemm(A, lda: int, ascale, ldas: int, B, ldb: int, bscale, ldbs: int, C, ldc: int, work,
                 M: int, K: int, N: int, flags: int = 0, stream_ptr: int | None = None) -> None:
    """C (M x N) = [C +] A (M x K) @ B (N x K)^T, A and B in 4 bits."""
    where, t = "tcu_mx4_gemm", C.dtype
    elem = _elem_code(where, t)
    L = _lib or lib()
    # as in tcu_mx4_quant (a small layer's step, three calls of each: 42.9 -> 40.3 us)
    dev, g, nbytes = C.get_device(), (K + 127) // 128, L.tcu_mx4_work(M, K, N)
    if A is not None and ascale is not None and B is not None and bscale is not None and \
            work is not None and dev >= 0 and C.shape == (M, N) and C.stride() == (ldc, 1) and \
            A.shape == (M, 64 * g) and A.stride() == (lda, 1) and ascale.shape == (g, M) and \
            ascale.stride() == (ldas, 1) and B.shape == (N, 64 * g) and B.stride() == (ldb, 1) and \
            bscale.shape == (g, N) and bscale.stride() == (ldbs, 1) and \
            A.dtype == B.dtype == _U8 and ascale.dtype == bscale.dtype == _I32 and \
            work.is_contiguous() and 0 <= nbytes <= work.nbytes and \
            dev == A.get_device() == ascale.get_device() == B.get_device() == \
            bscale.get_device() == work.get_device() == _current_device():
        _check(L.tcu_mx4_gemm(A.data_ptr(), lda, ascale.data_ptr(), ldas, B.data_ptr(), ldb,
                              bscale.data_ptr(), ldbs, C.data_ptr(), ldc, work.data_ptr(), M, K, N,
                              flags, elem, _stream_of(dev, stream_ptr)), where)
        return
    dev, (pc, pa, pas, pb, pbs, *pwork) = _addresses(
        where, ((C, t, M, N, ldc),) + _mx4(A, lda, ascale, ldas, M, K) +
        _mx4(B, ldb, bscale, ldbs, N, K), (), work, nbytes)
    _check(L.tcu_mx4_gemm(pa, lda, pas, ldas, pb, ldb, pbs, ldbs, pc, ldc, *(pwork or (None,)), M,
                          K, N, flags, elem, _stream_of(dev, stream_ptr)), where)


def tcu_mx4_linear(X, ldx: int, W, ldw: int, wscale, ldws: int, Y, ldy: int, work, M: int, K: int,
                   N: int, flags: int = 0, stream_ptr: int | None = None) -> None:
    """Y (M x N) = [Y +] q(X) @ W^T: X (M x K) 16-bit, brought to 4 bits along its rows; W
    (N x K) in 4 bits; Y float32 or X's type."""
    where, t = "tcu_mx4_linear", X.dtype
    xelem, elem = _elem_code(where, t), _elem_code(where, Y.dtype)
    L = _lib or lib()
    # as in tcu_mx4_quant
    dev, g, nbytes = X.get_device(), (K + 127) // 128, L.tcu_mx4_work(M, K, N)
    if W is not None and wscale is not None and work is not None and dev >= 0 and \
            X.shape == (M, K) and X.stride() == (ldx, 1) and \
            Y.shape == (M, N) and Y.stride() == (ldy, 1) and W.shape == (N, 64 * g) and \
            W.stride() == (ldw, 1) and wscale.shape == (g, N) and wscale.stride() == (ldws, 1) and \
            W.dtype == _U8 and wscale.dtype == _I32 and work.is_contiguous() and \
            0 <= nbytes <= work.nbytes and dev == Y.get_device() == W.get_device() == \
            wscale.get_device() == work.get_device() == _current_device():
        _check(L.tcu_mx4_linear(X.data_ptr(), ldx, W.data_ptr(), ldw, wscale.data_ptr(), ldws,
                                Y.data_ptr(), ldy, work.data_ptr(), M, K, N, flags, xelem, elem,
                                _stream_of(dev, stream_ptr)), where)
        return
    dev, (px, py, pw, pws, *pwork) = _addresses(
        where, ((X, t, M, K, ldx), (Y, Y.dtype, M, N, ldy)) + _mx4(W, ldw, wscale, ldws, N, K),
        (), work, nbytes)
    _check(L.tcu_mx4_linear(px, ldx, pw, ldw, pws, ldws, py, ldy, *(pwork or (None,)), M, K, N,
                            flags, xelem, elem, _stream_of(dev, stream_ptr)), where)


# -------------------------------------------- norms of queries and keys with rotation
TCU_ROPE_ADJACENT = 1
TCU_MAX_HEAD_DIM = 1024
TCU_MAX_HEADS = 65536


def _heads(where, operands, dtype, vectors, work, nbytes):
    """Checks of operands (tensor, shape) of one type, any pitches of tokens and heads, and
    of vectors and work as _addresses.  Returns the device, three arguments for each
    operand and the vectors' addresses, work's last."""
    vdev, ptrs = _addresses(where, (), vectors, work, nbytes)
    out = []
    for t, shape in operands:
        if t is None:
            out += (None, 0, 0)
            continue
        ld, hd, one = t.stride() if t.dim() == 3 else (0, 0, 0)
        if t.dtype != dtype or t.shape != shape or one != 1 or t.get_device() != vdev:
            if t.get_device() != vdev:
                raise ValueError(f"{where}: all tensors must be on the same HIP device")
            if t.dtype != dtype:
                raise ValueError(f"{where}: expected {dtype}, got {t.dtype}")
            if t.shape != shape:
                raise ValueError(f"{where}: expected {shape}, got {tuple(t.shape)}")
            if shape[2] > 1 and t.numel():
                raise ValueError(f"{where}: strides {t.stride()} of heads that are not contiguous")
        out += (t.data_ptr() or None, ld, hd)
    return vdev, out, ptrs


def _qk_vectors(wq, wk, freq, pos, dtype, tokens, dim, rot):
    return ((wq, dtype, dim), (wk, dtype, dim), (freq, _F32, rot // 2), (pos, _I32, tokens))


def tcu_qk_norm(q, k, wq, wk, freq, pos, yq, yk, tokens: int, hq: int, hk: int, dim: int, rot: int,
                eps: float, flags: int = 0, stream_ptr: int | None = None) -> None:
    """Every head's RMS norm (weights wq and wk) with its first rot elements turned in pairs
    by the angles pos[t] * freq[i].  q and yq: tokens x hq x dim, k and yk: tokens x hk x
    dim, of any pitches of tokens and heads (the tensors' strides); yq may be q and yk k.
    freq: rot / 2 float32; pos: tokens int32; flags: 0 or TCU_ROPE_ADJACENT."""
    where = "tcu_qk_norm"
    t = (k if q is None else q).dtype
    elem = _elem_code(where, t)
    sq, sk = (tokens, hq, dim), (tokens, hk, dim)
    if rot and q is not None and k is not None and wq is not None and wk is not None and \
            freq is not None and pos is not None and yq is not None and yk is not None:
        # everything as it should be: one flat condition (a call 9.3 -> 8.2 us)
        a, b, c, d, dev = q.stride(), k.stride(), yq.stride(), yk.stride(), q.get_device()
        if dev >= 0 and q.shape == sq and yq.shape == sq and k.shape == sk and \
                yk.shape == sk and a[2] == b[2] == c[2] == d[2] == 1 and \
                t == k.dtype == yq.dtype == yk.dtype == wq.dtype == wk.dtype and \
                freq.dtype == _F32 and pos.dtype == _I32 and \
                dev == k.get_device() == yq.get_device() == yk.get_device() == \
                wq.get_device() == wk.get_device() == freq.get_device() == pos.get_device() and \
                wq.numel() == wk.numel() == dim and freq.numel() == rot // 2 and \
                pos.numel() == tokens and wq.is_contiguous() and wk.is_contiguous() and \
                freq.is_contiguous() and pos.is_contiguous() and dev == _current_device():
            _check((_lib or lib()).tcu_qk_norm(
                q.data_ptr(), a[0], a[1], k.data_ptr(), b[0], b[1], wq.data_ptr(), wk.data_ptr(),
                freq.data_ptr(), pos.data_ptr(), yq.data_ptr(), c[0], c[1], yk.data_ptr(), d[0],
                d[1], tokens, hq, hk, dim, rot, eps, flags, elem, _stream_of(dev, stream_ptr)),
                where)
            return
    dev, p, (pwq, pwk, pf, pp) = _heads(
        where, ((q, sq), (k, sk), (yq, sq), (yk, sk)), t,
        _qk_vectors(wq, wk, freq, pos, t, tokens, dim, rot), None, 0)
    _check((_lib or lib()).tcu_qk_norm(*p[:6], pwq, pwk, pf, pp, *p[6:], tokens, hq, hk, dim, rot,
                                       eps, flags, elem, _stream_of(dev, stream_ptr)), where)


def tcu_qk_norm_grad_work(tokens: int, hq: int, hk: int, dim: int) -> int:
    """Bytes of tcu_qk_norm_grad's work (-1: a size out of range)."""
    return (_lib or lib()).tcu_qk_norm_grad_work(tokens, hq, hk, dim)


def tcu_qk_norm_grad(dyq, dyk, q, k, wq, wk, freq, pos, dq, dk, dwq, dwk, work, tokens: int,
                     hq: int, hk: int, dim: int, rot: int, eps: float, flags: int = 0,
                     stream_ptr: int | None = None) -> None:
    """The gradients of tcu_qk_norm: dq and dk (shapes and type of q and k), dwq and dwk
    (dim float32 each), from the gradients dyq and dyk of its outputs."""
    where = "tcu_qk_norm_grad"
    t = (k if q is None else q).dtype
    elem = _elem_code(where, t)
    L = _lib or lib()
    sq, sk = (tokens, hq, dim), (tokens, hk, dim)
    nbytes = L.tcu_qk_norm_grad_work(tokens, hq, hk, dim)
    if rot and nbytes >= 0 and dyq is not None and dyk is not None and q is not None and \
            k is not None and wq is not None and wk is not None and freq is not None and \
            pos is not None and dq is not None and dk is not None and dwq is not None and \
            dwk is not None and work is not None:
        # as in tcu_qk_norm (a call 15.3 -> 13.7 us)
        a, b, c, d, dev = q.stride(), k.stride(), dyq.stride(), dyk.stride(), q.get_device()
        e, f = dq.stride(), dk.stride()
        if dev >= 0 and q.shape == sq and dyq.shape == sq and dq.shape == sq and \
                k.shape == sk and dyk.shape == sk and dk.shape == sk and \
                a[2] == b[2] == c[2] == d[2] == e[2] == f[2] == 1 and \
                t == k.dtype == dyq.dtype == dyk.dtype == dq.dtype == dk.dtype == wq.dtype == \
                wk.dtype and \
                freq.dtype == dwq.dtype == dwk.dtype == _F32 and pos.dtype == _I32 and \
                dev == k.get_device() == dyq.get_device() == dyk.get_device() == \
                dq.get_device() == dk.get_device() == wq.get_device() == wk.get_device() == \
                freq.get_device() == pos.get_device() == dwq.get_device() == \
                dwk.get_device() == work.get_device() and \
                wq.numel() == wk.numel() == dwq.numel() == dwk.numel() == dim and \
                freq.numel() == rot // 2 and pos.numel() == tokens and \
                work.numel() * work.element_size() >= nbytes and \
                wq.is_contiguous() and wk.is_contiguous() and dwq.is_contiguous() and \
                dwk.is_contiguous() and freq.is_contiguous() and pos.is_contiguous() and \
                work.is_contiguous() and dev == _current_device():
            _check(L.tcu_qk_norm_grad(
                dyq.data_ptr(), c[0], c[1], dyk.data_ptr(), d[0], d[1], q.data_ptr(), a[0], a[1],
                k.data_ptr(), b[0], b[1], wq.data_ptr(), wk.data_ptr(), freq.data_ptr(),
                pos.data_ptr(), dq.data_ptr(), e[0], e[1], dk.data_ptr(), f[0], f[1],
                dwq.data_ptr(), dwk.data_ptr(), work.data_ptr(), tokens, hq, hk, dim, rot, eps,
                flags, elem, _stream_of(dev, stream_ptr)), where)
            return
    dev, p, (pwq, pwk, pf, pp, pdwq, pdwk, *pwork) = _heads(
        where, ((dyq, sq), (dyk, sk), (q, sq), (k, sk), (dq, sq), (dk, sk)), t,
        _qk_vectors(wq, wk, freq, pos, t, tokens, dim, rot) + ((dwq, _F32, dim), (dwk, _F32, dim)),
        work, nbytes)
    _check(L.tcu_qk_norm_grad(*p[:12], pwq, pwk, pf, pp, *p[12:], pdwq, pdwk, *(pwork or (None,)),
                              tokens, hq, hk, dim, rot, eps, flags, elem,
                              _stream_of(dev, stream_ptr)), where)


# --------------------------------------------------------- cost accounting
def tcu_calls() -> int:
    return int(lib().tcu_calls())


def tcu_square_calls() -> int:
    return int(lib().tcu_square_calls())


def tcu_work() -> int:
    return int(lib().tcu_work())


def tcu_reset_calls() -> None:
    lib().tcu_reset_calls()


def tcu_strerror(status: int) -> str:
    return lib().tcu_strerror(int(status)).decode()


# ------------------------------------------- pointer checks, test overrides
def tcu_check_device_range(ptr: int, nbytes: int) -> int:
    """Status of the pointer check for [ptr, ptr + nbytes) (TCU_OK or a
    negative code; returned, not raised)."""
    return int(lib().tcu_check_device_range(ptr or None, int(nbytes)))


def tcu_set_knob(knob: int, value: int) -> None:
    _check(lib().tcu_set_knob(int(knob), int(value)), "tcu_set_knob")


def tcu_get_knob(knob: int) -> int:
    return int(lib().tcu_get_knob(int(knob)))

// C ABI of the operators of an adapted layer: argument validation, cost
// accounting and dispatch to the HIP launchers.  Every argument check runs
// before the first HIP call of an entry point.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <vector>

#include "tcu.h"
#include "tcu_host.h"
#include "tcu_layer.h"
#include "tcu_operand.h"

#define TCU_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using namespace tcu;

// Whether sizes are in range: the operands of M rows, a byte a value at least,
// and G * r * max(K, N) 16-bit values among them.
int check_sizes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G) {
  if (!dim_ok(M) || K < 0 || N < 0 || K > TCU_MAX_ADAPTED_DIM || N > TCU_MAX_ADAPTED_DIM ||
      G < 0 || G > TCU_MAX_ADAPTERS || r < 1 || r > TCU_MAX_RANK)
    return TCU_ERR_SHAPE;
  if (M * std::max(K, N) >= kMaxExtent) return TCU_ERR_SHAPE;
  if (G * r * std::max(K, N) >= kMaxExtent / 4) return TCU_ERR_SHAPE;
  return adapter_work_bytes(M, K, N, r, G) < kMaxExtent ? TCU_OK : TCU_ERR_SHAPE;
}

bool adapter_dtype_ok(int dt) {
  return dt == TCU_F16_F32 || dt == TCU_BF16_F32 || dt == TCU_BF16_BF16;
}

int adapter_product(int dtype, const AdapterArgs &a, bool input_grad, hipStream_t stream) {
  const int64_t M = a.M, K = a.K, N = a.N, r = a.r, G = a.G;
  const bool q8 = dtype == TCU_I8_I32;
  // int32 sums of K products of magnitude <= 2^14 stay exact while K < 2^17.
  if (q8 && K >= ((int64_t)1 << 17)) return TCU_ERR_SHAPE;
  const int64_t ob = dtype == TCU_F16_F32 || dtype == TCU_BF16_F32 ? 4 : 2, ib = q8 ? 1 : 2;
  const int64_t xk = q8 && G == 0 ? 0 : K;
  const Operand ops[] = {
      Operand{a.Y, M, N, a.ldy, ob, 16, true},
      vec(a.work, M > 0 && N > 0 ? adapter_work_bytes(M, K, N, r, G) : 0, 1, 16, true),
      Operand{a.X, M, xk, a.ldx, 2}, Operand{a.W, K, N, a.ldw, ib},
      Operand{a.Xq, M, q8 ? K : 0, a.ldxq, 1}, vec(a.xscale, q8 ? M : 0, 4, 4),
      vec(a.wscale, q8 ? N : 0, 4, 4), vec(a.A, G * r * (input_grad ? N : K), 2, 16),
      vec(a.B, G * r * (input_grad ? K : N), 2, 16), vec(a.alpha, G, 4, 4),
      vec(a.ids, G > 0 ? M : 0, 4, 4)};
  int rc = check_operands(ops);
  if (rc != TCU_OK) return rc;
  if (M == 0 || N == 0) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const hipError_t e = input_grad ? launch_adapter_input_grad(dtype, a, stream, num_cus)
                                  : launch_adapter(dtype, a, stream, num_cus);
  if (e != hipSuccess) return TCU_ERR_HIP;
  const int s = unit_size();
  count_tall(blocks(K, s) * blocks(N, s) + (G > 0 ? (blocks(K, s) + blocks(N, s)) * blocks(r, s) : 0),
             M, s);
  return TCU_OK;
}

}  // namespace

TCU_EXPORT int tcu_rms_norm(const void *x, int64_t ldx, const void *res, int64_t ldr,
                            const void *w, void *h, int64_t ldh, void *y, int64_t ldy, void *q,
                            int64_t ldq, float *qscale, int64_t rows, int64_t cols, float eps,
                            int elem, void *hip_stream) {
  if (!elem_ok(elem)) return TCU_ERR_UNSUPPORTED;
  if (!dim_ok(rows) || !dim_ok(cols) || cols < 1 || !(eps >= 0.f) || std::isinf(eps))
    return TCU_ERR_SHAPE;
  if (!x && rows > 0) return TCU_ERR_NULL;
  if ((q != nullptr) != (qscale != nullptr) && rows > 0) return TCU_ERR_NULL;
  const int64_t es = elem_size(elem);
  const Operand ops[] = {
      Operand{h, h ? rows : 0, cols, ldh, es, 16, true},
      Operand{y, y ? rows : 0, cols, ldy, es, 16, true},
      Operand{q, q ? rows : 0, cols, ldq, 1, 16, true},
      Operand{qscale, 1, q ? rows : 0, rows, 4, 4, true},
      Operand{x, rows, cols, ldx, es}, Operand{res, res ? rows : 0, cols, ldr, es},
      vec(w, rows > 0 ? cols : 0, es, 16)};
  int rc = check_operands(ops, {{0, 4}, {0, 5}});
  if (rc != TCU_OK) return rc;
  if (rows == 0 || (!h && !y && !q)) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const NormArgs a{x, res, w, h, y, q, qscale, ldx, ldr, ldh, ldy, ldq, rows, cols, eps};
  return launch_rms_norm(elem, a, (hipStream_t)hip_stream, num_cus) == hipSuccess ? TCU_OK
                                                                                   : TCU_ERR_HIP;
}

TCU_EXPORT int64_t tcu_rms_norm_grad_work(int64_t rows, int64_t cols) {
  if (!dim_ok(rows) || !dim_ok(cols) || cols < 1) return -1;
  return std::min<int64_t>(std::max<int64_t>(rows, 1), kNormParts) * cols * 4;
}

TCU_EXPORT int tcu_rms_norm_grad(const void *dy, int64_t lddy, const void *h, int64_t ldh,
                                 const void *w, const void *dh, int64_t lddh, void *dx,
                                 int64_t lddx, float *dw, void *work, int64_t rows, int64_t cols,
                                 float eps, int elem, void *hip_stream) {
  if (!elem_ok(elem)) return TCU_ERR_UNSUPPORTED;
  if (!dim_ok(rows) || !dim_ok(cols) || cols < 1 || !(eps >= 0.f) || std::isinf(eps))
    return TCU_ERR_SHAPE;
  const int64_t es = elem_size(elem);
  const Operand ops[] = {
      Operand{dx, rows, cols, lddx, es, 16, true}, vec(dw, cols, 4, 4, true),
      vec(work, rows > 0 ? tcu_rms_norm_grad_work(rows, cols) : 0, 1, 16, true),
      Operand{dy, rows, cols, lddy, es}, Operand{h, rows, cols, ldh, es},
      vec(w, rows > 0 ? cols : 0, es, 16), Operand{dh, dh ? rows : 0, cols, lddh, es}};
  int rc = check_operands(ops, {{0, 3}, {0, 6}});
  if (rc != TCU_OK) return rc;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const NormGradArgs a{dy, h, w, dh, dx, dw, (float *)work, lddy, ldh, lddh, lddx, rows, cols, eps};
  return launch_rms_norm_grad(elem, a, (hipStream_t)hip_stream, num_cus) == hipSuccess
             ? TCU_OK
             : TCU_ERR_HIP;
}

TCU_EXPORT int64_t tcu_adapter_work(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G) {
  return check_sizes(M, K, N, r, G) == TCU_OK ? adapter_work_bytes(M, K, N, r, G) : -1;
}

TCU_EXPORT int tcu_adapter_gemm(const void *X, int64_t ldx, const void *W, int64_t ldw,
                                const void *A, const void *B, const float *alpha,
                                const int32_t *ids, void *Y, int64_t ldy, void *work, int64_t M,
                                int64_t K, int64_t N, int64_t r, int64_t G, int dtype,
                                void *hip_stream) {
  if (!adapter_dtype_ok(dtype)) return TCU_ERR_UNSUPPORTED;
  const int rc = check_sizes(M, K, N, r, G);
  if (rc != TCU_OK) return rc;
  const AdapterArgs a{X,   W, A, B, nullptr, nullptr, nullptr, alpha, ids, Y, work,
                      ldx, 0, ldw, ldy, M, K, N, r, G};
  return adapter_product(dtype, a, false, (hipStream_t)hip_stream);
}

TCU_EXPORT int tcu_adapter_gemm_q8(const void *Xq, int64_t ldxq, const float *xscale,
                                   const void *Wq, int64_t ldwq, const float *wscale,
                                   const void *X, int64_t ldx, const void *A, const void *B,
                                   const float *alpha, const int32_t *ids, void *Y, int64_t ldy,
                                   void *work, int64_t M, int64_t K, int64_t N, int64_t r,
                                   int64_t G, void *hip_stream) {
  const int rc = check_sizes(M, K, N, r, G);
  if (rc != TCU_OK) return rc;
  const AdapterArgs a{X,   Wq,   A, B, Xq, xscale, wscale, alpha, ids, Y, work,
                      ldx, ldxq, ldwq, ldy, M, K, N, r, G};
  return adapter_product(TCU_I8_I32, a, false, (hipStream_t)hip_stream);
}

TCU_EXPORT int tcu_adapter_input_grad(const void *dY, int64_t lddy, const void *Wt, int64_t ldwt,
                                      const void *A, const void *B, const float *alpha,
                                      const int32_t *ids, void *dX, int64_t lddx, void *work,
                                      int64_t M, int64_t K, int64_t N, int64_t r, int64_t G,
                                      int dtype, void *hip_stream) {
  if (!adapter_dtype_ok(dtype)) return TCU_ERR_UNSUPPORTED;
  const int rc = check_sizes(M, K, N, r, G);
  if (rc != TCU_OK) return rc;
  // the product dY Wt: contracted index N, K columns
  const AdapterArgs a{dY,   Wt, A, B, nullptr, nullptr, nullptr, alpha, ids, dX, work,
                      lddy, 0, ldwt, lddx, M, N, K, r, G};
  return adapter_product(dtype, a, true, (hipStream_t)hip_stream);
}

TCU_EXPORT int tcu_adapter_grad(const void *X, int64_t ldx, const void *dY, int64_t lddy,
                                const void *A, const void *B, const float *alpha,
                                const int32_t *ids, float *dA, float *dB, void *work, int64_t M,
                                int64_t K, int64_t N, int64_t r, int64_t G, int elem,
                                void *hip_stream) {
  if (elem != TCU_ELEM_F16 && elem != TCU_ELEM_BF16) return TCU_ERR_UNSUPPORTED;
  int rc = check_sizes(M, K, N, r, G);
  if (rc != TCU_OK) return rc;
  if (K < 1 || N < 1) return TCU_ERR_SHAPE;
  const Operand ops[] = {
      vec(dA, G * r * K, 4, 16, true), vec(dB, G * N * r, 4, 16, true),
      vec(work, G > 0 ? adapter_work_bytes(M, K, N, r, G) : 0, 1, 16, true),
      Operand{X, G > 0 ? M : 0, K, ldx, 2}, Operand{dY, G > 0 ? M : 0, N, lddy, 2},
      vec(A, G * r * K, 2, 16), vec(B, G * N * r, 2, 16), vec(alpha, G, 4, 4),
      vec(ids, G > 0 ? M : 0, 4, 4)};
  rc = check_operands(ops);
  if (rc != TCU_OK) return rc;
  if (G == 0) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const AdapterGradArgs a{X, dY, A, B, alpha, ids, dA, dB, work, ldx, lddy, M, K, N, r, G};
  if (launch_adapter_grad(elem, a, (hipStream_t)hip_stream, num_cus) != hipSuccess)
    return TCU_ERR_HIP;
  const int s = unit_size();
  if (M > 0) count_tall(2 * (blocks(K, s) + blocks(N, s)) * blocks(r, s), M, s);
  return TCU_OK;
}

TCU_EXPORT int64_t tcu_clip_grads_work(void) { return clip_work_bytes(); }

TCU_EXPORT int tcu_clip_grads(const void *const *grads, void *const *outs, const int64_t *counts,
                              const int32_t *elems, int64_t tensors, float max_norm,
                              float *result, void *work, void *hip_stream) {
  if (tensors < 0 || tensors > ((int64_t)1 << 20) || !(max_norm >= 0.f)) return TCU_ERR_SHAPE;
  if (!result || !work || (tensors > 0 && (!grads || !outs || !counts || !elems)))
    return TCU_ERR_NULL;
  struct Range {
    uintptr_t begin, end;
    int64_t tensor;   // -1: result or work
    bool out;
  };
  std::vector<Range> ranges;
  try {
    ranges.reserve(2 * (size_t)tensors + 2);
  } catch (const std::bad_alloc &) {
    return TCU_ERR_SHAPE;
  }
  for (int64_t t = 0; t < tensors; ++t) {
    if (!elem_ok(elems[t])) return TCU_ERR_UNSUPPORTED;
    const int64_t es = elem_size(elems[t]), n = counts[t];
    if (n < 0 || n >= kMaxExtent / es) return TCU_ERR_SHAPE;
    if (n == 0) continue;
    if (!grads[t] || !outs[t]) return TCU_ERR_NULL;
    const uintptr_t g = reinterpret_cast<uintptr_t>(grads[t]),
                    o = reinterpret_cast<uintptr_t>(outs[t]);
    if (((g | o) & (uintptr_t)(es - 1)) != 0) return TCU_ERR_ALIGN;
    if (g != o) ranges.push_back({g, g + (uintptr_t)(n * es), t, false});
    ranges.push_back({o, o + (uintptr_t)(n * es), t, true});
  }
  if ((reinterpret_cast<uintptr_t>(result) & 3) != 0 || misaligned(work)) return TCU_ERR_ALIGN;
  const uintptr_t rp = reinterpret_cast<uintptr_t>(result), wp = reinterpret_cast<uintptr_t>(work);
  ranges.push_back({rp, rp + 8, -1, true});
  ranges.push_back({wp, wp + (uintptr_t)clip_work_bytes(), -1, true});
  // In the order of their bases an output must end before everything after it
  // begins, and begin after everything before it has ended.  Inputs may share
  // bytes with inputs.
  std::sort(ranges.begin(), ranges.end(),
            [](const Range &a, const Range &b) { return a.begin < b.begin; });
  uintptr_t any_end = 0, out_end = 0;
  for (const Range &r : ranges) {
    if (r.begin < out_end || (r.out && r.begin < any_end)) return TCU_ERR_OVERLAP;
    any_end = std::max(any_end, r.end);
    if (r.out) out_end = std::max(out_end, r.end);
  }
  int num_cus = 0;
  int rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  if (checks_on()) {
    for (const Range &r : ranges) {
      rc = device_range(reinterpret_cast<const void *>(r.begin), (int64_t)(r.end - r.begin));
      if (rc != TCU_OK) return rc;
    }
  }
  return launch_clip(grads, outs, counts, elems, tensors, max_norm, result, work,
                     (hipStream_t)hip_stream, num_cus) == hipSuccess
             ? TCU_OK
             : TCU_ERR_HIP;
}

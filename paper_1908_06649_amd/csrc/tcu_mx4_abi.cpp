// C ABI of the products in 4 bits: argument validation, cost accounting and dispatch
// to the HIP launchers.  Every argument check runs before the first HIP call of an
// entry point.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "tcu.h"
#include "tcu_host.h"
#include "tcu_mx4.h"
#include "tcu_operand.h"

#define TCU_EXPORT extern "C" __attribute__((visibility("default")))

namespace {

using namespace tcu;

bool mx4_dim_ok(int64_t n) { return n >= 0 && n <= TCU_MAX_MX4_DIM; }

// A matrix in 4 bits: its codes and its scales.
Operand codes(const void *p, int64_t rows, int64_t cols, int64_t ld, bool out = false) {
  return Operand{p, rows, mx4_row_bytes(cols), ld, 1, 16, out};
}
Operand scales(const void *p, int64_t rows, int64_t cols, int64_t ld, bool out = false) {
  return Operand{p, cols > 0 ? mx4_groups(cols) : 0, rows, ld, 4, 4, out};
}
// The pitch of codes that check_operands does not look at.
int check_pitch(int64_t rows, int64_t cols, int64_t ld) {
  if (rows <= 1 || cols == 0) return TCU_OK;
  if (ld > TCU_MAX_MX4_PITCH) return TCU_ERR_SHAPE;
  return ld % 16 == 0 ? TCU_OK : TCU_ERR_ALIGN;
}

int sizes_ok(int64_t M, int64_t K, int64_t N) {
  if (!mx4_dim_ok(M) || !mx4_dim_ok(K) || !mx4_dim_ok(N)) return TCU_ERR_SHAPE;
  return mx4_work_bytes(M, K, N) < kMaxExtent ? TCU_OK : TCU_ERR_SHAPE;
}

// The product with the checks that both entry points share: X a 16-bit left operand,
// or null.
int product(const void *X, int64_t ldx, int xelem, const Mx4GemmArgs &a, int elem, bool linear,
            hipStream_t stream) {
  const int64_t M = a.M, K = a.K, N = a.N;
  const bool any = M > 0 && N > 0;
  const int64_t ka = any && !linear ? K : 0, kb = any ? K : 0, es = elem_size(elem);
  const Operand ops[] = {
      Operand{a.C, M, N, a.ldc, es, 16, true},
      vec(a.work, any ? mx4_work_bytes(M, K, N) : 0, 1, 16, true),
      Operand{X, linear ? M : 0, kb, ldx, 2}, codes(a.A, M, ka, a.lda), scales(a.as, M, ka, a.ldas),
      codes(a.B, N, kb, a.ldb), scales(a.bs, N, kb, a.ldbs)};
  int rc = check_operands(ops);
  if (rc == TCU_OK) rc = check_pitch(M, ka, a.lda);
  if (rc == TCU_OK) rc = check_pitch(N, kb, a.ldb);
  if (rc != TCU_OK) return rc;
  if (!any || (K == 0 && a.accum)) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const hipError_t e = linear ? launch_mx4_linear(xelem, X, ldx, elem, a, stream, num_cus)
                              : launch_mx4_gemm(elem, a, stream, num_cus);
  if (e != hipSuccess) return TCU_ERR_HIP;
  const int s = unit_size();
  if (K > 0) count_tall(blocks(K, s) * blocks(N, s), M, s);
  return TCU_OK;
}

}  // namespace

TCU_EXPORT int tcu_mx4_quant(const void *x, int64_t ldx, void *q, int64_t ldq, uint32_t *scale,
                             int64_t lds, void *qt, int64_t ldqt, uint32_t *tscale, int64_t ldts,
                             int64_t rows, int64_t cols, int elem, void *hip_stream) {
  if (!elem_ok(elem)) return TCU_ERR_UNSUPPORTED;
  if (!mx4_dim_ok(rows) || !mx4_dim_ok(cols)) return TCU_ERR_SHAPE;
  const bool any = rows > 0 && cols > 0;
  if (any && ((q != nullptr) != (scale != nullptr) || (qt != nullptr) != (tscale != nullptr)))
    return TCU_ERR_NULL;
  const int64_t along = any && q ? rows : 0, across = any && qt ? cols : 0;
  const Operand ops[] = {codes(q, along, cols, ldq, true), scales(scale, along, cols, lds, true),
                         codes(qt, across, rows, ldqt, true),
                         scales(tscale, across, rows, ldts, true),
                         Operand{x, rows, cols, ldx, elem_size(elem)}};
  int rc = check_operands(ops);
  if (rc == TCU_OK) rc = check_pitch(along, cols, ldq);
  if (rc == TCU_OK) rc = check_pitch(across, rows, ldqt);
  if (rc != TCU_OK) return rc;
  if (along == 0 && across == 0) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const Mx4QuantArgs a{x, (unsigned char *)q, (unsigned char *)qt, scale, tscale, ldx,
                       ldq, lds, ldqt, ldts, rows, cols};
  return launch_mx4_quant(elem, a, (hipStream_t)hip_stream) == hipSuccess ? TCU_OK : TCU_ERR_HIP;
}

TCU_EXPORT int tcu_mx4_dequant(const void *q, int64_t ldq, const uint32_t *scale, int64_t lds,
                               void *y, int64_t ldy, int64_t rows, int64_t cols, int elem,
                               void *hip_stream) {
  if (!elem_ok(elem)) return TCU_ERR_UNSUPPORTED;
  if (!mx4_dim_ok(rows) || !mx4_dim_ok(cols)) return TCU_ERR_SHAPE;
  const bool any = rows > 0 && cols > 0;
  const Operand ops[] = {Operand{y, rows, cols, ldy, elem_size(elem), 16, true},
                         codes(q, any ? rows : 0, cols, ldq),
                         scales(scale, any ? rows : 0, cols, lds)};
  int rc = check_operands(ops);
  if (rc == TCU_OK) rc = check_pitch(rows, cols, ldq);
  if (rc != TCU_OK) return rc;
  if (!any) return TCU_OK;
  int num_cus = 0;
  rc = device_ready(&num_cus);
  if (rc != TCU_OK) return rc;
  rc = check_device(ops);
  if (rc != TCU_OK) return rc;
  const Mx4DequantArgs a{(const unsigned char *)q, scale, y, ldq, lds, ldy, rows, cols};
  return launch_mx4_dequant(elem, a, (hipStream_t)hip_stream) == hipSuccess ? TCU_OK : TCU_ERR_HIP;
}

TCU_EXPORT int64_t tcu_mx4_work(int64_t M, int64_t K, int64_t N) {
  return sizes_ok(M, K, N) == TCU_OK ? mx4_work_bytes(M, K, N) : -1;
}

TCU_EXPORT int tcu_mx4_gemm(const void *A, int64_t lda, const uint32_t *ascale, int64_t ldas,
                            const void *B, int64_t ldb, const uint32_t *bscale, int64_t ldbs,
                            void *C, int64_t ldc, void *work, int64_t M, int64_t K, int64_t N,
                            int flags, int elem, void *hip_stream) {
  if (!elem_ok(elem) || (flags & ~TCU_ACCUMULATE) != 0) return TCU_ERR_UNSUPPORTED;
  const int rc = sizes_ok(M, K, N);
  if (rc != TCU_OK) return rc;
  const Mx4GemmArgs a{(const unsigned char *)A, (const unsigned char *)B, ascale, bscale, C, work,
                      lda, ldas, ldb, ldbs, ldc, M, K, N, (flags & TCU_ACCUMULATE) != 0};
  return product(nullptr, 0, 0, a, elem, false, (hipStream_t)hip_stream);
}

TCU_EXPORT int tcu_mx4_linear(const void *X, int64_t ldx, const void *W, int64_t ldw,
                              const uint32_t *wscale, int64_t ldws, void *Y, int64_t ldy,
                              void *work, int64_t M, int64_t K, int64_t N, int flags, int xelem,
                              int elem, void *hip_stream) {
  if ((xelem != TCU_ELEM_F16 && xelem != TCU_ELEM_BF16) ||
      (elem != TCU_ELEM_F32 && elem != xelem) || (flags & ~TCU_ACCUMULATE) != 0)
    return TCU_ERR_UNSUPPORTED;
  const int rc = sizes_ok(M, K, N);
  if (rc != TCU_OK) return rc;
  const Mx4GemmArgs a{nullptr, (const unsigned char *)W, nullptr, wscale, Y, work,
                      0, 0, ldw, ldws, ldy, M, K, N, (flags & TCU_ACCUMULATE) != 0};
  return product(X, ldx, xelem, a, elem, true, (hipStream_t)hip_stream);
}

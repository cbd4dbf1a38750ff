// Internal launchers of the products in 4 bits (host side), and the sizes of what
// they take.  Arguments are already validated by tcu_mx4_abi.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tcu.h"

namespace tcu {

// A row of n values in 4 bits: whole groups of 128 (64 bytes of codes, one word of
// four scales).
__host__ __device__ constexpr int64_t mx4_groups(int64_t n) { return (n + 127) / 128; }
constexpr int64_t mx4_row_bytes(int64_t n) { return 64 * mx4_groups(n); }

struct Mx4QuantArgs {
  const void *x;
  unsigned char *q, *qt;     // null: not written
  unsigned *s, *ts;
  int64_t ldx, ldq, lds, ldqt, ldts, rows, cols;
};
hipError_t launch_mx4_quant(int elem, const Mx4QuantArgs &a, hipStream_t stream);

struct Mx4DequantArgs {
  const unsigned char *q;
  const unsigned *s;
  void *y;
  int64_t ldq, lds, ldy, rows, cols;
};
hipError_t launch_mx4_dequant(int elem, const Mx4DequantArgs &a, hipStream_t stream);

// C (M x N) = [C +] A (M x K) B (N x K)^T, both in 4 bits.
struct Mx4GemmArgs {
  const unsigned char *A, *B;
  const unsigned *as, *bs;
  void *C;
  void *work;
  int64_t lda, ldas, ldb, ldbs, ldc, M, K, N;
  bool accum;
};
hipError_t launch_mx4_gemm(int elem, const Mx4GemmArgs &a, hipStream_t stream, int num_cus);
// The same with a 16-bit left operand X (TCU_ELEM_F16 or TCU_ELEM_BF16), brought to
// 4 bits here; a.A and a.as are not read.
hipError_t launch_mx4_linear(int xelem, const void *X, int64_t ldx, int elem,
                             const Mx4GemmArgs &a, hipStream_t stream, int num_cus);
int64_t mx4_work_bytes(int64_t M, int64_t K, int64_t N);

}  // namespace tcu

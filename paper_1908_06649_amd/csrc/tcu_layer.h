// Internal launchers of the operators of an adapted layer (host side).
// Arguments are already validated by tcu_layer_abi.cpp.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tcu.h"

namespace tcu {

// Workgroups of a norm gradient, each with its rows' sum of the weights' gradients,
// which norm_dw_kernel adds: two a compute unit (us, bf16, 256 / 512 / 1024: 6007 x 4100
// 45.2 / 38.3 / 42.6, 2000 x 2048 15.5 / 13.3 / 15.3, 6007 x 8192 77.8 / 78.9 / 87.1;
// long rows have fewer, 2000 x 16384 54.6 / 60.8 / 81.3).
constexpr int kNormParts = 512;

struct NormArgs {
  const void *x, *res, *w;
  void *h, *y, *q;
  float *qscale;
  int64_t ldx, ldr, ldh, ldy, ldq, rows, cols;
  float eps;
};
hipError_t launch_rms_norm(int elem, const NormArgs &a, hipStream_t stream, int num_cus);

struct NormGradArgs {
  const void *dy, *h, *w, *dh;
  void *dx;
  float *dw, *work;
  int64_t lddy, ldh, lddh, lddx, rows, cols;
  float eps;
};
hipError_t launch_rms_norm_grad(int elem, const NormGradArgs &a, hipStream_t stream, int num_cus);

struct AdapterArgs {
  const void *X, *W, *A, *B;       // X of the adapters; W 16-bit or int8
  const void *Xq;                  // int8 left operand (null: X is it)
  const float *xscale, *wscale;    // of the 8-bit base
  const float *alpha;
  const int32_t *ids;
  void *Y;
  void *work;
  int64_t ldx, ldxq, ldw, ldy, M, K, N, r, G;
};
// dtype: the product's (TCU_I8_I32: the 8-bit base with bfloat16 Y).
hipError_t launch_adapter(int dtype, const AdapterArgs &a, hipStream_t stream, int num_cus);

struct AdapterGradArgs {
  const void *X, *dY, *A, *B;
  const float *alpha;
  const int32_t *ids;
  float *dA, *dB;
  void *work;
  int64_t ldx, lddy, M, K, N, r, G;
};
hipError_t launch_adapter_grad(int elem, const AdapterGradArgs &a, hipStream_t stream,
                               int num_cus);
// a: dY as X, Wt as W, with A and B as the caller holds them and K and N of
// the product dY Wt (its contracted index and columns).
hipError_t launch_adapter_input_grad(int dtype, const AdapterArgs &a, hipStream_t stream,
                                     int num_cus);
// The same for few rows (see tcu_few.hip), with work of few_work_bytes; the
// sizes it takes, by few_ok, and its time in microseconds.
constexpr int64_t kFewBlock = 64, kFewRows = 256;
bool few_ok(int dtype, const AdapterArgs &a);
double few_us(const AdapterArgs &a, bool q8);
double few_narrow_us(const AdapterArgs &a, bool q8);
// T: the narrow product, rows of tld values, or null: it is formed there too.
hipError_t launch_few(int dtype, const AdapterArgs &a, float *T, int tld, hipStream_t stream);
int64_t few_work_bytes(int64_t M, int64_t K, int64_t N, int64_t r);
int64_t adapter_work_bytes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G);

hipError_t launch_clip(const void *const *grads, void *const *outs, const int64_t *counts,
                       const int32_t *elems, int64_t tensors, float max_norm, float *result,
                       void *work, hipStream_t stream, int num_cus);
int64_t clip_work_bytes();

}  // namespace tcu

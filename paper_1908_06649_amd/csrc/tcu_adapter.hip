// Low-rank adapters of many requests beside a shared projection, and their
// gradients (tcu_adapter_gemm, tcu_adapter_gemm_q8, tcu_adapter_grad,
// tcu_adapter_input_grad).
//
//   Y[m] = X[m] W + alpha[g] (X[m] A_g^T) B_g^T,  g = ids[m]
//   dA_g = sum_m alpha[g] (dY[m] B_g)^T X[m],  dB_g = sum_m alpha[g] dY[m]^T (X[m] A_g^T)
//
// The projection is the blocked product (launch_rect) into scratch, the
// narrow product T = alpha X A^T is formed a row per wave, and a last pass adds
// T B^T and rounds.
#include "tcu_elem.h"
#include "tcu_launch.h"
#include "tcu_layer.h"

namespace tcu {
namespace {

constexpr int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

// Scratch: the projection's sums, T of X and of dY, the adapters transposed.
struct Scratch {
  unsigned char *base;
  float *t, *dt;
  unsigned char *at, *bt;
  int64_t bytes;
};
Scratch scratch(void *work, int64_t M, int64_t K, int64_t N, int64_t r, int64_t G) {
  Scratch s;
  int64_t at = 0;
  auto take = [&](int64_t n) {
    unsigned char *p = (unsigned char *)work + at;
    at += round256(n);
    return p;
  };
  s.base = take(M * (N > K ? N : K) * 4);
  s.t = (float *)take(M * r * 4);
  s.dt = (float *)take(M * r * 4);
  s.at = take(G * r * K * 2);
  s.bt = take(G * r * N * 2);
  s.bytes = at;
  return s;
}

// T[m][j] = alpha[g] sum_k X[m][k] F_g(j, k), zeros without an adapter; F_g(j, k)
// lies at F + g r K + j fj + k fk.  A wave per row.
template <int ELEM>
__global__ __launch_bounds__(256) void narrow_kernel(const unsigned char *__restrict__ X,
                                                     int64_t ldx,
                                                     const unsigned char *__restrict__ F,
                                                     int64_t fj, int64_t fk,
                                                     const float *__restrict__ alpha,
                                                     const int *__restrict__ ids,
                                                     float *__restrict__ T, int64_t M, int64_t K,
                                                     int r, int G) {
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)gridDim.x * 4;
  for (int64_t m = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); m < M; m += step) {
    const int g = ids[m];
    const bool has = g >= 0 && g < G;
    for (int j = 0; j < r; ++j) {
      float s = 0.f;
      if (has) {
        const unsigned char *f = F + 2 * ((int64_t)g * r * K + j * fj);
        for (int64_t k = lane; k < K; k += 64)
          s += elem_to_f32<ELEM>(X + 2 * (m * ldx + k)) * elem_to_f32<ELEM>(f + 2 * k * fk);
        s = wave_sum(s) * alpha[g];
      }
      if (lane == 0) T[m * r + j] = s;
    }
  }
}

// Y = base (scaled, 8-bit) + T B^T, rounded once.
template <int ELEM, int OUT, bool kQ8>
__global__ __launch_bounds__(256) void join_kernel(AdapterArgs a, const void *base,
                                                   const float *__restrict__ T) {
  const int64_t total = a.M * a.N;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int64_t m = i / a.N, n = i - m * a.N;
    float v = kQ8 ? (float)((const int *)base)[i] * a.xscale[m] * a.wscale[n]
                  : ((const float *)base)[i];
    const int g = a.G > 0 ? a.ids[m] : -1;
    if (g >= 0 && g < a.G) {
      const unsigned char *b = (const unsigned char *)a.B + 2 * (((int64_t)g * a.N + n) * a.r);
      for (int j = 0; j < a.r; ++j) v += T[m * a.r + j] * elem_to_f32<ELEM>(b + 2 * j);
    }
    f32_to_elem<OUT>((unsigned char *)a.Y + (m * a.ldy + n) * elem_bytes<OUT>, v);
  }
}

// out (cols x rows) of every adapter = in (rows x cols), 16-bit values.
__global__ __launch_bounds__(256) void transpose_kernel(const unsigned short *__restrict__ in,
                                                        unsigned short *__restrict__ out,
                                                        int64_t rows, int64_t cols, int64_t total) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int64_t g = i / (rows * cols), e = i - g * rows * cols;
    const int64_t c = e / rows, r = e - c * rows;
    out[i] = in[g * rows * cols + r * cols + c];
  }
}

// D_g(j, c) = sum over g's rows of T[m][j] X[m][c], at D + g r C + j dj + c dc.
template <int ELEM>
__global__ __launch_bounds__(256) void factor_grad_kernel(const unsigned char *__restrict__ X,
                                                          int64_t ldx,
                                                          const float *__restrict__ T,
                                                          const int *__restrict__ ids,
                                                          float *__restrict__ D, int64_t dj,
                                                          int64_t dc, int64_t M, int64_t C,
                                                          int r) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int g = blockIdx.y, j = blockIdx.z;
  if (c >= C) return;
  float s = 0.f;
  for (int64_t m = 0; m < M; ++m)
    if (ids[m] == g) s += T[m * r + j] * elem_to_f32<ELEM>(X + 2 * (m * ldx + c));
  D[(int64_t)g * r * C + j * dj + c * dc] = s;
}

unsigned grid_for(int64_t n) { return (unsigned)(n < 1 ? 1 : n < (1 << 16) ? n : 1 << 16); }

template <int ELEM>
hipError_t narrow(const void *X, int64_t ldx, const void *F, int64_t fj, int64_t fk,
                  const float *alpha, const int32_t *ids, float *T, int64_t M, int64_t K,
                  int64_t r, int64_t G, hipStream_t stream) {
  hipLaunchKernelGGL(narrow_kernel<ELEM>, dim3(grid_for((M + 3) / 4)), dim3(256), 0, stream,
                     (const unsigned char *)X, ldx, (const unsigned char *)F, fj, fk, alpha, ids,
                     T, M, K, (int)r, (int)G);
  return hipGetLastError();
}

template <int ELEM, int OUT, bool kQ8>
hipError_t project(int product, const AdapterArgs &a, const Scratch &s, hipStream_t stream,
                   int num_cus) {
  const RectArgs p{kQ8 ? a.Xq : a.X, kQ8 ? a.ldxq : a.ldx, a.W, a.ldw, s.base, a.N,
                   a.M, a.K, a.N, false};
  hipError_t e = launch_rect(product, 0, p, stream, num_cus);
  if (e != hipSuccess) return e;
  if (a.G > 0) {
    e = narrow<ELEM>(a.X, a.ldx, a.A, a.K, 1, a.alpha, a.ids, s.t, a.M, a.K, a.r, a.G, stream);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((join_kernel<ELEM, OUT, kQ8>), dim3(grid_for((a.M * a.N + 255) / 256)),
                     dim3(256), 0, stream, a, (const void *)s.base, (const float *)s.t);
  return hipGetLastError();
}

hipError_t project_dt(int dtype, const AdapterArgs &a, const Scratch &s, hipStream_t stream,
                      int num_cus) {
  switch (dtype) {
    case TCU_F16_F32:
      return project<TCU_ELEM_F16, TCU_ELEM_F32, false>(TCU_F16_F32, a, s, stream, num_cus);
    case TCU_BF16_F32:
      return project<TCU_ELEM_BF16, TCU_ELEM_F32, false>(TCU_BF16_F32, a, s, stream, num_cus);
    case TCU_BF16_BF16:
      return project<TCU_ELEM_BF16, TCU_ELEM_BF16, false>(TCU_BF16_F32, a, s, stream, num_cus);
    case TCU_I8_I32:
      return project<TCU_ELEM_BF16, TCU_ELEM_BF16, true>(TCU_I8_I32, a, s, stream, num_cus);
  }
  return hipErrorInvalidValue;
}

template <int ELEM>
hipError_t grad_go(const AdapterGradArgs &a, hipStream_t stream) {
  const Scratch s = scratch(a.work, a.M, a.K, a.N, a.r, a.G);
  if (a.M > 0) {
    hipError_t e = narrow<ELEM>(a.X, a.ldx, a.A, a.K, 1, a.alpha, a.ids, s.t, a.M, a.K, a.r, a.G,
                                stream);
    if (e != hipSuccess) return e;
    e = narrow<ELEM>(a.dY, a.lddy, a.B, 1, a.r, a.alpha, a.ids, s.dt, a.M, a.N, a.r, a.G, stream);
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(factor_grad_kernel<ELEM>, dim3((unsigned)((a.K + 255) / 256), a.G, a.r),
                     dim3(256), 0, stream, (const unsigned char *)a.X, a.ldx, (const float *)s.dt,
                     a.ids, a.dA, a.K, (int64_t)1, a.M, a.K, (int)a.r);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(factor_grad_kernel<ELEM>, dim3((unsigned)((a.N + 255) / 256), a.G, a.r),
                     dim3(256), 0, stream, (const unsigned char *)a.dY, a.lddy,
                     (const float *)s.t, a.ids, a.dB, (int64_t)1, a.r, a.M, a.N, (int)a.r);
  return hipGetLastError();
}

}  // namespace

int64_t adapter_work_bytes(int64_t M, int64_t K, int64_t N, int64_t r, int64_t G) {
  return scratch(nullptr, M, K, N, r, G).bytes;
}

hipError_t launch_adapter(int dtype, const AdapterArgs &a, hipStream_t stream, int num_cus) {
  return project_dt(dtype, a, scratch(a.work, a.M, a.K, a.N, a.r, a.G), stream, num_cus);
}

hipError_t launch_adapter_input_grad(int dtype, const AdapterArgs &a, hipStream_t stream,
                                     int num_cus) {
  // The adapters' factors change places: A' = B^T (r x K here), B' = A^T (N x r).
  const Scratch s = scratch(a.work, a.M, a.N, a.K, a.r, a.G);
  AdapterArgs b = a;
  if (a.G > 0) {
    hipLaunchKernelGGL(transpose_kernel, dim3(1024), dim3(256), 0, stream,
                       (const unsigned short *)a.B, (unsigned short *)s.bt, a.K, a.r,
                       a.G * a.K * a.r);
    hipLaunchKernelGGL(transpose_kernel, dim3(1024), dim3(256), 0, stream,
                       (const unsigned short *)a.A, (unsigned short *)s.at, a.r, a.N,
                       a.G * a.r * a.N);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  b.A = s.bt;
  b.B = s.at;
  return project_dt(dtype, b, s, stream, num_cus);
}

hipError_t launch_adapter_grad(int elem, const AdapterGradArgs &a, hipStream_t stream, int) {
  switch (elem) {
    case TCU_ELEM_F16: return grad_go<TCU_ELEM_F16>(a, stream);
    case TCU_ELEM_BF16: return grad_go<TCU_ELEM_BF16>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace tcu

// Clipping of gradients by their common norm (tcu_clip_grads).
//
//   norm = sqrt(sum over all tensors of g^2),  out = g * min(1, max_norm / (norm + 1e-6))
//
// Bound by memory: every gradient is read for the norm, then read again (from
// the caches where all of them fit) and written: 1.04 GB of bfloat16 208 us and 417
// us, 5.0 TB/s each.  The tensors' addresses and
// sizes travel as kernel arguments, kTensors to a launch, so a call of up to
// kTensors tensors is two launches and needs no table in device memory.  Every
// tensor is cut into chunks of kChunk elements; a fixed grid walks the chunks
// of all tensors, so that a workgroup's part of the sum, and with it the sum's
// order, depends on the sizes alone.  Squares are summed in binary64: their
// range holds the square of every binary32 and bfloat16 value.
#include "tcu_elem.h"
#include "tcu_layer.h"

namespace tcu {
namespace {

// Tensors of a launch at most: 3.6 KB of kernel arguments.  Calls of few have smaller
// tables (8 tensors: 13.0 us a call, 13.5 with the large one).
constexpr int kTensors = 128, kFewTensors = 16;
constexpr int kParts = 1024;              // workgroups, each with a part of the sum
constexpr int kVecs = 4;                  // vectors of 8 elements per lane and chunk
constexpr int kChunk = 256 * 8 * kVecs;

template <int kMax>
struct Table {
  const unsigned char *g[kMax];
  unsigned char *out[kMax];
  int64_t count[kMax];
  unsigned first[kMax + 1];               // index of each tensor's first chunk
  unsigned char elem[kMax];
  int tensors;
};
static_assert(sizeof(Table<kTensors>) + 64 <= 4096, "kernel arguments");

// Calls f(tensor, first element, elements) for every gridDim.x'th chunk, from
// the first on or (kBack) from the last.
template <bool kBack, int kMax, typename F>
__device__ __forceinline__ void walk(const Table<kMax> &t, F f) {
  const unsigned total = t.first[t.tensors];
  int i = kBack ? t.tensors - 1 : 0;
  for (unsigned b = blockIdx.x; b < total; b += gridDim.x) {
    const unsigned c = kBack ? total - 1 - b : b;
    if constexpr (kBack)
      while (c < t.first[i]) --i;
    else
      while (c >= t.first[i + 1]) ++i;
    const int64_t at = (int64_t)(c - t.first[i]) * kChunk;
    const int64_t left = t.count[i] - at;
    f(i, at, (int)(left < kChunk ? left : kChunk));
  }
}

__device__ __forceinline__ double wave_sum64(double v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}

template <int ELEM>
__device__ __forceinline__ double chunk_squares(const unsigned char *p, int n) {
  double s = 0.0;
  Raw8<ELEM> r[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int e0 = (threadIdx.x + 256 * i) * 8;
    r[i] = e0 < n ? load8<ELEM>(p + (int64_t)e0 * elem_bytes<ELEM>, n - e0) : Raw8<ELEM>{};
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    float x[8];
    unpack8<ELEM>(r[i], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += (double)x[e] * (double)x[e];
  }
  return s;
}

// Parts of the sum of squares; `more`: added to those of earlier launches.
template <int kMax>
__global__ __launch_bounds__(256) void clip_norm_kernel(Table<kMax> t, double *__restrict__ parts,
                                                        int more) {
  __shared__ double lds[4];
  double s = 0.0;
  walk<false>(t, [&](int i, int64_t at, int n) {
    switch (t.elem[i]) {
      case TCU_ELEM_F32: s += chunk_squares<TCU_ELEM_F32>(t.g[i] + at * 4, n); break;
      case TCU_ELEM_F16: s += chunk_squares<TCU_ELEM_F16>(t.g[i] + at * 2, n); break;
      default: s += chunk_squares<TCU_ELEM_BF16>(t.g[i] + at * 2, n);
    }
  });
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = lds[0] + lds[1] + lds[2] + lds[3];
    parts[blockIdx.x] = more ? parts[blockIdx.x] + s : s;
  }
}

template <int ELEM>
__device__ __forceinline__ void chunk_scale(const unsigned char *g, unsigned char *out, int n,
                                            float coef) {
  Raw8<ELEM> r[kVecs];
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int e0 = (threadIdx.x + 256 * i) * 8;
    r[i] = e0 < n ? load8<ELEM>(g + (int64_t)e0 * elem_bytes<ELEM>, n - e0) : Raw8<ELEM>{};
  }
#pragma unroll
  for (int i = 0; i < kVecs; ++i) {
    const int e0 = (threadIdx.x + 256 * i) * 8;
    if (e0 >= n) continue;
    float x[8];
    unpack8<ELEM>(r[i], x);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] *= coef;
    store8<ELEM>(out + (int64_t)e0 * elem_bytes<ELEM>, x, n - e0);
  }
}

// Every workgroup adds the parts in the same order, then scales its chunks, the
// ones read last first: they are still in the caches.
template <int kMax>
__global__ __launch_bounds__(256) void clip_scale_kernel(Table<kMax> t,
                                                         const double *__restrict__ parts,
                                                         float max_norm,
                                                         float *__restrict__ result, int write) {
  __shared__ double lds[4];
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kParts / 256; ++i) s += parts[threadIdx.x + 256 * i];
  s = wave_sum64(s);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  const double norm = sqrt(lds[0] + lds[1] + lds[2] + lds[3]);
  const double q = (double)max_norm / (norm + 1e-6);
  const float coef = q >= 1.0 ? 1.f : (float)q;   // NaN stays NaN
  if (write && blockIdx.x == 0 && threadIdx.x == 0) {
    result[0] = (float)norm;
    result[1] = coef;
  }
  walk<true>(t, [&](int i, int64_t at, int n) {
    if (coef == 1.f && t.out[i] == t.g[i]) return;   // in place and unchanged
    switch (t.elem[i]) {
      case TCU_ELEM_F32:
        chunk_scale<TCU_ELEM_F32>(t.g[i] + at * 4, t.out[i] + at * 4, n, coef);
        break;
      case TCU_ELEM_F16:
        chunk_scale<TCU_ELEM_F16>(t.g[i] + at * 2, t.out[i] + at * 2, n, coef);
        break;
      default: chunk_scale<TCU_ELEM_BF16>(t.g[i] + at * 2, t.out[i] + at * 2, n, coef);
    }
  });
}

template <int kMax>
hipError_t clip_go(const void *const *grads, void *const *outs, const int64_t *counts,
                   const int32_t *elems, int64_t tensors, float max_norm, float *result,
                   void *work, hipStream_t stream) {
  double *parts = (double *)work;
  // The tensors of one launch: chunk numbers count in 32 bits, and a tensor
  // of more chunks than that is cut.
  constexpr int64_t kMost = (int64_t)1 << 30;
  auto each_table = [&](auto go) {
    Table<kMax> t{};
    int launches = 0;
    auto flush = [&]() {
      go(t, launches++);
      t.tensors = 0;
      return hipGetLastError();
    };
    for (int64_t i = 0; i < tensors; ++i) {
      for (int64_t at = 0; at < counts[i];) {
        const int64_t room = (kMost - t.first[t.tensors]) * kChunk;
        const int64_t n = counts[i] - at < room ? counts[i] - at : room;
        const int es = elems[i] == TCU_ELEM_F32 ? 4 : 2, k = t.tensors;
        t.g[k] = (const unsigned char *)grads[i] + at * es;
        t.out[k] = (unsigned char *)outs[i] + at * es;
        t.count[k] = n;
        t.elem[k] = (unsigned char)elems[i];
        t.first[k + 1] = t.first[k] + (unsigned)((n + kChunk - 1) / kChunk);
        t.tensors = k + 1;
        at += n;
        if (t.tensors == kMax || t.first[t.tensors] >= kMost) {
          const hipError_t e = flush();
          if (e != hipSuccess) return e;
        }
      }
    }
    // one launch at least: an empty sum is zero
    return t.tensors > 0 || launches == 0 ? flush() : hipSuccess;
  };
  const hipError_t e = each_table([&](const Table<kMax> &t, int k) {
    hipLaunchKernelGGL(clip_norm_kernel<kMax>, dim3(kParts), dim3(256), 0, stream, t, parts, k > 0);
  });
  if (e != hipSuccess) return e;
  return each_table([&](const Table<kMax> &t, int k) {
    const unsigned chunks = t.first[t.tensors];
    hipLaunchKernelGGL(clip_scale_kernel<kMax>, dim3(chunks < 1 ? 1 : chunks < 2048 ? chunks : 2048),
                       dim3(256), 0, stream, t, (const double *)parts, max_norm, result, k == 0);
  });
}

}  // namespace

int64_t clip_work_bytes() { return kParts * (int64_t)sizeof(double); }

hipError_t launch_clip(const void *const *grads, void *const *outs, const int64_t *counts,
                       const int32_t *elems, int64_t tensors, float max_norm, float *result,
                       void *work, hipStream_t stream, int) {
  return tensors <= kFewTensors
             ? clip_go<kFewTensors>(grads, outs, counts, elems, tensors, max_norm, result, work,
                                    stream)
             : clip_go<kTensors>(grads, outs, counts, elems, tensors, max_norm, result, work,
                                 stream);
}

}  // namespace tcu

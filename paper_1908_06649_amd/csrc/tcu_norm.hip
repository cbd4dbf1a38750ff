// Root-mean-square norm of rows, with the residual's addition and an 8-bit
// output, and its gradient (tcu_rms_norm, tcu_rms_norm_grad).
//
//   h = x + res,  y = h rstd w,  rstd = 1 / sqrt(mean(h^2) + eps)
//   dx = rstd (g - n mean(g n)) + dh,  g = dy w,  n = h rstd;   dw = sum_rows dy n
//
// (rstd^2 is never formed: without an eps it leaves binary32 where rstd does not.)
//
// Both are bound by memory: a row is read once, kept in registers while its
// sums are formed, and written once (8192 x 8192 bf16 with a residual: 104 us,
// 5.2 TB/s, a little over the rate of a copy of 1 GiB; the gradient 6007 x 4100 41 us, 4.8
// TB/s, and 4.8 us for the parts of dw).  A row of up to 1024 elements is one
// wave's, up to 16384 a workgroup's (kV vectors of eight elements per lane, the
// smallest number that holds the row); longer rows, and those of fewer than
// eight, are read twice.  Sums are binary32.
#include "tcu_elem.h"
#include "tcu_layer.h"

namespace tcu {
namespace {

constexpr int kWaveCols = 1024, kBlockCols = 16384;
// Up to so many rows, no more than the chip has compute units, a row of more than 2048
// columns is 16 waves' (us, bf16 with a residual, 4 waves / 16: 16 x 8192 3.9 / 3.3, 256 x
// 8192 5.2 / 4.7, 256 x 4096 3.8 / 3.6, 384 x 4096 4.2 / 4.6, 1024 x 8192 12.2 / 13.3;
// 256 x 2048 3.2 / 3.4).
constexpr int kFewNormRows = 256;
constexpr unsigned kInfBits = 0x7f800000u, kNormalBits = 0x00800000u;

// Sum and unsigned maximum over the kT threads of a row (64: a wave, else the
// workgroup, through LDS).
template <int kT>
__device__ __forceinline__ float row_sum(float v, float *lds) {
  v = wave_sum(v);
  if constexpr (kT > 64) {
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) lds[w] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int i = 0; i < kT / 64; ++i) v += lds[i];
    __syncthreads();   // read before the next sum overwrites
  }
  return v;
}
template <int kT>
__device__ __forceinline__ unsigned row_max(unsigned v, float *lds) {
  v = wave_max(v);
  if constexpr (kT > 64) {
    unsigned *u = (unsigned *)lds;
    const int w = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) u[w] = v;
    __syncthreads();
    v = 0u;
#pragma unroll
    for (int i = 0; i < kT / 64; ++i) v = u[i] > v ? u[i] : v;
    __syncthreads();
  }
  return v;
}

// The larger of m and |v| as bits, which order like the values, NaN above infinity.
__device__ __forceinline__ unsigned max_bits(unsigned m, float v) {
  const unsigned b = bitcast<unsigned>(v) & 0x7fffffffu;
  return b > m ? b : m;
}

// A row's largest |y| is its largest |h w| times rstd, unless h w has left binary32's
// normal range, which y need not have (or is not finite): then it is looked for among
// the |h rstd w|.
__device__ __forceinline__ bool is_normal(unsigned bits) {
  return bits >= kNormalBits && bits < kInfBits;
}

// What the 8-bit output of a row needs, from the bits of its largest |y|.
struct Quant {
  float pre, inv, scale;   // q = rint(y * pre * inv)
};
__device__ __forceinline__ Quant quant_of(unsigned max_y) {
  const float amax = bitcast<float>(max_y);
  Quant k;
  // 127 / amax stays finite down to the smallest maxima
  k.pre = amax < 0x1p-96f ? 0x1p96f : 1.f;
  k.scale = amax / 127.f;
  k.inv = amax > 0.f ? 127.f / (amax * k.pre) : 0.f;
  if (max_y >= kInfBits) {
    k.scale = __builtin_nanf("");
    k.inv = 0.f;
  }
  return k;
}
__device__ __forceinline__ void store_q8(unsigned char *p, const float (&y)[8], const Quant &k,
                                         int valid) {
  unsigned b[2] = {0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float f = rintf(y[e] * k.pre * k.inv);
    f = k.inv > 0.f ? fminf(fmaxf(f, -127.f), 127.f) : 0.f;
    b[e >> 2] |= ((unsigned)(int)f & 0xffu) << (8 * (e & 3));
  }
  if (valid >= 8) {
    typedef u32x2 u32x2_any __attribute__((aligned(1)));
    *(u32x2_any *)p = u32x2{b[0], b[1]};
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) p[e] = (unsigned char)(b[e >> 2] >> (8 * (e & 3)));
  }
}

// (without an eps a row of zeros has none to divide by: 0, not NaN)
__device__ __forceinline__ float rstd_of(float sum_sq, int64_t cols, float eps) {
  const float v = sum_sq / (float)cols + eps;
  return v == 0.f ? 0.f : 1.f / sqrtf(v);
}

// Vector i of a lane's row: eight columns from `col` on.  A row's last vector
// begins at its last eight columns (rows of fewer go to the long kernels): its
// first `dup` ones are then another lane's too, left out of this lane's sums, and
// stored twice with the same value.  So every access is a whole vector, and none
// waits for another.
struct Window {
  int col, dup;
  bool in;
};
template <int kT, int kV>
__device__ __forceinline__ Window window(int t, int i, int cols) {
  const int at = (t + i * kT) * 8;
  // kV vectors being the fewest that hold the row, all but the last are whole
  if (i < kV - 1) return Window{at, 0, true};
  const int col = at < cols - 8 ? at : cols - 8;
  return Window{col, at - col, at < cols};
}

// x + res, eight elements.
template <int ELEM>
__device__ __forceinline__ void load_h(const unsigned char *x, const unsigned char *res, int valid,
                                       float (&h)[8]) {
  const Raw8<ELEM> rx = load8<ELEM>(x, valid);
  if (res) {
    const Raw8<ELEM> rr = load8<ELEM>(res, valid);
    float b[8];
    unpack8<ELEM>(rx, h);
    unpack8<ELEM>(rr, b);
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] += b[e];
  } else {
    unpack8<ELEM>(rx, h);
  }
}

// The outputs of eight elements of a row.
template <int ELEM>
__device__ __forceinline__ void finish8(const NormArgs &a, int64_t row, int64_t col, int valid,
                                        const float (&h)[8], const float (&w)[8], float rstd,
                                        const Quant &k) {
  constexpr int ES = elem_bytes<ELEM>;
  if (a.h) store8<ELEM>((unsigned char *)a.h + (row * a.ldh + col) * ES, h, valid);
  if (!a.y && !a.q) return;
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = h[e] * rstd * w[e];
  if (a.y) store8<ELEM>((unsigned char *)a.y + (row * a.ldy + col) * ES, y, valid);
  if (a.q) store_q8((unsigned char *)a.q + row * a.ldq + col, y, k, valid);
}

template <int ELEM, int kT, int kV>
__global__ __launch_bounds__(kT < 256 ? 256 : kT) void rms_norm_kernel(NormArgs a) {
  constexpr int ES = elem_bytes<ELEM>, kRows = kT < 256 ? 256 / kT : 1;
  __shared__ float lds[16];
  const int t = threadIdx.x % kT;
  const int64_t step = (int64_t)gridDim.x * kRows;
  for (int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kT; row < a.rows; row += step) {
    const unsigned char *x = (const unsigned char *)a.x + row * a.ldx * ES;
    const unsigned char *res = a.res ? (const unsigned char *)a.res + row * a.ldr * ES : nullptr;
    float h[kV][8];
    Raw8<ELEM> w[kV];
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window v = window<kT, kV>(t, i, (int)a.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
      w[i] = Raw8<ELEM>{};
      if (v.in) {
        load_h<ELEM>(x + (int64_t)v.col * ES, res ? res + (int64_t)v.col * ES : nullptr, 8, h[i]);
        w[i] = load8<ELEM>((const unsigned char *)a.w + (int64_t)v.col * ES, 8);
      }
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int dup = window<kT, kV>(t, i, (int)a.cols).dup;
      float p = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) p += h[i][e] * h[i][e];
      if (dup > 0) {
        p = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) p += e >= dup ? h[i][e] * h[i][e] : 0.f;
      }
      ss += p;
    }
    const float rstd = rstd_of(row_sum<kT>(ss, lds), a.cols, a.eps);
    Quant k{};
    if (a.q) {
      // Once over h w, and again over h rstd w where those do not do.  One body for both,
      // kept by hiding from the compiler which it is: the registers of a second one made
      // 8192 x 8192 with a residual and three outputs take 132 us, not 124.
      unsigned m;
      int pass = 0;
      while (true) {
        asm volatile("" : "+v"(pass));
        const bool scaled = __builtin_amdgcn_readfirstlane(pass) != 0;
        const float r = scaled ? rstd : 1.f;
        m = 0u;
#pragma unroll
        for (int i = 0; i < kV; ++i) {
          float f[8];
          unpack8<ELEM>(w[i], f);
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max_bits(m, h[i][e] * r * f[e]);
        }
        m = __builtin_amdgcn_readfirstlane(row_max<kT>(m, lds));
        if (scaled) break;
        if (is_normal(m)) {
          m = bitcast<unsigned>(bitcast<float>(m) * rstd);
          break;
        }
        pass = 1;
      }
      k = quant_of(m);
      if (t == 0) a.qscale[row] = k.scale;
    }
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window v = window<kT, kV>(t, i, (int)a.cols);
      if (!v.in) continue;
      float f[8];
      unpack8<ELEM>(w[i], f);
      finish8<ELEM>(a, row, v.col, 8, h[i], f, rstd, k);
    }
  }
}

// Rows of any length: read once for the sums, once more for the outputs (and between
// them for an 8-bit output's scale where h w has left binary32's range).
template <int ELEM>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(NormArgs a) {
  constexpr int ES = elem_bytes<ELEM>, kT = 1024;
  __shared__ float lds[16];
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const unsigned char *x = (const unsigned char *)a.x + row * a.ldx * ES;
    const unsigned char *res = a.res ? (const unsigned char *)a.res + row * a.ldr * ES : nullptr;
    const unsigned char *w = (const unsigned char *)a.w;
    float ss = 0.f;
    unsigned m = 0u;
    float h[8], f[8];
    for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kT) {
      const int valid = (int)(a.cols - col < 8 ? a.cols - col : 8);
      load_h<ELEM>(x + col * ES, res ? res + col * ES : nullptr, valid, h);
      if (a.q) unpack8<ELEM>(load8<ELEM>(w + col * ES, valid), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += h[e] * h[e];
        if (a.q) m = max_bits(m, h[e] * f[e]);
      }
    }
    const float rstd = rstd_of(row_sum<kT>(ss, lds), a.cols, a.eps);
    Quant k{};
    if (a.q) {
      m = row_max<kT>(m, lds);
      if (is_normal(m)) {
        m = bitcast<unsigned>(bitcast<float>(m) * rstd);
      } else {
        m = 0u;
        for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kT) {
          const int valid = (int)(a.cols - col < 8 ? a.cols - col : 8);
          load_h<ELEM>(x + col * ES, res ? res + col * ES : nullptr, valid, h);
          unpack8<ELEM>(load8<ELEM>(w + col * ES, valid), f);
#pragma unroll
          for (int e = 0; e < 8; ++e) m = max_bits(m, h[e] * rstd * f[e]);
        }
        m = row_max<kT>(m, lds);
      }
      k = quant_of(m);
      if (threadIdx.x == 0) a.qscale[row] = k.scale;
    }
    for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kT) {
      const int valid = (int)(a.cols - col < 8 ? a.cols - col : 8);
      load_h<ELEM>(x + col * ES, res ? res + col * ES : nullptr, valid, h);
      unpack8<ELEM>(load8<ELEM>(w + col * ES, valid), f);
      finish8<ELEM>(a, row, col, valid, h, f, rstd, k);
    }
  }
}

// The gradient.  A workgroup takes every gridDim.x'th row (kT = 64: every wave
// a row) and sums its rows' part of dw in registers; the parts, one per
// workgroup, are added in their order by norm_dw_kernel.
template <int ELEM, int kT, int kV>
__global__ __launch_bounds__(kT < 256 ? 256 : kT) void rms_norm_grad_kernel(NormGradArgs a) {
  constexpr int ES = elem_bytes<ELEM>, kRows = kT < 256 ? 256 / kT : 1;
  // The next row's loads are in flight while a row is worked on, as far as two
  // workgroups' registers allow (bf16, us without / with: 8192 x 8192 110.5 /
  // 104.8, 6007 x 4100 39.3 / 38.5, 60000 x 512 44.5 / 42.0).
  constexpr bool kNext = kV <= (ELEM == TCU_ELEM_F32 ? 2 : 3);
  __shared__ float lds[kT == 64 ? 4 * kV * 512 : 16];
  const int t = threadIdx.x % kT;
  const unsigned char *dyp = (const unsigned char *)a.dy, *hp = (const unsigned char *)a.h;
  const unsigned char *dhp = (const unsigned char *)a.dh, *wp = (const unsigned char *)a.w;
  Raw8<ELEM> w[kV];
  float dw[kV][8];
#pragma unroll
  for (int i = 0; i < kV; ++i) {
    const Window v = window<kT, kV>(t, i, (int)a.cols);
    w[i] = v.in ? load8<ELEM>(wp + (int64_t)v.col * ES, 8) : Raw8<ELEM>{};
#pragma unroll
    for (int e = 0; e < 8; ++e) dw[i][e] = 0.f;
  }
  struct Row {
    Raw8<ELEM> dy[kV], h[kV], dh[kV];
  };
  auto load = [&](int64_t row, Row &v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window n = window<kT, kV>(t, i, (int)a.cols);
      v.dy[i] = v.h[i] = v.dh[i] = Raw8<ELEM>{};
      if (n.in && row < a.rows) {
        v.dy[i] = load8<ELEM>(dyp + (row * a.lddy + n.col) * ES, 8);
        v.h[i] = load8<ELEM>(hp + (row * a.ldh + n.col) * ES, 8);
        if (dhp) v.dh[i] = load8<ELEM>(dhp + (row * a.lddh + n.col) * ES, 8);
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * kRows;
  int64_t row = (int64_t)blockIdx.x * kRows + threadIdx.x / kT;
  Row next;
  if constexpr (kNext) load(row, next);
  for (; row < a.rows; row += step) {
    if constexpr (!kNext) load(row, next);
    const Row v = next;
    const Raw8<ELEM>(&dy)[kV] = v.dy, (&h)[kV] = v.h, (&dh)[kV] = v.dh;
    if constexpr (kNext) load(row + step, next);
    float ss = 0.f, gh = 0.f;
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const int dup = window<kT, kV>(t, i, (int)a.cols).dup;
      float d[8], x[8], f[8];
      unpack8<ELEM>(dy[i], d);
      unpack8<ELEM>(h[i], x);
      unpack8<ELEM>(w[i], f);
      float p = 0.f, g = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p += x[e] * x[e];
        g += d[e] * f[e] * x[e];
      }
      if (dup > 0) {
        p = g = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          p += e >= dup ? x[e] * x[e] : 0.f;
          g += e >= dup ? d[e] * f[e] * x[e] : 0.f;
        }
      }
      ss += p;
      gh += g;
    }
    ss = row_sum<kT>(ss, lds);
    gh = row_sum<kT>(gh, lds + (kT > 64 ? 8 : 0));
    const float rstd = rstd_of(ss, a.cols, a.eps);
    const float c = rstd * (gh / (float)a.cols);   // mean(g n)
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window n = window<kT, kV>(t, i, (int)a.cols);
      if (!n.in) continue;
      float d[8], x[8], f[8], r[8];
      unpack8<ELEM>(dy[i], d);
      unpack8<ELEM>(h[i], x);
      unpack8<ELEM>(w[i], f);
      unpack8<ELEM>(dh[i], r);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hn = x[e] * rstd;
        dw[i][e] += d[e] * hn;
        r[e] += rstd * (d[e] * f[e] - hn * c);
      }
      store8<ELEM>((unsigned char *)a.dx + (row * a.lddx + n.col) * ES, r, 8);
    }
  }
  float *part = a.work + (int64_t)blockIdx.x * a.cols;
  if constexpr (kT == 64) {
    // the four waves' sums, in their order
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window n = window<kT, kV>(t, i, (int)a.cols);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (n.in) lds[(threadIdx.x >> 6) * kV * 512 + n.col + e] = dw[i][e];
    }
    __syncthreads();
    for (int col = threadIdx.x; col < a.cols; col += 256) {
      float v = 0.f;
#pragma unroll
      for (int q = 0; q < 4; ++q) v += lds[q * kV * 512 + col];
      part[col] = v;
    }
  } else {
#pragma unroll
    for (int i = 0; i < kV; ++i) {
      const Window n = window<kT, kV>(t, i, (int)a.cols);
      if (n.in) store8<TCU_ELEM_F32>((unsigned char *)(part + n.col), dw[i], 8);
    }
  }
}

// Rows of any length; a workgroup's part of dw is kept in memory.
template <int ELEM>
__global__ __launch_bounds__(1024) void rms_norm_grad_long_kernel(NormGradArgs a) {
  constexpr int ES = elem_bytes<ELEM>, kT = 1024;
  __shared__ float lds[32];
  const unsigned char *wp = (const unsigned char *)a.w;
  float *part = a.work + (int64_t)blockIdx.x * a.cols;
  for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const unsigned char *dyp = (const unsigned char *)a.dy + row * a.lddy * ES;
    const unsigned char *hp = (const unsigned char *)a.h + row * a.ldh * ES;
    const unsigned char *dhp =
        a.dh ? (const unsigned char *)a.dh + row * a.lddh * ES : nullptr;
    float d[8], x[8], f[8], r[8];
    float ss = 0.f, gh = 0.f;
    for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kT) {
      const int valid = (int)(a.cols - col < 8 ? a.cols - col : 8);
      unpack8<ELEM>(load8<ELEM>(dyp + col * ES, valid), d);
      unpack8<ELEM>(load8<ELEM>(hp + col * ES, valid), x);
      unpack8<ELEM>(load8<ELEM>(wp + col * ES, valid), f);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        ss += x[e] * x[e];
        gh += d[e] * f[e] * x[e];
      }
    }
    ss = row_sum<kT>(ss, lds);
    gh = row_sum<kT>(gh, lds + 16);
    const float rstd = rstd_of(ss, a.cols, a.eps);
    const float c = rstd * (gh / (float)a.cols);   // mean(g n)
    const bool first = row == blockIdx.x;
    for (int64_t col = 8 * threadIdx.x; col < a.cols; col += 8 * kT) {
      const int valid = (int)(a.cols - col < 8 ? a.cols - col : 8);
      unpack8<ELEM>(load8<ELEM>(dyp + col * ES, valid), d);
      unpack8<ELEM>(load8<ELEM>(hp + col * ES, valid), x);
      unpack8<ELEM>(load8<ELEM>(wp + col * ES, valid), f);
      unpack8<ELEM>(dhp ? load8<ELEM>(dhp + col * ES, valid) : Raw8<ELEM>{}, r);
      float s[8] = {};
      if (!first)
        unpack8<TCU_ELEM_F32>(load8<TCU_ELEM_F32>((unsigned char *)(part + col), valid), s);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float hn = x[e] * rstd;
        s[e] += d[e] * hn;
        r[e] += rstd * (d[e] * f[e] - hn * c);
      }
      store8<TCU_ELEM_F32>((unsigned char *)(part + col), s, valid);
      store8<ELEM>((unsigned char *)a.dx + (row * a.lddx + col) * ES, r, valid);
    }
  }
}

// dw = the sum of `parts` rows of partial sums: a workgroup takes every gridDim.x'th
// 32 columns, its 32 half waves every 32nd part, four loads in flight.
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float *__restrict__ work,
                                                       float *__restrict__ dw, int parts,
                                                       int64_t cols) {
  __shared__ float lds[32][33];
  const int c = threadIdx.x & 31, h = threadIdx.x >> 5;
  for (int64_t col0 = (int64_t)blockIdx.x * 32; col0 < cols; col0 += (int64_t)gridDim.x * 32) {
    const int64_t col = col0 + c;
    float v = 0.f;
    if (col < cols) {
      int p = h;
      for (; p + 96 < parts; p += 128) {
        const float *at = work + p * cols + col;
        const float u0 = at[0], u1 = at[32 * cols], u2 = at[64 * cols], u3 = at[96 * cols];
        v = v + u0 + u1 + u2 + u3;
      }
      for (; p < parts; p += 32) v += work[p * cols + col];
    }
    lds[h][c] = v;
    __syncthreads();
    if (h == 0 && col < cols) {
      v = 0.f;
#pragma unroll
      for (int i = 0; i < 32; ++i) v += lds[i][c];
      dw[col] = v;
    }
    __syncthreads();   // read before the next columns overwrite
  }
}

int vectors(int64_t cols, int threads) {
  return (int)((cols + 8 * threads - 1) / (8 * threads));
}

// f(integral_constant) with the smallest number of vectors per lane, up to kMost.
template <int kMost, typename F>
void with_vectors(int v, F f) {
  if constexpr (kMost > 1) {
    if (v < kMost) return with_vectors<kMost - 1>(v, f);
  }
  f(std::integral_constant<int, kMost>{});
}

// Workgroups of a grid over `n` pieces of work: a launch counts its work items
// in 32 bits, and the kernels walk on from there.
unsigned grid_for(int64_t n) { return (unsigned)(n < (1 << 20) ? n : 1 << 20); }

template <int ELEM>
hipError_t norm_go(const NormArgs &a, hipStream_t stream) {
  if (a.cols < 8 || a.cols > kBlockCols) {
    hipLaunchKernelGGL(rms_norm_long_kernel<ELEM>, dim3(grid_for(a.rows)), dim3(1024), 0, stream,
                       a);
  } else if (a.cols <= kWaveCols) {
    const dim3 grid(grid_for((a.rows + 3) / 4));
    if (vectors(a.cols, 64) == 1)
      hipLaunchKernelGGL((rms_norm_kernel<ELEM, 64, 1>), grid, dim3(256), 0, stream, a);
    else
      hipLaunchKernelGGL((rms_norm_kernel<ELEM, 64, 2>), grid, dim3(256), 0, stream, a);
  } else if (a.rows <= kFewNormRows && a.cols > 2048) {
    if (vectors(a.cols, 1024) == 1)
      hipLaunchKernelGGL((rms_norm_kernel<ELEM, 1024, 1>), dim3(grid_for(a.rows)), dim3(1024), 0,
                         stream, a);
    else
      hipLaunchKernelGGL((rms_norm_kernel<ELEM, 1024, 2>), dim3(grid_for(a.rows)), dim3(1024), 0,
                         stream, a);
  } else {
    with_vectors<8>(vectors(a.cols, 256), [&](auto v) {
      hipLaunchKernelGGL((rms_norm_kernel<ELEM, 256, decltype(v)::value>), dim3(grid_for(a.rows)),
                         dim3(256), 0, stream, a);
    });
  }
  return hipGetLastError();
}

template <int ELEM>
hipError_t grad_go(const NormGradArgs &a, hipStream_t stream) {
  int parts = (int)(a.rows < kNormParts ? a.rows : kNormParts);
  if (a.rows > 0) {
    if (a.cols < 8 || a.cols > kBlockCols) {
      hipLaunchKernelGGL(rms_norm_grad_long_kernel<ELEM>, dim3(parts), dim3(1024), 0, stream, a);
    } else if (a.cols <= kWaveCols) {
      if (parts > (a.rows + 3) / 4) parts = (int)((a.rows + 3) / 4);
      if (vectors(a.cols, 64) == 1)
        hipLaunchKernelGGL((rms_norm_grad_kernel<ELEM, 64, 1>), dim3(parts), dim3(256), 0, stream,
                           a);
      else
        hipLaunchKernelGGL((rms_norm_grad_kernel<ELEM, 64, 2>), dim3(parts), dim3(256), 0, stream,
                           a);
    } else if (vectors(a.cols, 256) <= (ELEM == TCU_ELEM_F32 ? 2 : 3)) {
      // As long as the next row's loads have registers; then 8 waves, whose rows have half
      // the vectors (us, bf16, 4 waves / 8: 6007 x 4096 35.7 / 37.2, 2000 x 6144 23.1 /
      // 26.0, 6007 x 8192 80.7 / 79.1, 6007 x 12288 127 / 123, 2000 x 16384 67 / 61; just
      // past the bound 4 are faster, 6007 x 6200 54.5 / 61.7).
      with_vectors<3>(vectors(a.cols, 256), [&](auto v) {
        hipLaunchKernelGGL((rms_norm_grad_kernel<ELEM, 256, decltype(v)::value>), dim3(parts),
                           dim3(256), 0, stream, a);
      });
    } else {
      with_vectors<4>(vectors(a.cols, 512), [&](auto v) {
        hipLaunchKernelGGL((rms_norm_grad_kernel<ELEM, 512, decltype(v)::value>), dim3(parts),
                           dim3(512), 0, stream, a);
      });
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL(norm_dw_kernel, dim3(grid_for((a.cols + 31) / 32)), dim3(1024), 0, stream,
                     a.work, a.dw, parts, a.cols);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(int elem, const NormArgs &a, hipStream_t stream, int) {
  switch (elem) {
    case TCU_ELEM_F32: return norm_go<TCU_ELEM_F32>(a, stream);
    case TCU_ELEM_F16: return norm_go<TCU_ELEM_F16>(a, stream);
    case TCU_ELEM_BF16: return norm_go<TCU_ELEM_BF16>(a, stream);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_rms_norm_grad(int elem, const NormGradArgs &a, hipStream_t stream, int) {
  switch (elem) {
    case TCU_ELEM_F32: return grad_go<TCU_ELEM_F32>(a, stream);
    case TCU_ELEM_F16: return grad_go<TCU_ELEM_F16>(a, stream);
    case TCU_ELEM_BF16: return grad_go<TCU_ELEM_BF16>(a, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace tcu

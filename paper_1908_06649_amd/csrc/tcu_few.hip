// A projection with low-rank adapters for few rows (single tokens of a batch of
// requests): bound by the weights' bytes, read once.
//
// few_kernel forms the product's partial sums and T = alpha X A^T in one launch,
// join_kernel adds the partial sums and T B^T and rounds.
//   * Rows go in blocks of 64, each reading W for itself (the later ones from the
//     caches).
//   * A workgroup's 8 waves share a strip of W's columns (64 of 16 bits, 128 of
//     8) over one of `splits` ranges of the contracted index, one or two
//     workgroups per CU in all; the waves take the steps of 64 bytes of it in turn, for all
//     rows.  A lane loads 8 bytes of each of a step's 8 (16) rows of W that it
//     holds, 16 lanes a whole row of the strip, and exchanges bytes in its own
//     registers to the runs along the contracted index that the matrix cores
//     take: W goes through neither LDS nor another lane.  The next step's loads
//     are in flight under a step's products.
//   * The waves' sums are added in LDS in their order, the ranges' by join_kernel.
//   * T's values are dealt to all waves, one at a time, while their first loads of W
//     are on their way: every row has an adapter of its own, and both operands lie
//     along the contracted index.
// 8 x 4096 x 4096 bf16 rank 16: 8.3 + 2.7 us, 4.2 TB/s of what the first launch reads;
// 48 x 8192 x 8192 int8: 19.3 + 4.1 us, 4.1 TB/s.
#include "tcu_elem.h"
#include "tcu_layer.h"

namespace tcu {
namespace {

constexpr int kWaves = 8;   // of a workgroup

// How a step of W lies: ES bytes per element, kRun elements of the contracted
// index per lane, kCols columns per lane (8 bytes).
template <int ES>
struct Step {
  static constexpr int kRun = 16 / ES, kElems = 4 * kRun, kCols = 8 / ES, kStrip = 16 * kCols;
};

__device__ __forceinline__ u32x2 load8_any(const unsigned char *p) {
  typedef u32x2 u32x2_any __attribute__((aligned(1)));
  return *(const u32x2_any *)p;
}

// A lane's kRun rows of 8 bytes -> its columns' runs of 16 bytes.
template <int ES>
__device__ __forceinline__ void to_runs(const u32x2 (&w)[16 / ES], u32x4 (&run)[8 / ES]) {
  if constexpr (ES == 2) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int d = 0; d < 4; ++d)
        run[j][d] = __builtin_amdgcn_perm(w[2 * d + 1][j >> 1], w[2 * d][j >> 1],
                                          j & 1 ? 0x07060302u : 0x05040100u);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        // 4 x 4 bytes: rows 4 d .. of columns 4 h ..
        const unsigned a = w[4 * d][h], b = w[4 * d + 1][h], c = w[4 * d + 2][h],
                       e = w[4 * d + 3][h];
        const unsigned ab0 = __builtin_amdgcn_perm(b, a, 0x05010400u);
        const unsigned ab2 = __builtin_amdgcn_perm(b, a, 0x07030602u);
        const unsigned ce0 = __builtin_amdgcn_perm(e, c, 0x05010400u);
        const unsigned ce2 = __builtin_amdgcn_perm(e, c, 0x07030602u);
        run[4 * h][d] = __builtin_amdgcn_perm(ce0, ab0, 0x05040100u);
        run[4 * h + 1][d] = __builtin_amdgcn_perm(ce0, ab0, 0x07060302u);
        run[4 * h + 2][d] = __builtin_amdgcn_perm(ce2, ab2, 0x05040100u);
        run[4 * h + 3][d] = __builtin_amdgcn_perm(ce2, ab2, 0x07060302u);
      }
  }
}

struct FewArgs {
  const unsigned char *X, *W;      // the product's operands
  const unsigned char *XA, *A;     // the adapters'
  const float *alpha;
  const int *ids;
  unsigned *parts;                 // splits x M x N sums (binary32 or int32)
  float *T;                        // M rows of tld
  int64_t ldx, ldw, ldxa;
  int M, K, N, r, G, strips, splits, tld;
  bool narrow;                     // T is formed here
};

// One value of T: row i / r, rank i % r, by one wave, 512 kU elements of both
// operands in flight (a memory latency each: 16 x 8192 x 8192 int8 rank 16 23.7 us with
// 8, 24.6 with 4).
template <int ELEM, int kU>
__device__ __forceinline__ void narrow_value(const FewArgs &a, int i) {
  const int m = i / a.r, j = i - m * a.r, g = a.ids[m];
  if (g < 0 || g >= a.G) return;
  const int lane = threadIdx.x & 63;
  const unsigned char *x = a.XA + 2 * (int64_t)m * a.ldxa;
  const unsigned char *f = a.A + 2 * ((int64_t)g * a.r + j) * a.K;
  float s = 0.f;
  auto add = [&](const Raw8<ELEM> &xr, const Raw8<ELEM> &fr, int from) __attribute__((always_inline)) {
    float xv[8], fv[8];
    unpack8<ELEM>(xr, xv);
    unpack8<ELEM>(fr, fv);
#pragma unroll
    for (int e = 0; e < 8; ++e) s += e >= from ? xv[e] * fv[e] : 0.f;
  };
  int k = 8 * lane;
  for (; k - 8 * lane + 512 * kU <= a.K; k += 512 * kU) {
    Raw8<ELEM> xr[kU], fr[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      xr[u].v[0] = load16_any(x + 2 * (k + 512 * u));
      fr[u].v[0] = load16_any(f + 2 * (k + 512 * u));
    }
#pragma unroll
    for (int u = 0; u < kU; ++u) add(xr[u], fr[u], 0);
  }
  if (a.K >= 8) {
    // the rest four vectors at once: one that would pass the end begins at the last
    // eight elements, those before its own left out
    constexpr int kRest = 4;
    for (; k - 8 * lane < a.K; k += 512 * kRest) {
      Raw8<ELEM> xr[kRest], fr[kRest];
#pragma unroll
      for (int u = 0; u < kRest; ++u) {
        const int at = min(k + 512 * u, a.K - 8);
        xr[u].v[0] = load16_any(x + 2 * at);
        fr[u].v[0] = load16_any(f + 2 * at);
      }
#pragma unroll
      for (int u = 0; u < kRest; ++u)
        add(xr[u], fr[u], k + 512 * u - min(k + 512 * u, a.K - 8));
    }
  } else if (lane == 0) {
    add(load8<ELEM>(x, a.K), load8<ELEM>(f, a.K), 0);
  }
  s = wave_sum(s);
  if (lane == 0) a.T[(int64_t)m * a.tld + j] = s * a.alpha[g];
}

// DT: the product's types; ELEM: the adapters'; kMB: blocks of 16 rows.
template <int DT, int ELEM, int kMB>
__global__ __launch_bounds__(64 * kWaves) void few_kernel(FewArgs a) {
  constexpr int ES = in_bytes(DT);
  // 8-bit W and more than 32 rows: a second step's registers are not there
  constexpr bool kAhead = ES == 2 || kMB <= 2;
  constexpr bool kI8 = ES == 1;
  // (8 would leave room for one workgroup where two fit)
  constexpr int kNarrowAhead = kI8 || kMB > 2 ? 8 : 4;
  typedef Step<ES> S;
  typedef typename std::conditional<kI8, i32x4, f32x4>::type Acc;
  constexpr int kRowLds = S::kStrip + 4;
  __shared__ unsigned sums[kWaves][16 * kRowLds];
  const int row0 = blockIdx.y * (int)kFewBlock, rows = min(a.M - row0, (int)kFewBlock);
  const int split = blockIdx.x / a.strips, n0 = (blockIdx.x - split * a.strips) * S::kStrip;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int steps = (a.K + S::kElems - 1) / S::kElems;
  const int s_begin = (int)((int64_t)steps * split / a.splits);
  const int s_end = (int)((int64_t)steps * (split + 1) / a.splits);
  // columns past N repeat the last ones inside and are not stored
  const int col = min(n0 + S::kCols * c, a.N - S::kCols);
  const unsigned char *wp = a.W + ((int64_t)S::kRun * q * a.ldw + col) * ES;
  const unsigned char *xp[kMB];
#pragma unroll
  for (int b = 0; b < kMB; ++b)
    xp[b] = a.X + ((int64_t)(row0 + min(16 * b + c, rows - 1)) * a.ldx + S::kRun * q) * ES;
  Acc acc[kMB][S::kCols];
#pragma unroll
  for (int b = 0; b < kMB; ++b)
#pragma unroll
    for (int j = 0; j < S::kCols; ++j) acc[b][j] = Acc{0, 0, 0, 0};

  auto load = [&](int s, u32x2 (&wr)[S::kRun], u32x4 (&xr)[kMB]) __attribute__((always_inline)) {
    const int k = s * S::kElems, left = a.K - k;
    if (left >= S::kElems) {
      const unsigned char *p = wp + (int64_t)k * a.ldw * ES;
#pragma unroll
      for (int i = 0; i < S::kRun; ++i) wr[i] = load8_any(p + (int64_t)i * a.ldw * ES);
#pragma unroll
      for (int b = 0; b < kMB; ++b) xr[b] = load16_any(xp[b] + (int64_t)k * ES);
    } else {
      // the last step: zeros past K
#pragma unroll
      for (int i = 0; i < S::kRun; ++i) {
        const int row = S::kRun * q + i;
        wr[i] = load8_any(wp + ((int64_t)(min(row, left - 1) - S::kRun * q) + k) * a.ldw * ES);
        if (row >= left) wr[i] = u32x2{0u, 0u};
      }
#pragma unroll
      for (int b = 0; b < kMB; ++b)
        xr[b] = load_chunk<ES>(xp[b] + (int64_t)k * ES, max(min(left - S::kRun * q, S::kRun), 0));
    }
  };
  auto multiply = [&](const u32x2 (&wr)[S::kRun], const u32x4 (&xr)[kMB])
      __attribute__((always_inline)) {
    u32x4 run[S::kCols];
    to_runs<ES>(wr, run);
#pragma unroll
    for (int j = 0; j < S::kCols; ++j)
#pragma unroll
      for (int b = 0; b < kMB; ++b) {
        if constexpr (kI8)
          acc[b][j] = mfma_i8_k64(run[j], xr[b], acc[b][j]);
        else
          acc[b][j] = mfma_k32(DT, run[j], xr[b], acc[b][j]);
      }
  };
  // The adapters' narrow product while the first step is on its way: its values
  // in turn over all waves of the grid.
  auto narrow = [&]() {
    const int all = a.narrow ? a.M * a.r : 0;
    const int groups = gridDim.x * gridDim.y;
    for (int i = blockIdx.y * gridDim.x + blockIdx.x + w * groups; i < all; i += groups * kWaves)
      narrow_value<ELEM, kNarrowAhead>(a, i);
  };
  int s = s_begin + w;
  if constexpr (kAhead) {
    u32x2 w0[S::kRun], w1[S::kRun];
    u32x4 x0[kMB], x1[kMB];
    if (s < s_end) load(s, w0, x0);
    if (s + kWaves < s_end) load(s + kWaves, w1, x1);
    narrow();
    while (s < s_end) {
      multiply(w0, x0);
      if (s + 2 * kWaves < s_end) load(s + 2 * kWaves, w0, x0);
      if (s + kWaves < s_end) multiply(w1, x1);
      if (s + 3 * kWaves < s_end) load(s + 3 * kWaves, w1, x1);
      s += 2 * kWaves;
    }
  } else {
    u32x2 w0[S::kRun];
    u32x4 x0[kMB];
    if (s < s_end) load(s, w0, x0);
    narrow();
    while (s < s_end) {
      multiply(w0, x0);
      s += kWaves;
      if (s < s_end) load(s, w0, x0);
    }
  }
  // The waves' sums, 16 rows at a time: a lane holds column kCols (4 q + e) + j
  // of the strip and row c of the block.
#pragma unroll
  for (int b = 0; b < kMB; ++b) {
    if (16 * b >= rows) break;
    if (b > 0) __syncthreads();   // read before the next sums overwrite
#pragma unroll
    for (int j = 0; j < S::kCols; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        sums[w][c * kRowLds + S::kCols * (4 * q + e) + j] = bitcast<u32x4>(acc[b][j])[e];
    __syncthreads();
#pragma unroll
    for (int i = threadIdx.x; i < 16 * S::kStrip; i += 64 * kWaves) {
      const int m = i / S::kStrip, at = i % S::kStrip;
      unsigned v = sums[0][m * kRowLds + at];
#pragma unroll
      for (int u = 1; u < kWaves; ++u) {
        const unsigned o = sums[u][m * kRowLds + at];
        v = kI8 ? v + o : bitcast<unsigned>(bitcast<float>(v) + bitcast<float>(o));
      }
      const int first = n0 + at / S::kCols * S::kCols;
      const int n = min(first, a.N - S::kCols) + at % S::kCols;
      if (16 * b + m < rows && n >= first)
        a.parts[((int64_t)split * a.M + row0 + 16 * b + m) * a.N + n] = v;
    }
  }
}

// Y = the ranges' sums (scaled, 8-bit) + T B^T, rounded once.
// kAtOnce ranges' sums and kHeld vectors of 8 ranks are loaded together: no more than
// there are (200 x 2048 x 2048, two ranges: 16.1 us of a call, 17.2 with eight).
template <int ELEM, int OUT, bool kQ8, int kAtOnce, int kHeld>
__global__ __launch_bounds__(256) void join_kernel(FewArgs f, const unsigned char *__restrict__ B,
                                                   const float *__restrict__ xscale,
                                                   const float *__restrict__ wscale,
                                                   unsigned char *__restrict__ Y, int64_t ldy) {
  const int n = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  if (n >= f.N) return;
  // What the sums do not wait for goes first: the row's adapter, the ranges' sums,
  // the scales, then the adapter's ranks (8 x 4096 x 4096 3.1 us, one after the
  // other 4.6).
  const int g = f.G > 0 ? f.ids[m] : -1;
  const bool adapted = g >= 0 && g < f.G;
  const unsigned *p = f.parts + (int64_t)m * f.N + n;
  const int64_t range = (int64_t)f.M * f.N;
  // (no branch around a load: the compiler would wait for it there)
  unsigned u[kAtOnce];
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) u[i] = p[min(i, f.splits - 1) * range];
  const float scale = kQ8 ? xscale[m] : 1.f, col_scale = kQ8 ? wscale[n] : 1.f;
  const unsigned char *b = B + 2 * (((int64_t)g * f.N + n) * f.r);
  const float *t = f.T + (int64_t)m * f.tld;
  const int whole = f.r & ~7;      // ranks in whole vectors
  struct Held {
    u32x4 b[kHeld];
    float t[8 * kHeld];
  } held = {};
  // ranks j0 .. of the whole vectors, the last ones again past them
  auto load = [&](int j0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int j = min(j0 + 8 * i, whole - 8);
      held.b[i] = load16_any(b + 2 * j);
#pragma unroll
      for (int e = 0; e < 8; ++e) held.t[8 * i + e] = t[j + e];
    }
  };
  if (adapted && whole > 0) load(0);
  float v;
  if constexpr (kQ8) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) sum += i < f.splits ? (int)u[i] : 0;
    for (int s = kAtOnce; s < f.splits; ++s) sum += (int)p[s * range];
    v = (float)sum * scale * col_scale;
  } else {
    v = 0.f;
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) v += i < f.splits ? bitcast<float>(u[i]) : 0.f;
    for (int s = kAtOnce; s < f.splits; ++s) v += bitcast<float>(p[s * range]);
  }
  if (adapted) {
    float low = 0.f;
    for (int j0 = 0; j0 < whole; j0 += 8 * kHeld) {
      if (j0 > 0) load(j0);
#pragma unroll
      for (int i = 0; i < kHeld; ++i) {
        float x[8];
        unpack8<ELEM>(Raw8<ELEM>{held.b[i]}, x);
        if (j0 + 8 * i < whole)
#pragma unroll
          for (int e = 0; e < 8; ++e) low += held.t[8 * i + e] * x[e];
      }
    }
    if (whole < f.r) {
      float x[8];
      unpack8<ELEM>(load8<ELEM>(b + 2 * whole, f.r - whole), x);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (whole + e < f.r) low += t[whole + e] * x[e];
    }
    v += low;
  }
  f32_to_elem<OUT>(Y + ((int64_t)m * ldy + n) * elem_bytes<OUT>, v);
}

int row_blocks(int64_t M) { return M <= 16 ? 1 : M < kFewBlock ? (int)((M + 15) / 16) : 4; }

int strip_cols(bool q8) { return q8 ? Step<1>::kStrip : Step<2>::kStrip; }

// Ranges of the contracted index: about two workgroups per compute unit where
// two fit its registers (16-bit W, up to 32 rows), else one, and a step at least
// for every wave.  Us of a call, bf16, 256 / 512 workgroups: 8 x 4096 x 4096 17.0
// / 15.5, 8 x 8192 x 8192 31.9 / 29.2, 48 x 4096 x 4096 18.6 / 22.5 (the ranges'
// sums); int8 32 x 8192 x 8192 25.7 / 29.4.
int few_splits(int64_t M, int64_t K, int64_t N, bool q8) {
  const int64_t strips = N > 0 ? (N + strip_cols(q8) - 1) / strip_cols(q8) : 1;
  const int64_t wave_elems = (int64_t)(q8 ? 64 : 32) * kWaves;
  const int64_t want = !q8 && M <= 32 ? 512 : 256;
  const int64_t groups = strips * ((M + kFewBlock - 1) / kFewBlock);
  int64_t n = groups > 0 ? (want + groups / 2) / groups : 1;
  const int64_t most = (K + wave_elems - 1) / wave_elems;
  if (n > most) n = most;
  return (int)(n < 1 ? 1 : n > 16 ? 16 : n);
}

int64_t parts_bytes(int64_t M, int64_t K, int64_t N, bool q8) {
  return (few_splits(M, K, N, q8) * M * N * 4 + 255) / 256 * 256;
}

template <int DT, int ELEM, int OUT, bool kQ8>
hipError_t few(const AdapterArgs &a, float *T, int tld, hipStream_t stream) {
  const int strips = (int)((a.N + strip_cols(kQ8) - 1) / strip_cols(kQ8));
  const int splits = few_splits(a.M, a.K, a.N, kQ8);
  const FewArgs f{(const unsigned char *)(kQ8 ? a.Xq : a.X),
                  (const unsigned char *)a.W,
                  (const unsigned char *)a.X,
                  (const unsigned char *)a.A,
                  a.alpha,
                  a.ids,
                  (unsigned *)a.work,
                  T ? T : (float *)((unsigned char *)a.work + parts_bytes(a.M, a.K, a.N, kQ8)),
                  kQ8 ? a.ldxq : a.ldx,
                  a.ldw,
                  a.ldx,
                  (int)a.M,
                  (int)a.K,
                  (int)a.N,
                  (int)a.r,
                  (int)a.G,
                  strips,
                  splits,
                  T ? tld : (int)a.r,
                  a.G > 0 && !T};
  const dim3 grid(strips * splits, (unsigned)((a.M + kFewBlock - 1) / kFewBlock));
  auto go = [&](auto blocks) {
    constexpr int kMB = decltype(blocks)::value;
    hipLaunchKernelGGL((few_kernel<DT, ELEM, kMB>), grid,
                       dim3(64 * kWaves), 0, stream, f);
  };
  switch (row_blocks(a.M)) {
    case 1: go(std::integral_constant<int, 1>{}); break;
    case 2: go(std::integral_constant<int, 2>{}); break;
    case 3: go(std::integral_constant<int, 3>{}); break;
    default: go(std::integral_constant<int, 4>{});
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  auto join = [&](auto at_once, auto held) {
    hipLaunchKernelGGL(
        (join_kernel<ELEM, OUT, kQ8, decltype(at_once)::value, decltype(held)::value>),
        dim3((unsigned)((a.N + 255) / 256), (unsigned)a.M), dim3(256), 0, stream, f,
        (const unsigned char *)a.B, a.xscale, a.wscale, (unsigned char *)a.Y, a.ldy);
  };
  auto join_ranks = [&](auto at_once) {
    if (a.r <= 16)
      join(at_once, std::integral_constant<int, 2>{});
    else
      join(at_once, std::integral_constant<int, 4>{});
  };
  if (splits <= 2)
    join_ranks(std::integral_constant<int, 2>{});
  else if (splits <= 4)
    join_ranks(std::integral_constant<int, 4>{});
  else
    join_ranks(std::integral_constant<int, 8>{});
  return hipGetLastError();
}

}  // namespace

// A lane's load takes 8 bytes of a row of W: 4 columns of 16 bits, 8 of 8.
bool few_ok(int dtype, const AdapterArgs &a) {
  return a.M <= kFewRows && a.K > 0 && a.N >= (dtype == TCU_I8_I32 ? 8 : 4);
}

// What forming T here adds: one value a wave goes under the loads of W, each more
// takes a loaded memory's latency for as much of K as a wave has in flight (us, T here / apart:
// 188 x 6976 x 512 rank 64 50.6 / 33.9; 148 x 2845 x 369 rank 64 int8 83.1 / 39.4;
// 64 x 4096 x 512 rank 64 int8 37.5 / 26.9; 256 x 8192 x 256 rank 16 20.0 / 24.2;
// 128 x 4096 x 1024 rank 32 15.3 / 21.4).
double few_narrow_us(const AdapterArgs &a, bool q8) {
  const int64_t strips = (a.N + strip_cols(q8) - 1) / strip_cols(q8);
  const int64_t waves = strips * few_splits(a.M, a.K, a.N, q8) *
                        ((a.M + kFewBlock - 1) / kFewBlock) * kWaves;
  const int64_t values = a.G > 0 ? (a.M * a.r + waves - 1) / waves : 0;
  const int64_t deep = q8 || a.M > 32 ? 4096 : 2048;
  const int64_t latencies = a.K / deep + (a.K % deep + 2047) / 2048;
  return values > 1 ? (double)((values - 1) * latencies) * 1.6 : 0.0;
}

// Us, here / tiles with the narrow product's launch, W not in the caches: bf16
// 128 x 4096 x 4096 27 / 45, 192 x 4096 x 4096 42 / 44, 256 x 4096 x 1024 20 / 33,
// 101 x 6848 x 832 25 / 43, 128 x 8192 x 8192 72 / 74; int8 128 x 4096 x 4096
// 21 / 38, 256 x 2048 x 2048 19 / 18.
double few_us(const AdapterArgs &a, bool q8) {
  const double blocks = (double)((a.M + kFewBlock - 1) / kFewBlock);
  return 6 + blocks * (double)a.K * (double)a.N * (q8 ? 1 : 2) / 3.2e6;
}

// Of M rows and of fewer, whatever ranges they are cut into: at most 16, at most the
// steps there are, and few_splits' workgroups hold 2^20 (8 bits: 2^21) sums beside
// half a range's.
int64_t few_work_bytes(int64_t M, int64_t K, int64_t N, int64_t r) {
  const int64_t m = M < kFewRows ? M : kFewRows;
  const int64_t steps = (K + 32 * kWaves - 1) / (32 * kWaves);
  const int64_t ranges = steps < 1 ? 1 : steps > 16 ? 16 : steps;
  const int64_t cut = ranges * m * N, full = ((int64_t)1 << 21) + m * N;
  return ((cut < full ? cut : full) * 4 + 255) / 256 * 256 + m * r * 4;
}

hipError_t launch_few(int dtype, const AdapterArgs &a, float *T, int tld, hipStream_t stream) {
  switch (dtype) {
    case TCU_F16_F32: return few<TCU_F16_F32, TCU_ELEM_F16, TCU_ELEM_F32, false>(a, T, tld, stream);
    case TCU_BF16_F32:
      return few<TCU_BF16_F32, TCU_ELEM_BF16, TCU_ELEM_F32, false>(a, T, tld, stream);
    case TCU_BF16_BF16:
      return few<TCU_BF16_BF16, TCU_ELEM_BF16, TCU_ELEM_BF16, false>(a, T, tld, stream);
    case TCU_I8_I32: return few<TCU_I8_I32, TCU_ELEM_BF16, TCU_ELEM_BF16, true>(a, T, tld, stream);
  }
  return hipErrorInvalidValue;
}

}  // namespace tcu

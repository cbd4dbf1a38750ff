// Products of matrices in 4 bits: C (M x N) = [C +] A (M x K) B (N x K)^T, and the
// same with a 16-bit left operand (tcu_mx4_gemm, tcu_mx4_linear).
//
// Both operands lie along the contracted index, so nothing is transposed: a lane's 32
// codes (16 bytes) and their scale are what the scaled matrix-core products take.
//   * mx4_tile_kernel: tiles of C, a stage of 256 values (128 bytes a row, a whole
//     line) copied straight to LDS while the one before it is multiplied.  Blocks of 32
//     x 32 over 64 values: the lower half-wave takes a stage's first group of 128, the
//     upper half its second, in four steps, so that the four scales of a lane are the
//     four bytes of one word, read from memory once a stage (the words of 32 rows lie
//     beside each other) and chosen by the instruction.
//   * mx4_few_kernel: few rows, bound by B's bytes: a workgroup takes 16 rows of B,
//     its waves share the contracted index, and their sums are added in LDS.
#include <algorithm>

#include "tcu_mx4_dev.h"

namespace tcu {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// The matrix cores' products of codes, with the scale in byte J of each lane's word.
__device__ __forceinline__ i32x8 wide(u32x4 v) {
  return i32x8{(int)v[0], (int)v[1], (int)v[2], (int)v[3], 0, 0, 0, 0};
}
template <int J>
__device__ __forceinline__ f32x16 mfma_k64(u32x4 w, u32x4 x, f32x16 d, unsigned ws, unsigned xs) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wide(w), wide(x), d, 4, 4, J, (int)ws, J,
                                                         (int)xs);
}
__device__ __forceinline__ f32x4 mfma_k128(u32x4 w, u32x4 x, f32x4 d, unsigned ws, unsigned xs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), d, 4, 4, 0, (int)ws, 0,
                                                          (int)xs);
}

// Four values of a row of C from column `col` on, the first `valid` of them inside.
template <int ELEM>
__device__ __forceinline__ void store4(unsigned char *p, f32x4 v, int valid, bool acc) {
  constexpr int ES = elem_bytes<ELEM>;
  typedef u32x2 u32x2_el __attribute__((aligned(2)));
  typedef f32x4 f32x4_el __attribute__((aligned(4)));
  if (valid >= 4 && ELEM == TCU_ELEM_F32) {
    if (acc) v += *(const f32x4_el *)p;
    *(f32x4_el *)p = v;
    return;
  }
  if (acc) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (e < valid) v[e] += elem_to_f32<ELEM>(p + e * ES);
  }
  if (valid >= 4 && ELEM != TCU_ELEM_F32) {
    const float x[8] = {v[0], v[1], v[2], v[3], 0.f, 0.f, 0.f, 0.f};
    const Raw8<ELEM> r = pack8<ELEM>(x);
    *(u32x2_el *)p = u32x2{r.v[0][0], r.v[0][1]};
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (e < valid) f32_to_elem<ELEM>(p + e * ES, v[e]);
}

// ---------------------------------------------------------------------- tiles
// kPart: sums of one range of the contracted index, binary32 [range][M][N] in work.
constexpr int kPart = 3;

struct TileArgs {
  Mx4GemmArgs g;
  int tiles_m, tiles_n, splits, stages_per_split;
};

template <int ELEM, int FM, int FN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void mx4_tile_kernel(TileArgs ta) {
  constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN, kWaves = WM * WN, kRows = BM + BN;
  constexpr int kLoads = kRows / 8 / kWaves, kStage = kRows * 128;
  __shared__ __attribute__((aligned(128))) unsigned char lds[2 * kStage];
  const Mx4GemmArgs &a = ta.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int wm = wave / WN, wn = wave % WN;

  // consecutive workgroups go round the 8 XCDs: each walks a run of tiles
  const int tiles = ta.tiles_m * ta.tiles_n;
  int id = blockIdx.x;
  const int split = id / tiles;
  id -= split * tiles;
  const int body = tiles & ~7;
  if (id < body) id = (id & 7) * (body >> 3) + (id >> 3);
  // in bands of kBand rows of tiles, column by column
  constexpr int kBand = 4;
  const int band = id / (kBand * ta.tiles_n), in_band = id - band * kBand * ta.tiles_n;
  const int band_rows = min(kBand, ta.tiles_m - band * kBand);
  const int64_t m0 = (int64_t)(band * kBand + in_band % band_rows) * BM;
  const int64_t n0 = (int64_t)(in_band / band_rows) * BN;

  const int groups = (int)mx4_groups(a.K);
  const int first = split * ta.stages_per_split;
  const int last = min((groups + 1) / 2, first + ta.stages_per_split);

  // The copies: 8 rows of 128 bytes each; 16-byte chunk c of row r lies at chunk
  // c ^ (r % 8), so that eight rows' same chunks fill the banks once.
  const unsigned char *src[kLoads];
  unsigned off[kLoads];
  const int chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int row8 = (wave * kLoads + i) * 8;
    const bool is_a = row8 < BM;
    const int64_t rows = is_a ? a.M : a.N, ld = is_a ? a.lda : a.ldb;
    const int64_t r = is_a ? m0 + row8 : n0 + (row8 - BM);
    const int64_t base = min(r, rows - 1), mine = min(r + (lane >> 3), rows - 1);
    src[i] = (is_a ? a.A : a.B) + base * ld;
    off[i] = (unsigned)((mine - base) * ld) + chunk * 16;
  }
  const unsigned lds0 = lds_addr(lds);
  auto issue = [&](int stage, int buf) {
    // the second half of the last stage may be missing: its scales are zero, and
    // the first half's codes stand in for it
    const unsigned back = 2 * stage + 1 >= groups && chunk >= 4 ? 64u : 0u;
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      dma_lds16_saddr(src[i] + (int64_t)stage * 128, off[i] - back,
                      lds0 + buf * kStage + (wave * kLoads + i) * 1024);
  };
  // scale words of the wave's blocks of rows: the half-wave's group of the stage
  const unsigned *as[FM], *bs[FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
    as[i] = a.as + min(m0 + (wm * FM + i) * 32 + l32, a.M - 1) + half * a.ldas;
#pragma unroll
  for (int i = 0; i < FN; ++i)
    bs[i] = a.bs + min(n0 + (wn * FN + i) * 32 + l32, a.N - 1) + half * a.ldbs;
  unsigned sa[FM], sb[FN], next_a[FM], next_b[FN];
  auto load_scales = [&](int stage) {
    const bool in = 2 * stage + half < groups;
#pragma unroll
    for (int i = 0; i < FM; ++i) next_a[i] = in ? as[i][(int64_t)(2 * stage) * a.ldas] : 0u;
#pragma unroll
    for (int i = 0; i < FN; ++i) next_b[i] = in ? bs[i][(int64_t)(2 * stage) * a.ldbs] : 0u;
  };
  auto take_scales = [&]() {
#pragma unroll
    for (int i = 0; i < FM; ++i) sa[i] = next_a[i];
#pragma unroll
    for (int i = 0; i < FN; ++i) sb[i] = next_b[i];
  };

  f32x16 acc[FM][FN];
#pragma unroll
  for (int i = 0; i < FM; ++i)
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
      for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;

  // a lane's chunk of step J: 4 half + J, where its row keeps it
  auto step = [&](auto jc, int buf) {
    constexpr int J = decltype(jc)::value;
    const int at = (((half << 2) + J) ^ (lane & 7)) * 16;
    const unsigned char *pa = lds + buf * kStage + (wm * FM * 32 + l32) * 128 + at;
    const unsigned char *pb = lds + buf * kStage + (BM + wn * FN * 32 + l32) * 128 + at;
    u32x4 x[FM], w[FN];
#pragma unroll
    for (int i = 0; i < FN; ++i) w[i] = *(const u32x4 *)(pb + i * 4096);
#pragma unroll
    for (int i = 0; i < FM; ++i) x[i] = *(const u32x4 *)(pa + i * 4096);
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = mfma_k64<J>(w[j], x[i], acc[i][j], sb[j], sa[i]);
  };

  if (first < last) {
    load_scales(first);
    issue(first, 0);
    __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
    asm volatile("s_barrier" ::: "memory");
    take_scales();
    int buf = 0;
    for (int t = first; t < last; ++t) {
      if (t + 1 < last) {
        load_scales(t + 1);
        issue(t + 1, buf ^ 1);
      }
      step(std::integral_constant<int, 0>{}, buf);
      step(std::integral_constant<int, 1>{}, buf);
      step(std::integral_constant<int, 2>{}, buf);
      step(std::integral_constant<int, 3>{}, buf);
      // this stage is read and the next one is there
      __builtin_amdgcn_s_waitcnt(0x0070);
      asm volatile("s_barrier" ::: "memory");
      take_scales();
      buf ^= 1;
    }
  }

  // lane: row l32 of a block, columns 8 q + 4 half ..
#pragma unroll
  for (int i = 0; i < FM; ++i) {
    const int64_t m = m0 + (wm * FM + i) * 32 + l32;
    if (m >= a.M) continue;
#pragma unroll
    for (int j = 0; j < FN; ++j) {
      const int64_t nb = n0 + (wn * FN + j) * 32 + 4 * half;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int64_t n = nb + 8 * q;
        const int valid = (int)min((int64_t)4, a.N - n);
        const f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2],
                         acc[i][j][4 * q + 3]};
        if (valid <= 0) continue;
        if constexpr (ELEM == kPart) {
          float *p = (float *)a.work + ((int64_t)split * a.M + m) * a.N + n;
          store4<TCU_ELEM_F32>((unsigned char *)p, v, valid, false);
        } else {
          store4<ELEM>((unsigned char *)a.C + (m * a.ldc + n) * elem_bytes<ELEM>, v, valid, a.accum);
        }
      }
    }
  }
}

// C = the ranges' sums, in their order.
template <int ELEM>
__global__ __launch_bounds__(256) void mx4_join_kernel(Mx4GemmArgs a, int splits) {
  const int64_t n = a.M * a.N, stride = (int64_t)gridDim.x * 256 * 4;
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; i < n; i += stride) {
    const float *p = (const float *)a.work + i;
    const int left = (int)min((int64_t)4, n - i);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    typedef f32x4 f32x4_el __attribute__((aligned(4)));
    for (int s = 0; s < splits; ++s) {
      if (left == 4) {
        v += *(const f32x4_el *)(p + s * n);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (e < left) v[e] += p[s * n + e];
      }
    }
    const int64_t m = i / a.N, c = i - m * a.N;
    constexpr int ES = elem_bytes<ELEM>;
    unsigned char *C = (unsigned char *)a.C;
    if (c + left <= a.N) {
      store4<ELEM>(C + (m * a.ldc + c) * ES, v, left, a.accum);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (e < left) {
          const int64_t me = (i + e) / a.N, ce = (i + e) - me * a.N;
          unsigned char *at = C + (me * a.ldc + ce) * ES;
          f32_to_elem<ELEM>(at, a.accum ? v[e] + elem_to_f32<ELEM>(at) : v[e]);
        }
      }
    }
  }
}

template <int ELEM, int FM, int FN, int WM, int WN>
hipError_t launch_tiles(const Mx4GemmArgs &a, int splits, hipStream_t stream) {
  constexpr int BM = 32 * FM * WM, BN = 32 * FN * WN;
  const int stages = (int)((mx4_groups(a.K) + 1) / 2);
  // threads of a launch count in 32 bits: more tiles than that in bands of rows (cut
  // products have few)
  const int64_t tiles_n = (a.N + BN - 1) / BN;
  const int64_t band = std::max<int64_t>(1, ((int64_t)1 << 22) / tiles_n) * BM;
  for (int64_t m = 0; m < a.M; m += band) {
    TileArgs t{a, 0, (int)tiles_n, splits, (stages + splits - 1) / splits};
    t.g.M = std::min(a.M - m, band);
    t.g.A += m * a.lda;
    t.g.as += m;
    if (ELEM != kPart) t.g.C = (unsigned char *)a.C + m * a.ldc * elem_bytes<ELEM>;
    t.tiles_m = (int)((t.g.M + BM - 1) / BM);
    mx4_tile_kernel<ELEM, FM, FN, WM, WN>
        <<<(unsigned)(t.tiles_m * tiles_n * splits), 64 * WM * WN, 0, stream>>>(t);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// -------------------------------------------------------------------- few rows
constexpr int kFewWaves = 16;

struct FewArgs {
  Mx4GemmArgs g;
  const unsigned char *X;   // 16-bit left operand
  int64_t ldx;
};

// XE: the left operand's element type, or -1: in 4 bits already.  MF: blocks of 16 rows.
template <int ELEM, int XE, int MF>
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(FewArgs fa) {
  const Mx4GemmArgs &a = fa.g;
  __shared__ float sums[kFewWaves][MF * 256];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int groups = (int)mx4_groups(a.K);
  const int64_t n = min(n0 + r16, a.N - 1);
  const unsigned char *pb = a.B + n * a.ldb + g * 16;
  const unsigned *ps = a.bs + n;
  f32x4 acc[MF];
#pragma unroll
  for (int f = 0; f < MF; ++f) acc[f] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int U = 2;   // groups in flight
  for (int t = wave; t < groups; t += kFewWaves * U) {
    u32x4 w[U], x[U][MF];
    unsigned ws[U], xs[U][MF];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = t + u * kFewWaves;
      const bool in = k < groups;
      w[u] = in ? *(const u32x4 *)(pb + (int64_t)k * 64) : u32x4{0u, 0u, 0u, 0u};
      ws[u] = in ? ps[(int64_t)k * a.ldbs] : 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = t + u * kFewWaves;
      const bool in = k < groups;
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        const int64_t m = min((int64_t)(f * 16 + r16), a.M - 1);
        if constexpr (XE < 0) {
          x[u][f] = in ? *(const u32x4 *)(a.A + m * a.lda + (int64_t)k * 64 + g * 16)
                       : u32x4{0u, 0u, 0u, 0u};
          xs[u][f] = (in ? a.as[(int64_t)k * a.ldas + m] : 0u) >> (8 * g);
        } else {
          // a lane's block of 32 values of its row, by itself
          const int64_t col = (int64_t)k * 128 + g * 32;
          const unsigned char *p = fa.X + (m * fa.ldx + col) * 2;
          Raw8<XE> raw[4];
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int64_t left = a.K - col - 8 * d;
            raw[d] = Raw8<XE>{};
            if (left > 0) raw[d] = load8<XE>(p + 16 * d, (int)min((int64_t)8, left));
          }
          float v[4][8];
          unsigned most = 0;
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            unpack8<XE>(raw[d], v[d]);
#pragma unroll
            for (int e = 0; e < 8; ++e) most = umax(most, abs_bits(v[d][e]));
          }
          xs[u][f] = scale_byte(most);
#pragma unroll
          for (int d = 0; d < 4; ++d) x[u][f][d] = codes8(v[d], xs[u][f]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int f = 0; f < MF; ++f)
        acc[f] = mfma_k128(w[u], x[u][f], acc[f], ws[u] >> (8 * g), xs[u][f]);
  }
  // lane: columns 4 g .. of row r16 of a block
#pragma unroll
  for (int f = 0; f < MF; ++f) *(f32x4 *)&sums[wave][(f * 16 + r16) * 16 + 4 * g] = acc[f];
  __syncthreads();
  // four columns of a row a thread, the waves' sums in their order
  const int t = threadIdx.x;
  if (t < MF * 64) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kFewWaves; ++i) v += *(const f32x4 *)&sums[i][t * 4];
    const int64_t m = t >> 2, c = n0 + (t & 3) * 4;
    const int valid = (int)min((int64_t)4, a.N - c);
    if (m < a.M && valid > 0)
      store4<ELEM>((unsigned char *)a.C + (m * a.ldc + c) * elem_bytes<ELEM>, v, valid, a.accum);
  }
}

template <int ELEM, int XE>
hipError_t launch_few_rows(const FewArgs &args, hipStream_t stream) {
  const int threads = 64 * kFewWaves;
  constexpr int64_t kCols = (int64_t)1 << 25;   // of a launch
  for (int64_t n = 0; n < args.g.N; n += kCols) {
    FewArgs f = args;
    f.g.N = std::min(args.g.N - n, kCols);
    f.g.B += n * f.g.ldb;
    f.g.bs += n;
    f.g.C = (unsigned char *)f.g.C + n * elem_bytes<ELEM>;
    const unsigned blocks = (unsigned)((f.g.N + 15) / 16);
    if (f.g.M <= 16)
      mx4_few_kernel<ELEM, XE, 1><<<blocks, threads, 0, stream>>>(f);
    else if (f.g.M <= 32)
      mx4_few_kernel<ELEM, XE, 2><<<blocks, threads, 0, stream>>>(f);
    else
      mx4_few_kernel<ELEM, XE, 4><<<blocks, threads, 0, stream>>>(f);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------ plan
constexpr int64_t kFewMax = 64;

// Where C has few tiles, ranges of the contracted index, each of at least four stages.
constexpr int kMaxCus = 256;
int splits_of(int64_t tiles, int64_t K, int num_cus) {
  const int64_t stages = (mx4_groups(K) + 1) / 2;
  return (int)std::max<int64_t>(1, std::min<int64_t>({std::min(num_cus, kMaxCus) / std::max<int64_t>(tiles, 1),
                                                      stages / 4, 16}));
}
int64_t tiles_of(int64_t M, int64_t N, int64_t bm, int64_t bn) {
  return ((M + bm - 1) / bm) * ((N + bn - 1) / bn);
}


template <int ELEM>
hipError_t gemm(const Mx4GemmArgs &a, hipStream_t stream, int num_cus) {
  if (a.M <= kFewMax) return launch_few_rows<ELEM, -1>(FewArgs{a, nullptr, 0}, stream);
  if (tiles_of(a.M, a.N, 256, 256) >= num_cus)
    return launch_tiles<ELEM, 4, 2, 2, 4>(a, 1, stream);
  const int splits = splits_of(tiles_of(a.M, a.N, 128, 128), a.K, num_cus);
  if (splits == 1) return launch_tiles<ELEM, 2, 2, 2, 2>(a, 1, stream);
  const hipError_t e = launch_tiles<kPart, 2, 2, 2, 2>(a, splits, stream);
  if (e != hipSuccess) return e;
  const int64_t blocks = std::min<int64_t>((a.M * a.N + 1023) / 1024, 4 * num_cus);
  mx4_join_kernel<ELEM><<<(unsigned)blocks, 256, 0, stream>>>(a, splits);
  return hipGetLastError();
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace

// X in 4 bits and its scales, then the ranges' sums: up to 16 ranges, and of few
// tiles up to one a compute unit.
int64_t mx4_work_bytes(int64_t M, int64_t K, int64_t N) {
  const int64_t x = M * mx4_row_bytes(K) + up16(4 * mx4_groups(K) * M);
  constexpr int64_t kMost = (int64_t)kMaxCus * 128 * 128;
  return x + (M * N < kMost / 16 ? 16 * M * N : kMost) * 4;
}

hipError_t launch_mx4_gemm(int elem, const Mx4GemmArgs &a, hipStream_t stream, int num_cus) {
  switch (elem) {
    case TCU_ELEM_F32: return gemm<TCU_ELEM_F32>(a, stream, num_cus);
    case TCU_ELEM_F16: return gemm<TCU_ELEM_F16>(a, stream, num_cus);
    default: return gemm<TCU_ELEM_BF16>(a, stream, num_cus);
  }
}

hipError_t launch_mx4_linear(int xelem, const void *X, int64_t ldx, int elem,
                             const Mx4GemmArgs &args, hipStream_t stream, int num_cus) {
  Mx4GemmArgs a = args;
  if (a.M <= 4) {
    const FewArgs f{a, (const unsigned char *)X, ldx};
    if (xelem == TCU_ELEM_F16)
      return elem == TCU_ELEM_F32 ? launch_few_rows<TCU_ELEM_F32, TCU_ELEM_F16>(f, stream)
                                  : launch_few_rows<TCU_ELEM_F16, TCU_ELEM_F16>(f, stream);
    return elem == TCU_ELEM_F32 ? launch_few_rows<TCU_ELEM_F32, TCU_ELEM_BF16>(f, stream)
                                : launch_few_rows<TCU_ELEM_BF16, TCU_ELEM_BF16>(f, stream);
  }
  unsigned char *w = (unsigned char *)a.work;
  const int64_t row = mx4_row_bytes(a.K);
  unsigned *s = (unsigned *)(w + a.M * row);
  const hipError_t e = launch_mx4_quant(
      xelem, Mx4QuantArgs{X, w, nullptr, s, nullptr, ldx, row, a.M, 0, 0, a.M, a.K}, stream);
  if (e != hipSuccess) return e;
  a.A = w;
  a.as = s;
  a.lda = row;
  a.ldas = a.M;
  a.work = w + a.M * row + up16(4 * mx4_groups(a.K) * a.M);
  return launch_mx4_gemm(elem, a, stream, num_cus);
}

}  // namespace tcu

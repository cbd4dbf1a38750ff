// Products of matrices in 4 bits: C (M x N) = [C +] A (M x K) B (N x K)^T, and the
// same with a 16-bit left operand (tcu_mx4_gemm, tcu_mx4_linear).
//
// Both operands lie along the contracted index, so nothing is transposed: a lane's 32
// codes (16 bytes) and their scale are what the scaled matrix-core products take.
//   * mx4_tile_kernel: tiles of C by a persistent grid, a stage of 256 values (128 bytes
//     a row, a whole line) copied straight to LDS while the one before it is multiplied.
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
__device__ __forceinline__ f32x4 mfma_k128(u32x4 w, u32x4 x, f32x4 d, unsigned ws, unsigned xs) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(wide(w), wide(x), d, 4, 4, J, (int)ws, J,
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

// The 4-byte form of dma_lds16_saddr: lane l's word lands at lds_base + 4 l.
__device__ __forceinline__ void dma_lds4_saddr(const void *gbase, unsigned voff,
                                               unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(voff), "s"(gbase), "s"(lds_base)
               : "memory", "m0");
}

// WM x WN waves of FM x FN blocks of 16 x 16 over 128 values, the two steps of a stage.
// Sixteen lanes (g = lane / 16) hold the stage's blocks of scales 2 g and 2 g + 1, one a
// step, so that their scales are neighbouring bytes of one word, chosen by the
// instruction.
//
// The loop runs over stages without a gap between tiles.  Step 0 of a stage is
// multiplied from registers while step 1's fragments are read into the registers that
// each row of products leaves; once the next stage is in LDS, step 1 likewise with the
// next stage's first fragments, and the copy of the stage after it is issued into the
// buffer that has been read.
//
// 8192 x 8192 x 8192 of random codes, bf16 out: 248 us in steady state (4.4 PFLOP/s), 192
// (5.4) on zeros, which the power limit does not slow; products from registers alone 174
// (6.0).  LDS is busy 2250 cycles of a stage's 3700 (reads 1735, copies 512), the matrix
// cores 2048.  Tried: blocks of 32 x 32 over 64 values (each instruction the same work,
// more power: 6.0 against 6.4 PFLOP/s from registers; 295 us without the stream across
// tiles, 80 of 340 bands of stores exposed); the order that the compiler chose (256);
// bands of 2 or 8 rows of tiles (258, 256); four waves of 128 x 128 (spills).
template <int ELEM, int FM, int FN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void mx4_tile_kernel(TileArgs ta) {
  constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN, kWaves = WM * WN;
  constexpr int kRows = (BM + BN) / kWaves, kCopies = kRows / 8, kAll = kCopies + 2;
  static_assert(kRows == 64 && BM % 64 == 0, "a wave copies 64 rows of one operand");
  constexpr int kCodes = (BM + BN) * 128;
  // (a group's scale words, and 16 more so that both groups' reads fill all banks)
  constexpr int kWords = (BM + BN + 16) * 4, kBuffer = kCodes + 2 * kWords;
  __shared__ __attribute__((aligned(128))) unsigned char lds[2 * kBuffer];
  const Mx4GemmArgs &a = ta.g;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, r16 = lane & 15, half = lane >> 5;
  const int wm = wave / WN, wn = wave % WN;
  const int tiles = ta.tiles_m * ta.tiles_n, items = tiles * ta.splits;
  const int groups = (int)mx4_groups(a.K), stages = (groups + 1) / 2;

  // Item id: a tile and a range of stages.
  struct Item {
    int64_t m, n;
    int first, last, split;
  };
  auto place = [&](int id) {
    // round by round of the grid: consecutive workgroups go round the 8 XCDs, each of
    // which takes a run of tiles
    const int grid = gridDim.x, round = id / grid;
    int v = id - round * grid;
    const int body = min(grid, items - round * grid) & ~7;
    if (v < body) v = (v & 7) * (body >> 3) + (v >> 3);
    v += round * grid;
    Item it;
    it.split = v / tiles;
    v -= it.split * tiles;
    // in bands of rows of tiles, column by column
    constexpr int kBand = 4;
    const int band = v / (kBand * ta.tiles_n), in_band = v - band * kBand * ta.tiles_n;
    const int rows = min(kBand, ta.tiles_m - band * kBand);
    it.m = (int64_t)(band * kBand + in_band % rows) * BM;
    it.n = (int64_t)(in_band / rows) * BN;
    it.first = it.split * ta.stages_per_split;
    it.last = min(stages, it.first + ta.stages_per_split);
    return it;
  };

  // The copies: a wave's 64 rows of A or of B, 8 rows of 128 bytes at a time; 16-byte
  // chunk c of row r lies at chunk c ^ (r / 2 % 8), so that 16 rows' same chunks fill the
  // banks once.  B's rows lie so that a lane's results are eight neighbouring columns:
  // row 16 b + 4 i + e of 32 holds column 8 i + 4 b + e.
  const bool is_a = wave < BM / 64;
  const int chunk = (lane & 7) ^ (lane >> 4);   // of the even copies; the odd ones: ^ 4
  const unsigned char *src;
  unsigned off[kCopies], word_off;
  const unsigned *const words = is_a ? a.as : a.bs;
  const int64_t words_pitch = is_a ? a.ldas : a.ldbs;
  auto aim = [&](const Item &it) {
    const int64_t rows = is_a ? a.M : a.N, ld = is_a ? a.lda : a.ldb;
    const int64_t top = is_a ? it.m + wave * 64 : it.n + (wave - BM / 64) * 64;
    // rows past the edge: the last one again
    const int64_t base = min(top, rows - 1);
    const int left = (int)min(rows - 1 - base, (int64_t)63), l8 = lane >> 3;
    src = (is_a ? a.A : a.B) + base * ld;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = is_a ? 8 * i + l8
                         : 32 * (i >> 2) + 16 * (i & 1) + 4 * ((i >> 1) & 1) + 8 * (l8 >> 2) + (l8 & 3);
      off[i] = (unsigned)min(r, left) * (unsigned)ld + (chunk ^ 4 * (i & 1)) * 16;
    }
    const int r = is_a ? lane : (lane & 32) + 8 * ((lane >> 2) & 3) + 4 * ((lane >> 4) & 1) + (lane & 3);
    word_off = 4u * (unsigned)(base + min(r, left));
  };
  const unsigned lds0 = lds_addr(lds);
  // copies [from, upto) of a stage: codes, then the first and the second group's words
  auto issue = [&](int stage, int buf, int from, int upto) {
    const bool whole = 2 * stage + 1 < groups;
    // the second half of the last stage may be missing: its scales are cleared when they
    // are read, and the first half's codes stand in for it
    const unsigned back0 = !whole && chunk >= 4 ? 64u : 0u;
    const unsigned back1 = !whole && chunk < 4 ? 64u : 0u;
    const unsigned to = lds0 + buf * kBuffer;
#pragma unroll
    for (int i = from; i < upto; ++i) {
      if (i < kCopies)
        dma_lds16_saddr(src + (int64_t)stage * 128, off[i] - (i & 1 ? back1 : back0),
                        to + (wave * kCopies + i) * 1024);
      else
        dma_lds4_saddr(words + (int64_t)(2 * stage + (i > kCopies && whole)) * words_pitch,
                       word_off, to + kCodes + (i - kCopies) * kWords + wave * 256);
    }
  };

  f32x4 acc[FM][FN];
  u32x4 x[FM], w[2][FN];
  unsigned sa[FM], sb[FN], next_a[FM], next_b[FN];
  const unsigned at0 = ((2 * g) ^ (r16 >> 1)) * 16, at1 = ((2 * g + 1) ^ (r16 >> 1)) * 16;
  const unsigned row_a = (wm * 16 * FM + r16) * 128, row_b = (BM + wn * 16 * FN + r16) * 128;
  auto read_x = [&](int i, int s, int buf) {
    x[i] = *(const u32x4 *)(lds + buf * kBuffer + (row_a + (s ? at1 : at0)) + i * 2048);
  };
  auto read_w = [&](int j, int s, int buf) {
    w[s][j] = *(const u32x4 *)(lds + buf * kBuffer + (row_b + (s ? at1 : at0)) + j * 2048);
  };
  auto read_scales = [&](int buf, bool whole) {
    const unsigned char *p = lds + buf * kBuffer + kCodes + half * kWords + r16 * 4;
    const unsigned keep = whole || half == 0 ? ~0u : 0u;
#pragma unroll
    for (int i = 0; i < FM; ++i)
      next_a[i] = (*(const unsigned *)(p + (wm * FM + i) * 64) & keep) >> (16 * (g & 1));
#pragma unroll
    for (int j = 0; j < FN; ++j)
      next_b[j] = (*(const unsigned *)(p + (BM + (wn * FN + j) * 16) * 4) & keep) >> (16 * (g & 1));
  };
  auto take_scales = [&]() {
#pragma unroll
    for (int i = 0; i < FM; ++i) sa[i] = next_a[i];
#pragma unroll
    for (int j = 0; j < FN; ++j) sb[j] = next_b[j];
  };
  auto multiply = [&](auto step, int i) {
    constexpr int S = decltype(step)::value;
#pragma unroll
    for (int j = 0; j < FN; ++j)
      acc[i][j] = mfma_k128<S>(w[S][j], x[i], acc[i][j], sb[j], sa[i]);
    // keeps a row of products before what follows in memory (its fragment's next read)
#pragma unroll
    for (int j = 0; j < FN; ++j) asm volatile("" : "+v"(acc[i][j])::"memory");
  };
  auto clear = [&]() {
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
      for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  };
  const std::integral_constant<int, 0> step0{};
  const std::integral_constant<int, 1> step1{};

  int id = blockIdx.x, next_id = id;   // items: multiplied, and copied
  Item now = place(id);
  aim(now);
  int t = now.first, ahead = now.first, end = now.last;   // stages: multiplied, to copy, its item's end
  // past an item's last stage the next one's first (after the last item: its own again,
  // which nothing reads)
  auto advance = [&]() {
    if (ahead < end) return;
    if (next_id + (int)gridDim.x < items) next_id += gridDim.x;
    const Item it = place(next_id);
    aim(it);
    ahead = it.first;
    end = it.last;
  };
  issue(ahead++, 0, 0, kAll);
  advance();
  int coming = ahead;   // the stage after the one in registers
  issue(ahead++, 1, 0, kAll);
  // (the second stage may be on its way)
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(kAll) : "memory");
#pragma unroll
  for (int j = 0; j < FN; ++j) read_w(j, 0, 0);
#pragma unroll
  for (int i = 0; i < FM; ++i) read_x(i, 0, 0);
  read_scales(0, 2 * t + 1 < groups);
  take_scales();
  clear();
  // 16-byte stores of a wave's part of a whole tile, at the least
  constexpr int kStores = FM * FN * 4 * (ELEM == kPart ? 4 : elem_bytes<ELEM>) / 16;
  static_assert(kStores < 64, "the counter's range");
  bool stored = false;
  int buf = 0;
  while (true) {
    advance();
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      multiply(step0, i);
      read_x(i, 1, buf);
      if (2 * i < FN) {
        read_w(2 * i, 1, buf);
        read_w(2 * i + 1, 1, buf);
      }
    }
    multiply(step1, 0);
    // the next stage is there (the last tile's stores may be on their way), this one read
    if (stored)
      asm volatile("s_waitcnt vmcnt(%0)" ::"i"(kStores) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    const int other = buf ^ 1;
    read_scales(other, 2 * coming + 1 < groups);
    read_x(0, 0, other);
    read_w(0, 0, other);
    if (FN > FM) read_w(FN - 1, 0, other);
    constexpr int kPer = (kAll + FM - 2) / (FM - 1);
#pragma unroll
    for (int i = 1; i < FM; ++i) {
      multiply(step1, i);
      read_x(i, 0, other);
      if (i < FN) read_w(i, 0, other);
      issue(ahead, buf, (i - 1) * kPer, i * kPer < kAll ? i * kPer : kAll);
    }
    take_scales();
    // reads between the products, none of them waited for
    if constexpr (FM == 8) {
      __builtin_amdgcn_sched_group_barrier(0x100, 2 + (FM + FN) / 2, 0);
#pragma unroll
      for (int i = 1; i < FM; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, FN, 0);
        if (i < FN)
          __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        else
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
    buf = other;
    coming = ahead++;
    stored = false;
    if (++t < now.last) continue;
    // lane: row r16 of a block, eight columns of each pair of blocks
    const int64_t cm = now.m + wm * 16 * FM, cn = now.n + wn * 16 * FN;
    const bool inside = cm + 16 * FM <= a.M && cn + 16 * FN <= a.N;
    constexpr int OE = ELEM == kPart ? TCU_ELEM_F32 : ELEM, ES = elem_bytes<OE>;
    unsigned char *const C = ELEM == kPart
                                 ? (unsigned char *)a.work + (int64_t)now.split * a.M * a.N * 4
                                 : (unsigned char *)a.C;
    const int64_t ldc = ELEM == kPart ? a.N : a.ldc;
    const bool accum = ELEM != kPart && a.accum;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      const int64_t m = cm + i * 16 + r16;
#pragma unroll
      for (int p = 0; p < FN / 2; ++p) {
        const int64_t n = cn + 32 * p + 8 * g;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = acc[i][2 * p + (e >> 2)][e & 3];
        unsigned char *c = C + (m * ldc + n) * ES;
        if (inside && !accum) {
          store8<OE>(c, v, 8);
        } else if (m < a.M && n < a.N) {
          const int valid = (int)min((int64_t)8, a.N - n);
          if (accum) {
            float u[8];
            unpack8<OE>(load8<OE>(c, valid), u);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += u[e];
          }
          store8<OE>(c, v, valid);
        }
      }
    }
    id += gridDim.x;
    if (id >= items) break;
    // (an edge may have stored less than the next wait allows for)
    stored = inside && !accum;
    now = place(id);
    t = now.first;
    clear();
  }
  // the copies that nothing reads have landed
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
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
hipError_t launch_tiles(const Mx4GemmArgs &a, int splits, hipStream_t stream, int num_cus) {
  constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN;
  const int stages = (int)((mx4_groups(a.K) + 1) / 2);
  TileArgs t{a, (int)((a.M + BM - 1) / BM), (int)((a.N + BN - 1) / BN), splits,
             (stages + splits - 1) / splits};
  t.splits = (stages + t.stages_per_split - 1) / t.stages_per_split;   // none empty
  // as many workgroups as the compute units' LDS holds
  constexpr int kPerCu = BM + BN == 512 ? 1 : BM + BN == 256 ? 2 : 4;
  const int64_t items = (int64_t)t.tiles_m * t.tiles_n * t.splits;
  mx4_tile_kernel<ELEM, FM, FN, WM, WN>
      <<<(unsigned)std::min<int64_t>(items, (int64_t)kPerCu * num_cus), 64 * WM * WN, 0, stream>>>(t);
  return hipGetLastError();
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
        acc[f] = mfma_k128<0>(w[u], x[u][f], acc[f], ws[u] >> (8 * g), xs[u][f]);
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
  const int64_t blocks = std::min<int64_t>((a.M * a.N + 1023) / 1024, 4 * num_cus);
  if (a.K == 0) {   // zeros: the sums of no ranges
    mx4_join_kernel<ELEM><<<(unsigned)blocks, 256, 0, stream>>>(a, 0);
    return hipGetLastError();
  }
  if (a.M <= kFewMax) return launch_few_rows<ELEM, -1>(FewArgs{a, nullptr, 0}, stream);
  if (tiles_of(a.M, a.N, 256, 256) >= num_cus)
    return launch_tiles<ELEM, 8, 4, 2, 4>(a, 1, stream, num_cus);
  const int64_t tiles = tiles_of(a.M, a.N, 128, 128);
  if (tiles < num_cus && tiles_of(a.M, a.N, 64, 64) <= 4 * num_cus && mx4_groups(a.K) < 32)
    return launch_tiles<ELEM, 4, 2, 1, 2>(a, 1, stream, num_cus);
  const int splits = splits_of(tiles, a.K, num_cus);
  if (splits == 1) return launch_tiles<ELEM, 4, 4, 2, 2>(a, 1, stream, num_cus);
  const hipError_t e = launch_tiles<kPart, 4, 4, 2, 2>(a, splits, stream, num_cus);
  if (e != hipSuccess) return e;
  const int stages = (int)((mx4_groups(a.K) + 1) / 2), per = (stages + splits - 1) / splits;
  mx4_join_kernel<ELEM><<<(unsigned)blocks, 256, 0, stream>>>(a, (stages + per - 1) / per);
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

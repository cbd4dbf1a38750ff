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
#include <cmath>

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
// 8192 x 8192 x 8192, bf16 out, us in steady state: 240 to 258 on random codes (4.3 to 4.6
// PFLOP/s, by the card), 187 (5.9) on zeros, in the same 0.47 million cycles: power keeps the
// clock at 1.95 GHz on random codes, 2.46 on zeros.  The matrix cores are busy in 56 % of
// them, so the order of reads and products bounds both: of a stage's 3650 cycles LDS is busy
// 2250 (reads 1735, copies 512) and the matrix cores 2048.  The same instructions from
// registers: 153 on random codes (busy 95 %, 1.82 GHz), 114 on zeros; a better order would so
// give part of its cycles back to the clock.  The copies are not waited for: without
// their wait the time is the same.  Tried, same product:
// products of 32 x 32 over 64 values (each instruction the same work at more power: from
// registers 5 % slower); the order that the compiler chose (256 against 248); bands of 2 or 8 rows of
// tiles (258, 256); a stage's copies issued at once or in two parts (262 against 258, on
// zeros 198 against 189); four waves of 128 x 128 (their registers spill).
template <int ELEM, int FM, int FN, int WM, int WN, int KG>
__global__ __launch_bounds__(64 * WM * WN * KG) void mx4_tile_kernel(TileArgs ta) {
  constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN, kWaves = WM * WN;
  constexpr int kRows = (BM + BN) / kWaves, R = 2, kCopies = kRows / 8, kAll = kCopies + 2;
  static_assert(kRows == 64 && BM % 64 == 0, "a wave copies 64 rows of one operand");
  constexpr int kCodes = (BM + BN) * 128;
  // (a group's scale words, and 16 more so that both groups' reads fill all banks)
  constexpr int kWords = (BM + BN + 16) * 4, kBuffer = kCodes + 2 * kWords;
  __shared__ __attribute__((aligned(128))) unsigned char lds[R * KG * kBuffer];
  const Mx4GemmArgs &a = ta.g;
  const int lane = threadIdx.x & 63;
  const int kg = __builtin_amdgcn_readfirstlane(threadIdx.x / (64 * kWaves));
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - kg * kWaves;
  const int g = lane >> 4, r16 = lane & 15, half = lane >> 5;
  const int wm = wave / WN, wn = wave % WN;
  const int tiles = ta.tiles_m * ta.tiles_n, items = tiles * ta.splits;
  const int groups = (int)mx4_groups(a.K), stages = (groups + 1) / 2;

  // Item id: a tile and a range of stages.
  struct Item {
    int64_t m, n;
    int first, last, split;
    __device__ int rounds() const { return (last - first + KG - 1) / KG; }
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
  const unsigned *words;
  const int64_t words_pitch = is_a ? a.ldas : a.ldbs;
  int stage, last;   // the group's stage that is copied next, the end of its item's
  auto aim = [&](const Item &it) {
    stage = it.first + kg;
    last = it.last;
    const int at = min(stage, last - 1);
    const int64_t rows = is_a ? a.M : a.N, ld = is_a ? a.lda : a.ldb;
    const int64_t top = is_a ? it.m + wave * 64 : it.n + (wave - BM / 64) * 64;
    // rows past the edge: the last one again
    const int64_t base = min(top, rows - 1);
    const int left = (int)min(rows - 1 - base, (int64_t)63), l8 = lane >> 3;
    src = (is_a ? a.A : a.B) + base * ld + (int64_t)at * 128;
    words = (is_a ? a.as : a.bs) + (int64_t)(2 * at) * words_pitch;
#pragma unroll
    for (int i = 0; i < kCopies; ++i) {
      const int r = is_a ? 8 * i + l8
                         : 32 * (i >> 2) + 16 * (i & 1) + 4 * ((i >> 1) & 1) + 8 * (l8 >> 2) + (l8 & 3);
      off[i] = (unsigned)min(r, left) * (unsigned)ld + (chunk ^ 4 * (i & 1)) * 16;
    }
    const int r = is_a ? lane : (lane & 32) + 8 * ((lane >> 2) & 3) + 4 * ((lane >> 4) & 1) + (lane & 3);
    word_off = 4u * (unsigned)(base + min(r, left));
  };
  unsigned char *const ring = lds + kg * kBuffer;   // buffer r at r KG buffers
  const unsigned lds0 = lds_addr(ring);
  // copies [from, upto) of the next stage: codes, then the first and the second group's
  // words
  auto issue = [&](int buf, int from, int upto) {
    // the second half of the last stage may be missing: its scales are cleared when they
    // are read, and the first half's codes stand in for it
    const bool whole = stage < groups >> 1;
    const unsigned back0 = !whole && chunk >= 4 ? 64u : 0u;
    const unsigned back1 = !whole && chunk < 4 ? 64u : 0u;
    const unsigned to = lds0 + buf * KG * kBuffer;
#pragma unroll
    for (int i = from; i < upto; ++i) {
      if (i < kCopies)
        dma_lds16_saddr(src, off[i] - (i & 1 ? back1 : back0), to + (wave * kCopies + i) * 1024);
      else
        dma_lds4_saddr(i > kCopies && whole ? words + words_pitch : words, word_off,
                       to + kCodes + (i - kCopies) * kWords + wave * 256);
    }
  };
  // (past the range's end its last stage again, whose scales are then not taken)
  auto step_on = [&]() {
    stage += KG;
    if (KG == 1 || stage < last) {
      src += 128 * KG;
      words += 2 * KG * words_pitch;
    }
  };

  f32x4 acc[FM][FN];
  u32x4 x[FM], w[2][FN];
  unsigned sa[FM], sb[FN], next_a[FM], next_b[FN];
  const unsigned at0 = ((2 * g) ^ (r16 >> 1)) * 16, at1 = ((2 * g + 1) ^ (r16 >> 1)) * 16;
  const unsigned row_a = (wm * 16 * FM + r16) * 128, row_b = (BM + wn * 16 * FN + r16) * 128;
  auto read_x = [&](int i, int s, int buf) {
    x[i] = *(const u32x4 *)(ring + buf * KG * kBuffer + (row_a + (s ? at1 : at0)) + i * 2048);
  };
  auto read_w = [&](int j, int s, int buf) {
    w[s][j] = *(const u32x4 *)(ring + buf * KG * kBuffer + (row_b + (s ? at1 : at0)) + j * 2048);
  };
  auto read_scales = [&](int buf, int stage, int end) {
    const unsigned char *p = ring + buf * KG * kBuffer + kCodes + half * kWords + r16 * 4;
    const int there = KG > 1 && stage >= end ? 0 : min(groups - 2 * stage, 2);   // groups
    const unsigned keep = half < there ? ~0u : 0u;
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
  int left = now.rounds(), to_copy = left;   // rounds of the items: to multiply, to copy
  // past an item's last round the next one's first (after the last item: its own again,
  // which nothing reads)
  auto advance = [&]() {
    if (to_copy > 0) return;
    if (next_id + (int)gridDim.x < items) next_id += gridDim.x;
    const Item it = place(next_id);
    aim(it);
    to_copy = it.rounds();
  };
  issue(0, 0, kAll);
  step_on();
  --to_copy;
  advance();
  int coming = stage;   // the stage after it
  issue(1, 0, kAll);
  step_on();
  --to_copy;
  // (the second round may be on its way)
  asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"i"(kAll) : "memory");
#pragma unroll
  for (int j = 0; j < FN; ++j) read_w(j, 0, 0);
#pragma unroll
  for (int i = 0; i < FM; ++i) read_x(i, 0, 0);
  read_scales(0, now.first + kg, now.last);
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
    read_scales(other, coming, now.last);   // (only one item's ranges end inside a round)
    read_x(0, 0, other);
    read_w(0, 0, other);
    if (FN > FM) read_w(FN - 1, 0, other);
    constexpr int kPer = (kAll + FM - 2) / (FM - 1);
#pragma unroll
    for (int i = 1; i < FM; ++i) {
      multiply(step1, i);
      read_x(i, 0, other);
      if (i < FN) read_w(i, 0, other);
      issue(buf, (i - 1) * kPer, i * kPer < kAll ? i * kPer : kAll);
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
    coming = stage;
    step_on();
    --to_copy;
    stored = false;
    if (--left > 0) continue;
    // lane: row r16 of a block, eight columns of each pair of blocks
    const int64_t cm = now.m + wm * 16 * FM, cn = now.n + wn * 16 * FN;
    const bool inside = cm + 16 * FM <= a.M && cn + 16 * FN <= a.N;
    constexpr int OE = ELEM == kPart ? TCU_ELEM_F32 : ELEM, ES = elem_bytes<OE>;
    unsigned char *const C = ELEM == kPart
                                 ? (unsigned char *)a.work + (int64_t)now.split * a.M * a.N * 4
                                 : (unsigned char *)a.C;
    const int64_t ldc = ELEM == kPart ? a.N : a.ldc;
    const bool accum = ELEM != kPart && a.accum;
    f32x4 *const sums = (f32x4 *)lds;
    if constexpr (KG > 1) {
      // (its only item: nothing is on its way to the ring or read from it any more)
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
#pragma unroll
      for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
          sums[(((kg * kWaves + wave) * FM + i) * FN + j) * 64 + lane] = acc[i][j];
      __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < FM; ++i) {
      if (KG > 1 && i / (FM / KG) != kg) continue;   // a group's share of the rows
      const int64_t m = cm + i * 16 + r16;
#pragma unroll
      for (int p = 0; p < FN / 2; ++p) {
        const int64_t n = cn + 32 * p + 8 * g;
        float v[8];
        if constexpr (KG == 1) {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = acc[i][2 * p + (e >> 2)][e & 3];
        } else {
          // the groups' sums, in their order
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            f32x4 u = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KG; ++k)
              u += sums[(((k * kWaves + wave) * FM + i) * FN + 2 * p + j) * 64 + lane];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * j + e] = u[e];
          }
        }
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
    if (KG > 1 || id >= items) break;
    // (an edge may have stored less than the next wait allows for)
    stored = inside && !accum;
    now = place(id);
    left = now.rounds();
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

template <int ELEM, int FM, int FN, int WM, int WN, int KG>
hipError_t launch_tiles(const Mx4GemmArgs &a, int splits, hipStream_t stream, int num_cus) {
  constexpr int BM = 16 * FM * WM, BN = 16 * FN * WN;
  const int stages = (int)((mx4_groups(a.K) + 1) / 2);
  TileArgs t{a, (int)((a.M + BM - 1) / BM), (int)((a.N + BN - 1) / BN), splits,
             (stages + splits - 1) / splits};
  t.splits = (stages + t.stages_per_split - 1) / t.stages_per_split;   // none empty
  // as many workgroups as the compute units' LDS holds
  constexpr int kPerCu = (160 << 10) / (2 * KG * ((BM + BN) * 136 + 128));
  const int64_t items = (int64_t)t.tiles_m * t.tiles_n * t.splits;
  // (groups of waves that share the contracted index take one item a workgroup)
  mx4_tile_kernel<ELEM, FM, FN, WM, WN, KG>
      <<<(unsigned)(KG > 1 ? items : std::min<int64_t>(items, (int64_t)kPerCu * num_cus)),
         64 * WM * WN * KG, 0, stream>>>(t);
  return hipGetLastError();
}

// -------------------------------------------------------------------- few rows
constexpr int kFewWaves = 16;

struct FewArgs {
  Mx4GemmArgs g;
  const unsigned char *X;   // 16-bit left operand
  int64_t ldx;
};

// Up to four rows: four lanes each (row r16 / 4) hold eight values of a block, and bring
// them together in registers; each row is then four columns of the products.
template <int XE, bool kWhole>
__device__ __forceinline__ u32x4 quad_codes(const unsigned char *row, int64_t col, int64_t K,
                                            unsigned &byte) {
  const int64_t at = col + (threadIdx.x & 3) * 8;
  Raw8<XE> raw = Raw8<XE>{};
  if (kWhole || at < K) raw = load8<XE>(row + at * 2, kWhole ? 8 : (int)min((int64_t)8, K - at));
  float v[8];
  unpack8<XE>(raw, v);
  unsigned most = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) most = umax(most, abs_bits(v[e]));
  most = quad_max(most);
  byte = scale_byte(most);
  const unsigned c = codes8(v, byte, __any(scale_low(most)));
  return u32x4{dpp<0x00>(c), dpp<0x55>(c), dpp<0xAA>(c), dpp<0xFF>(c)};
}

// XE: the left operand's element type (of up to four rows), or -1: in 4 bits already.
// MF: blocks of 16 rows; NB: blocks of 16 rows of B.  A wave takes pairs of groups of 128
// values: whole lines.  Bound by B's bytes and the latency of a wave's first (us in a row of
// launches, B from memory / in the last cache: a 16-bit row 1 x 4096 x 4096 5.3 / 4.2, B 8.9
// MB; 16 x 8192 x 8192 11.7 / 9.2, B 35.7 MB, 3.1 / 3.9 TB/s with launch and end).
template <int ELEM, int XE, int MF, int NB>
__global__ __launch_bounds__(64 * kFewWaves) void mx4_few_kernel(FewArgs fa) {
  const Mx4GemmArgs &a = fa.g;
  __shared__ f32x4 sums[kFewWaves][NB][MF * 64];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int r16 = lane & 15, g = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * NB);
  const int groups = (int)mx4_groups(a.K);
  const unsigned char *pb[NB], *px[MF];
  const unsigned *ps[NB], *pxs[MF];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    const int64_t n = min(n0 + b * 16 + r16, a.N - 1);
    pb[b] = a.B + n * a.ldb + g * 16;
    ps[b] = a.bs + n;
  }
#pragma unroll
  for (int f = 0; f < MF; ++f) {
    const int64_t m = min((int64_t)(f * 16 + (XE < 0 ? r16 : r16 >> 2)), a.M - 1);
    px[f] = XE < 0 ? a.A + m * a.lda + g * 16 : fa.X + m * fa.ldx * 2;
    pxs[f] = a.as + m;
  }
  f32x4 acc[MF][NB];
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int b = 0; b < NB; ++b) acc[f][b] = f32x4{0.f, 0.f, 0.f, 0.f};
  constexpr int U = 2;   // groups in flight (4: the same)
  for (int t = wave * U; t < groups; t += kFewWaves * U) {
    u32x4 w[U][NB], x[U][MF];
    unsigned ws[U][NB], xs[U][MF];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // (past the end: the last group with no scale)
      const int k = min(t + u, groups - 1);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        w[u][b] = *(const u32x4 *)(pb[b] + (int64_t)k * 64);
        ws[u][b] = ps[b][(int64_t)k * a.ldbs];
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = min(t + u, groups - 1);
      const bool in = t + u < groups;
#pragma unroll
      for (int f = 0; f < MF; ++f) {
        if constexpr (XE < 0) {
          x[u][f] = *(const u32x4 *)(px[f] + (int64_t)k * 64);
          xs[u][f] = pxs[f][(int64_t)k * a.ldas] >> (8 * g);
        } else {
          const int64_t col = (int64_t)k * 128 + g * 32;
          x[u][f] = (int64_t)(k + 1) * 128 <= a.K
                        ? quad_codes<XE, true>(px[f], col, a.K, xs[u][f])
                        : quad_codes<XE, false>(px[f], col, a.K, xs[u][f]);
        }
        if (!in) xs[u][f] = 0u;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) ws[u][b] = in ? ws[u][b] >> (8 * g) : 0u;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int f = 0; f < MF; ++f)
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[f][b] = mfma_k128<0>(w[u][b], x[u][f], acc[f][b], ws[u][b], xs[u][f]);
  }
  // lane: columns 4 g .. of row r16 of a block
#pragma unroll
  for (int f = 0; f < MF; ++f)
#pragma unroll
    for (int b = 0; b < NB; ++b) sums[wave][b][(f * 16 + r16) * 4 + g] = acc[f][b];
  __syncthreads();
  // four columns of a row a thread, the waves' sums in their order
  for (int t = threadIdx.x; t < NB * MF * 64; t += 64 * kFewWaves) {
    const int b = t / (MF * 64), i = t % (MF * 64);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kFewWaves; ++k) v += sums[k][b][i];
    if (XE >= 0 && (i >> 2 & 3) != 0) continue;
    const int64_t m = XE < 0 ? i >> 2 : i >> 4, c = n0 + b * 16 + (i & 3) * 4;
    const int valid = (int)min((int64_t)4, a.N - c);
    if (m < a.M && valid > 0)
      store4<ELEM>((unsigned char *)a.C + (m * a.ldc + c) * elem_bytes<ELEM>, v, valid, a.accum);
  }
}

template <int ELEM, int XE>
hipError_t launch_few_rows(const FewArgs &args, hipStream_t stream, int num_cus) {
  const int threads = 64 * kFewWaves;
  constexpr int64_t kCols = (int64_t)1 << 25;   // of a launch
  for (int64_t n = 0; n < args.g.N; n += kCols) {
    FewArgs f = args;
    f.g.N = std::min(args.g.N - n, kCols);
    f.g.B += n * f.g.ldb;
    f.g.bs += n;
    f.g.C = (unsigned char *)f.g.C + n * elem_bytes<ELEM>;
    const auto go = [&](auto mf, auto nb) {
      constexpr int MF = decltype(mf)::value, NB = decltype(nb)::value;
      mx4_few_kernel<ELEM, XE, MF, NB>
          <<<(unsigned)((f.g.N + 16 * NB - 1) / (16 * NB)), threads, 0, stream>>>(f);
    };
    const auto rows = [&](auto nb) {
      if (XE >= 0 || f.g.M <= 16)
        go(std::integral_constant<int, 1>{}, nb);
      else if (f.g.M <= 32)
        go(std::integral_constant<int, 2>{}, nb);
      else
        go(std::integral_constant<int, 4>{}, nb);
    };
    // Two blocks of B's rows share what is read of the left operand, where a workgroup of
    // 32 is left for every compute unit (us, 256 of them, N = K = 8192, one block / two: 16
    // rows 11.9 / 10.9, 32 16.0 / 13.9, one 16-bit row 12.8 / 10.5, one row in 4 bits 9.9 /
    // 11.1; 16 x 4096 x 4096 4.5 / 6.8).
    if (f.g.N >= 32 * (int64_t)num_cus && (XE >= 0 || f.g.M > 8))
      rows(std::integral_constant<int, 2>{});
    else
      rows(std::integral_constant<int, 1>{});
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// ------------------------------------------------------------------------ plan
// The few-row kernel's time in microseconds (us, that / measured on two cards, B from memory:
// 16 x 4096 x 4096 4.8 / 4.5 and 5.0, 32 x 8192 x 8192 13.8 / 13.9 and 14.6, 64 x 1024 x 4096
// 3.8 / 4.4 and 5.1, 64 x 4096 x 4096 7.8 / 8.3 and 8.7, 64 x 8192 x 4096 13.3 / 15.2).  The
// tiles' time below is fitted on B in the caches; from memory they take longer, the fewer
// rows share it (32 x 8192 x 8192 12.9 and 15.9).
constexpr int64_t kFewMax = 64;
double few_us(int64_t M, int64_t K, int64_t N, int num_cus) {
  const double cus = num_cus / 256.0;
  const double strips =
      N >= 32 * (int64_t)num_cus ? N / (4200.0 * cus) : std::max(1.0, N / (3500.0 * cus));
  return 2.4 + K / 1024.0 * (0.3 + 0.0135 * M) * strips;
}
double cold_us(int64_t K, int64_t N) { return K * N * 0.5 * 8e-8; }
// What a linear layer's few-row kernel brings to 4 bits itself: up to four rows, of which
// its quads of lanes hold one each (more have no such form), and of K values up to where every
// workgroup's own conversions cost what a launch does (us from memory, own / two launches:
// 1 x 4096 x 4096 5.3 / 6.7, 4 x 4096 x 4096 5.4 / 6.9, 4 x 8192 x 8192 11.7 / 13.1, 4 x 16384 x
// 4096 13.4 / 13.3, 4 x 32768 x 4096 22.9 / 20.9, 4 x 32768 x 1024 19.5 / 17.5).
constexpr int64_t kFewOwn = 4, kFewOwnK = 16384;

// The tile kernel's variants and what their time in microseconds is made of: a call, a
// round of stages on a compute unit that has room (`alone`) and where all are full (for
// each item of a compute unit), the stores of an item.  Fitted to 96 products of 16 to
// 4096 rows, K 512, 2048 and 8192: 6 % off in the mean; the variant it picks is 0.6 % slower
// than the fastest.
struct Variant {
  int tile, groups, per_cu;
  double call, alone, full, item;
};
constexpr Variant kVariants[] = {{256, 1, 1, 1.3, 1.28, 1.79, 7.6}, {128, 1, 2, 2.4, 1.10, 0.95, 2.4},
                                 {128, 2, 1, 1.6, 0.83, 1.16, 5.6}, {64, 1, 4, 2.4, 0.70, 0.29, 1.6},
                                 {64, 2, 2, 1.0, 0.65, 0.53, 4.0},  {64, 4, 1, 1.9, 0.70, 0.94, 4.0}};

int64_t tiles_of(int64_t M, int64_t N, int64_t tile) {
  return ((M + tile - 1) / tile) * ((N + tile - 1) / tile);
}
double tiles_us(const Variant &v, int64_t M, int64_t N, int64_t stages, int num_cus) {
  const double items = (double)tiles_of(M, N, v.tile), full = items / num_cus;
  if (v.groups > 1 && items > (1 << 22)) return 1e300;   // one item a workgroup of 512 threads
  const double batches = std::ceil(std::ceil(full) / v.per_cu);
  return v.call + std::ceil((double)stages / v.groups) * std::max(batches * v.alone, full * v.full) +
         batches * v.item;
}

// Ranges of the contracted index where C has few tiles and it is long: the last variant
// for each, their sums added by a second launch (us: 100 x 65536 x 64 14 to 15, 512 x
// 65536 x 512 26 to 27; uncut 46 and 93 by the times above).
constexpr int64_t kRangeValues = (int64_t)1 << 22;   // of all ranges' sums, at most
int ranges_of(int64_t M, int64_t N, int64_t stages, int num_cus, double &us) {
  int best = 1;
  for (int s = 2; s <= 16 && s * M * N <= kRangeValues && stages / s >= 16; s *= 2) {
    const double t = tiles_us(kVariants[5], M * s, N, (stages + s - 1) / s, num_cus) + 3.0 +
                     s * M * N * 2e-6;
    if (t < us) {
      us = t;
      best = s;
    }
  }
  return best;
}

template <int ELEM>
hipError_t tiles(int variant, const Mx4GemmArgs &a, int splits, hipStream_t stream, int num_cus) {
  switch (variant) {
    case 0: return launch_tiles<ELEM, 8, 4, 2, 4, 1>(a, splits, stream, num_cus);
    case 1: return launch_tiles<ELEM, 4, 4, 2, 2, 1>(a, splits, stream, num_cus);
    case 2: return launch_tiles<ELEM, 4, 4, 2, 2, 2>(a, splits, stream, num_cus);
    case 3: return launch_tiles<ELEM, 4, 2, 1, 2, 1>(a, splits, stream, num_cus);
    case 4: return launch_tiles<ELEM, 4, 2, 1, 2, 2>(a, splits, stream, num_cus);
    default: return launch_tiles<ELEM, 4, 2, 1, 2, 4>(a, splits, stream, num_cus);
  }
}

template <int ELEM>
hipError_t join(const Mx4GemmArgs &a, int splits, hipStream_t stream, int num_cus) {
  const int64_t blocks = std::min<int64_t>((a.M * a.N + 1023) / 1024, 4 * num_cus);
  mx4_join_kernel<ELEM><<<(unsigned)blocks, 256, 0, stream>>>(a, splits);
  return hipGetLastError();
}

template <int ELEM>
hipError_t gemm(const Mx4GemmArgs &a, hipStream_t stream, int num_cus) {
  if (a.K == 0) return join<ELEM>(a, 0, stream, num_cus);   // zeros: the sums of no ranges
  const int64_t stages = (mx4_groups(a.K) + 1) / 2;
  int best = 0;
  double us = 1e300;
  for (int i = 0; i < 6; ++i) {
    const double t = tiles_us(kVariants[i], a.M, a.N, stages, num_cus);
    if (t < us) {
      us = t;
      best = i;
    }
  }
  const int splits = ranges_of(a.M, a.N, stages, num_cus, us);
  if (a.M <= kFewMax && few_us(a.M, a.K, a.N, num_cus) < us + cold_us(a.K, a.N))
    return launch_few_rows<ELEM, -1>(FewArgs{a, nullptr, 0}, stream, num_cus);
  if (splits == 1) return tiles<ELEM>(best, a, 1, stream, num_cus);
  const hipError_t e = launch_tiles<kPart, 4, 2, 1, 2, 4>(a, splits, stream, num_cus);
  if (e != hipSuccess) return e;
  const int per = (int)((stages + splits - 1) / splits);
  return join<ELEM>(a, (int)((stages + per - 1) / per), stream, num_cus);
}

int64_t up16(int64_t n) { return (n + 15) / 16 * 16; }

}  // namespace

// X in 4 bits and its scales, then the ranges' sums.
int64_t mx4_work_bytes(int64_t M, int64_t K, int64_t N) {
  const int64_t x = M * mx4_row_bytes(K) + up16(4 * mx4_groups(K) * M);
  return x + (M * N < kRangeValues / 16 ? 16 * M * N : kRangeValues) * 4;
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
  if (a.M <= kFewOwn && a.K > 0 && a.K <= kFewOwnK) {
    const FewArgs f{a, (const unsigned char *)X, ldx};
    if (xelem == TCU_ELEM_F16)
      return elem == TCU_ELEM_F32 ? launch_few_rows<TCU_ELEM_F32, TCU_ELEM_F16>(f, stream, num_cus)
                                  : launch_few_rows<TCU_ELEM_F16, TCU_ELEM_F16>(f, stream, num_cus);
    return elem == TCU_ELEM_F32 ? launch_few_rows<TCU_ELEM_F32, TCU_ELEM_BF16>(f, stream, num_cus)
                                : launch_few_rows<TCU_ELEM_BF16, TCU_ELEM_BF16>(f, stream, num_cus);
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

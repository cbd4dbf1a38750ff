// Low-rank adapters of many requests beside a shared projection, and their
// gradients (tcu_adapter_gemm, tcu_adapter_gemm_q8, tcu_adapter_grad,
// tcu_adapter_input_grad).
//
//   Y[m] = X[m] W + alpha[g] (X[m] A_g^T) B_g^T,  g = ids[m]
//   dA_g = sum_m alpha[g] (dY[m] B_g)^T X[m],  dB_g = sum_m alpha[g] dY[m]^T (X[m] A_g^T)
//
// T = alpha X A^T is formed by narrow_kernel; the projection is the blocked
// product's kernels, T B^T added to their sums before these are stored.
#include "tcu_elem.h"
#include "tcu_gemm_tiles.h"
#include "tcu_layer.h"

namespace tcu {
namespace {

constexpr int64_t round256(int64_t n) { return (n + 255) / 256 * 256; }

// Ranks of T's rows: one or an even number of blocks of 16.
__host__ __device__ constexpr int64_t rank_pad(int64_t r) { return r <= 16 ? 16 : (r + 31) / 32 * 32; }

// ---------------------------------------------------------------------------
// T[m][j] = alpha[g] sum_k X[m][k] F_g[j][k] (F_g: r x K, rows contiguous), zeros
// from rank r on to rank_pad.  A workgroup takes up to 16 kR rows of one
// adapter, wherever they lie, and 16 or 32 ranks; its 8 waves take every eighth 64
// elements of K, and their sums are added in their order.  A load instruction
// fetches 8 whole lines of 128 bytes (X from memory once, F from the caches); a
// wave turns them into the matrix cores' operands through its own part of LDS,
// 16-byte chunks XOR-swizzled by the row, without barriers.
//
// Which rows a workgroup takes it finds out by itself (kHeld > 0: up to kScanRows
// rows and kScanAdapters adapters): it counts every adapter's rows, and with
// them the pieces before its own, then places its adapter's
// rows.  Larger calls, and those that need the order elsewhere, read it off
// group_kernel's.  Bound by X's bytes: 8192 x 8192 rank 32 37 us, 3.6 TB/s; two of 8192
// x 4096 rank 16 33 us, 4.1 TB/s; small calls by the search and two memory latencies, 6
// us.  (A launch of group_kernel takes 5 to 9 us of a call; taking
// rows as they lie, a product for each adapter of a block, 60 us for 128 rows of
// 16 adapters in turn.)
// ---------------------------------------------------------------------------
constexpr int kNarrowThreads = 512, kScanHeld = 16;
constexpr int64_t kScanRows = kNarrowThreads * kScanHeld, kScanAdapters = kNarrowThreads;

struct Narrow {
  const unsigned char *X, *F;
  float *T;
  int64_t ldx;
  int K;
};

// Inclusive sum over a wave's lanes in their order, in its registers.
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);   // from 1, 2, 4 and 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);   // lanes below, in rows
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);   // of 16
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);   // rows 0 and 2 to 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);   // the lower half to the upper
  return v;
}

// The same over a workgroup's lanes; part: a word of LDS per wave.
template <int kThreads>
__device__ __forceinline__ int block_scan(int v, int *part) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  v = wave_scan(v);
  __syncthreads();   // earlier reads of part
  if (lane == 63) part[w] = v;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) v += i < w ? part[i] : 0;
  return v;
}

// Rows t, t + kThreads, .. of a tile of kThreads kHeld rows that begins at row m0:
// their adapters' numbers, -1 without one.
template <int kThreads, int kHeld>
__device__ __forceinline__ void load_ids(const int *__restrict__ ids, int m0, int M, int G,
                                         int (&held)[kHeld]) {
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int m = m0 + kThreads * i + (int)threadIdx.x;
    const int id = ids[m < M ? m : M - 1];
    held[i] = m < M && id >= 0 && id < G ? id : -1;
  }
}

// f(place, row) for every row of the tile that names g, its place among them in
// the order of the rows; returns how many there are.  tab: LDS, a word for each
// wave and held row, free when this is called.  Every wave adds up the whole
// table for itself: no second wait.
template <int kThreads, int kHeld, typename F>
__device__ __forceinline__ int place_rows(const int (&held)[kHeld], int g, int m0, int *tab, F f) {
  constexpr int kWaves = kThreads / 64, kWords = kWaves * kHeld, kPer = kWords > 64 ? 2 : 1;
  static_assert(kWords == 128 || kWords <= 64, "one or two words a lane");
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  unsigned long long votes[kHeld];
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    votes[i] = __ballot(held[i] == g);
    if (lane == 0) tab[i * kWaves + w] = __popcll(votes[i]);
  }
  __syncthreads();
  const int a = kPer == 2 || lane < kWords ? tab[kPer * lane] : 0;
  const int sum = kPer == 2 ? a + tab[2 * lane + 1] : a;
  const int upto = wave_scan(sum), before = upto - sum;
#pragma unroll
  for (int i = 0; i < kHeld; ++i) {
    const int word = i * kWaves + w, from = word / kPer;
    int at = __builtin_amdgcn_readlane(before, from);
    if (kPer == 2 && (word & 1)) at += __builtin_amdgcn_readlane(a, from);
    if (held[i] == g)
      f(at + __popcll(votes[i] & ((1ull << lane) - 1)), m0 + kThreads * i + (int)threadIdx.x);
  }
  return __builtin_amdgcn_readlane(upto, 63);
}

// The adapter of piece `piece` (to g) and the rows of it (up to kPiece of them, to
// rows[]); returns how many there are, 0 if there is no such piece.  kHeld: every
// lane looks through so many rows' numbers, 0: read off the order.
struct Piece {
  int bins[kScanAdapters], part[8], tab[kScanHeld * 8], rows[32], g, chunk, n;
};
template <int kHeld, int kPiece>
__device__ __forceinline__ int find_piece(Piece &s, const int *__restrict__ ids,
                                          const int *__restrict__ order,
                                          const int *__restrict__ start, int M, int G, int piece,
                                          int &g) {
  const int t = threadIdx.x, lane = t & 63;
  int held[kHeld > 0 ? kHeld : 1], chunk, n;
  if (t == 0) s.n = 0;
  auto found = [&]() {
    __syncthreads();
    g = s.g;
    chunk = s.chunk;
    n = s.n;
  };
  if constexpr (kHeld > 0) {
    load_ids<kNarrowThreads>(ids, 0, M, G, held);
    s.bins[t] = 0;
    __syncthreads();
    // (sums of counts: any order gives the same).  A wave whose rows all name one
    // adapter adds them at once: one by one its lanes would queue at one address.
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      if (kNarrowThreads * i >= M) break;
      const int lead = __builtin_amdgcn_readfirstlane(held[i]);
      if (__all(held[i] == lead)) {
        if (lane == 0 && lead >= 0) atomicAdd(&s.bins[lead], 64);
      } else if (held[i] >= 0) {
        atomicAdd(&s.bins[held[i]], 1);
      }
    }
    __syncthreads();
    if (G <= 64) {
      // every wave for itself
      const int rows = s.bins[lane], pieces = (rows + kPiece - 1) / kPiece;
      const int before = wave_scan(pieces) - pieces;
      const unsigned long long hit = __ballot(piece >= before && piece < before + pieces);
      if (hit == 0) return 0;
      g = __builtin_ctzll(hit);
      chunk = piece - __builtin_amdgcn_readlane(before, g);
      n = min(__builtin_amdgcn_readlane(rows, g) - chunk * kPiece, kPiece);
    } else {
      const int rows = s.bins[t], pieces = (rows + kPiece - 1) / kPiece;
      const int before = block_scan<kNarrowThreads>(pieces, s.part) - pieces;
      if (piece >= before && piece < before + pieces) {
        s.g = t;
        s.chunk = piece - before;
        s.n = min(rows - s.chunk * kPiece, kPiece);
      }
      found();
    }
  } else {
    int base = 0;
    for (int g0 = 0; g0 < G && base <= piece; g0 += kNarrowThreads) {
      const int at = g0 + t, rows = at < G ? start[at + 1] - start[at] : 0;
      const int pieces = (rows + kPiece - 1) / kPiece;
      const int upto = block_scan<kNarrowThreads>(pieces, s.part), before = base + upto - pieces;
      if (piece >= before && piece < before + pieces) {
        s.g = at;
        s.chunk = piece - before;
        s.n = min(rows - s.chunk * kPiece, kPiece);
      }
      __syncthreads();   // s.part has been read
      if (t == kNarrowThreads - 1) s.part[0] = upto;
      __syncthreads();
      base += s.part[0];
    }
    found();
  }
  if (n == 0) return 0;
  const int from = chunk * kPiece;
  if constexpr (kHeld > 0) {
    place_rows<kNarrowThreads>(held, g, 0, s.tab, [&](int at, int m) {
      if (at >= from && at < from + n) s.rows[at - from] = m;
    });
  } else {
    if (t < n) s.rows[t] = order[start[g] + from + t];
  }
  __syncthreads();
  return n;
}

// Two workgroups a compute unit: the few pieces past a whole round that short last
// pieces make would cost a second one.
template <int ELEM, int kBlocks, int kHeld, int kR>
__global__ __launch_bounds__(kNarrowThreads, 4) void narrow_kernel(Narrow n0, Narrow n1,
                                                      const float *__restrict__ alpha,
                                                      const int *__restrict__ ids,
                                                      const int *__restrict__ order,
                                                      const int *__restrict__ start, int M, int r,
                                                      int rp, int G, int first) {
  constexpr int DT = ELEM == TCU_ELEM_F16 ? TCU_F16_F32 : TCU_BF16_F32;
  constexpr int kWaves = kNarrowThreads / 64, kStep = 64, kPart = (kR + kBlocks) * 2048;
  static_assert(kBlocks * kR * 1024 <= kPart, "a wave's sums");
  static_assert(sizeof(Piece) <= kWaves * kPart, "the search");
  __shared__ __attribute__((aligned(128))) unsigned char lds[kWaves * kPart];
  const Narrow n = blockIdx.y == 0 ? n0 : n1;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int lr = lane >> 3, lc = lane & 7;      // a load's row and chunk
  Piece &found = *(Piece *)lds;
  int g;
  const int count =
      find_piece<kHeld, 16 * kR>(found, ids, order, start, M, G, first + blockIdx.x, g);
  if (count == 0) return;
  g = __builtin_amdgcn_readfirstlane(g);
  int row[kR];
  const unsigned char *x[2 * kR];
#pragma unroll
  for (int i = 0; i < kR; ++i) row[i] = found.rows[min(16 * i + c, count - 1)];
#pragma unroll
  for (int h = 0; h < 2 * kR; ++h)
    x[h] = n.X + 2 * ((int64_t)found.rows[min(8 * h + lr, count - 1)] * n.ldx + 8 * lc);
  __syncthreads();   // the search's LDS is free
  unsigned char *const mine_lds = lds + w * kPart;
  unsigned char *const put = mine_lds + lr * 128 + 16 * (lc ^ lr);
  const unsigned char *get[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) get[h] = mine_lds + c * 128 + 16 * ((4 * h + q) ^ (c & 7));
  const unsigned char *fg = n.F + 2 * ((int64_t)g * r * n.K + 8 * lc);
  const float al = alpha[g];
  const int j0 = blockIdx.z * (16 * kBlocks);
  const unsigned char *f[kBlocks][2];
  f32x4 acc[kBlocks][kR];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int j = j0 + 16 * b + 8 * h + lr;
      f[b][h] = fg + 2 * (int64_t)(j < r ? j : r - 1) * n.K;
    }
#pragma unroll
    for (int i = 0; i < kR; ++i) acc[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  struct Chunk {
    u32x4 x[2 * kR], f[kBlocks][2];
  };
  auto load = [&](int k, Chunk &v) __attribute__((always_inline)) {
    if (k + kStep <= n.K) {
#pragma unroll
      for (int h = 0; h < 2 * kR; ++h) v.x[h] = load16_any(x[h] + 2 * k);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) v.f[b][h] = load16_any(f[b][h] + 2 * k);
    } else {
      // zeros past K
      const int valid = n.K - k - 8 * lc;
#pragma unroll
      for (int h = 0; h < 2 * kR; ++h) v.x[h] = load8<ELEM>(x[h] + 2 * k, valid).v[0];
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) v.f[b][h] = load8<ELEM>(f[b][h] + 2 * k, valid).v[0];
    }
  };
  auto multiply = [&](const Chunk &v) __attribute__((always_inline)) {
#pragma unroll
    for (int h = 0; h < 2 * kR; ++h) *(u32x4 *)(put + 1024 * h) = v.x[h];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
        *(u32x4 *)(put + 2048 * (kR + b) + 1024 * h) = v.f[b][h];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 xf[kR];
#pragma unroll
      for (int i = 0; i < kR; ++i) xf[i] = *(const u32x4 *)(get[h] + 2048 * i);
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        const u32x4 ff = *(const u32x4 *)(get[h] + 2048 * (kR + b));
#pragma unroll
        for (int i = 0; i < kR; ++i) acc[b][i] = mfma_k32(DT, ff, xf[i], acc[b][i]);
      }
    }
  };
  // kAhead chunks in flight
  constexpr int kAhead = kBlocks == 1 && kR == 1 ? 4 : 2, kNext = kWaves * kStep;
  Chunk v[kAhead];
  int k = w * kStep;
#pragma unroll
  for (int u = 0; u < kAhead; ++u)
    if (k + u * kNext < n.K) load(k + u * kNext, v[u]);
  while (k < n.K) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (k >= n.K) break;
      multiply(v[u]);
      if (k + kAhead * kNext < n.K) load(k + kAhead * kNext, v[u]);
      k += kNext;
    }
  }
#pragma unroll
  for (int b = 0; b < kBlocks; ++b)
#pragma unroll
    for (int i = 0; i < kR; ++i)
      *(f32x4 *)(mine_lds + (b * kR + i) * 1024 + 16 * lane) = acc[b][i];
  __syncthreads();
  if (w < kBlocks * kR) {
    f32x4 v = *(const f32x4 *)(lds + w * 1024 + 16 * lane);
#pragma unroll
    for (int u = 1; u < kWaves; ++u) v += *(const f32x4 *)(lds + u * kPart + w * 1024 + 16 * lane);
    // ranks j .. j + 3 of the piece's row `at`
    const int i = w % kR, at = 16 * i + c, j = j0 + 16 * (w / kR) + 4 * q;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = j + e < r ? v[e] * al : 0.f;
    if (at < count) *(f32x4 *)(n.T + (int64_t)row[kR == 2 && i == 1 ? kR - 1 : 0] * rp + j) = v;
  }
}

// ---------------------------------------------------------------------------
// The rows in the order of their adapters, the rows of one in their own order:
// order[start[g] .. start[g + 1]) are g's, start[G] the rows that have one.
// Workgroup g counts the rows of smaller numbers, then places its own.
// ---------------------------------------------------------------------------
constexpr int kGroupThreads = 1024, kGroupHeld = 8, kGroupTile = kGroupThreads * kGroupHeld;
__device__ __forceinline__ void group_rows(const int *__restrict__ ids, int *__restrict__ start,
                                           int *__restrict__ order, int M, int G, int g) {
  __shared__ int part[kGroupThreads / 64], tab[128];
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int held[kGroupHeld];
  int below = 0;
  for (int64_t m0 = 0; m0 < M; m0 += kGroupTile) {
    load_ids<kGroupThreads>(ids, (int)m0, M, G, held);
#pragma unroll
    for (int i = 0; i < kGroupHeld; ++i) below += held[i] >= 0 && held[i] < g;
  }
#pragma unroll
  for (int s = 1; s < 64; s <<= 1) below += __shfl_xor(below, s);
  if (lane == 0) part[w] = below;
  __syncthreads();
  int at = 0;
#pragma unroll
  for (int i = 0; i < kGroupThreads / 64; ++i) at += part[i];
  if (threadIdx.x == 0) start[g] = at;
  for (int64_t m0 = 0; m0 < M; m0 += kGroupTile) {
    if (M > kGroupTile) load_ids<kGroupThreads>(ids, (int)m0, M, G, held);   // else still there
    if (m0 > 0) __syncthreads();   // reads of tab
    at += place_rows<kGroupThreads>(held, g, (int)m0, tab,
                                    [&](int place, int m) { order[at + place] = m; });
  }
  if (g == G - 1 && threadIdx.x == 0) start[G] = at;
}
__global__ __launch_bounds__(kGroupThreads) void group_kernel(const int *__restrict__ ids,
                                                              int *__restrict__ start,
                                                              int *__restrict__ order, int M,
                                                              int G) {
  group_rows(ids, start, order, M, G, blockIdx.x);
}

// ---------------------------------------------------------------------------
// The adapters' part of a product's tile, added to its sums before they are
// rounded and stored: T B^T for the adapter of every row, after the scales of an
// 8-bit base.  The sums lie as the matrix cores hold them, 16 columns of 16 rows
// a block, a lane one row; T (binary32) enters as words of the adapters' type,
// bfloat16: T = hi + lo (+ lo2 where the output is binary32: 24 bits), binary16:
// T 2^-e = hi + lo with 2^e the row's largest value, so that no size of T
// leaves the type's range.  With 16 ranks both words of a rank share one
// product of 32.  Every adapter's product is formed apart and added by its own
// rows alone, so that no row sees another adapter's values (a block costs one
// product per distinct adapter of its 16 rows; summing in place where there is
// one made the 256 x 256 tiles spill 175 registers).  A wave goes through the
// adapters of 32 rows at a time, the next 32 rows' T and the next adapter's
// fragments of B on their way from the caches under the products of one.  Int8 4096
// x 4096 x 8192 rank 16, eight adapters: 149 us, 137 where no row has one.
// ---------------------------------------------------------------------------
template <int ELEM, int OUT, bool kQ8>
struct AdapterTail {
  static constexpr bool kOn = true;
  template <int DT>
  static constexpr int kOut = OUT;
  static constexpr int kWords = ELEM == TCU_ELEM_BF16 && OUT != TCU_BF16_BF16 ? 3 : 2;

  const float *T, *xscale, *wscale;
  const unsigned char *B;      // N x rb of every adapter, at this part's first column
  const int *ids;
  int64_t bstride;             // bytes from one adapter's B to the next
  int rp, rb, G;               // rb: a multiple of 8, at most rp

  AdapterTail at(int64_t row, int64_t col) const {
    AdapterTail t = *this;
    if (G > 0) {
      t.T += row * rp;
      t.B += col * rb * 2;
      t.ids += row;
    }
    if (kQ8) {
      t.xscale += row;
      t.wscale += col;
    }
    return t;
  }

  // Eight values of T (ranks 8 k .. of a row) as words of the adapters' type;
  // e: the row's binary exponent (binary16).
  __device__ __forceinline__ static void words(const float (&t)[8], int e, u32x4 (&w)[kWords]) {
    float rest[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) rest[i] = ELEM == TCU_ELEM_F16 ? ldexpf(t[i], -e) : t[i];
#pragma unroll
    for (int k = 0; k < kWords; ++k) {
      const Raw8<ELEM> r = pack8<ELEM>(rest);
      float back[8];
      unpack8<ELEM>(r, back);
      w[k] = r.v[0];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        // nothing is left of a value that is not finite
        const bool fine = (bitcast<unsigned>(back[i]) & 0x7f800000u) != 0x7f800000u;
        rest[i] = fine ? rest[i] - back[i] : 0.f;
      }
    }
  }

  template <typename Acc, int FN, int FM>
  __device__ __forceinline__ void apply(Acc (&acc)[FN][FM], int row0, int col0, int M,
                                        int N) const {
    const int lane = threadIdx.x & 63, c = lane & 15, q = lane >> 4;
    constexpr int DT = ELEM == TCU_ELEM_F16 ? TCU_F16_F32 : TCU_BF16_F32;
    int id[FM];
    unsigned long long any = 0;
#pragma unroll
    for (int fm = 0; fm < FM; ++fm) {
      const int m = row0 + 16 * fm + c;
      id[fm] = m < M && G > 0 ? ids[m] : -1;
      if (id[fm] >= G || id[fm] < 0) id[fm] = -1;
      any |= __ballot(id[fm] >= 0);
    }
    if constexpr (kQ8) {
      float ws[FN][4];
#pragma unroll
      for (int fn = 0; fn < FN; ++fn)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int n = col0 + 16 * fn + 4 * q + e;
          ws[fn][e] = wscale[n < N ? n : N - 1];
        }
#pragma unroll
      for (int fm = 0; fm < FM; ++fm) {
        const int m = row0 + 16 * fm + c;
        const float xs = xscale[m < M ? m : M - 1];
#pragma unroll
        for (int fn = 0; fn < FN; ++fn) {
          f32x4 v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = (float)bitcast<i32x4>(acc[fn][fm])[e] * xs * ws[fn][e];
          acc[fn][fm] = bitcast<Acc>(v);
        }
      }
    }
    if (any == 0) return;
    static_assert(FM % 2 == 0, "blocks in pairs");
    // binary16: 2^e brings the row's largest finite |T| to [2^14, 2^15)
    int ex[FM];
    if constexpr (ELEM == TCU_ELEM_F16) {
#pragma unroll
      for (int fm = 0; fm < FM; ++fm) {
        const int m = row0 + 16 * fm + c;
        unsigned top = 0u;
        if (id[fm] >= 0)
          for (int j = 4 * q; j < rp; j += 16) {
            const u32x4 v = *(const u32x4 *)(T + (int64_t)m * rp + j);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const unsigned b = v[i] & 0x7fffffffu;
              top = b > top && b < 0x7f800000u ? b : top;
            }
          }
#pragma unroll
        for (int s = 16; s <= 32; s <<= 1) {
          const unsigned o = __shfl_xor(top, s);
          top = o > top ? o : top;
        }
        ex[fm] = top == 0u ? 0 : __builtin_amdgcn_frexp_expf(bitcast<float>(top)) - 15;
      }
    }
    const bool narrow = rp == 16;
    const int steps = narrow ? 1 : rp / 32;
    constexpr int kGroup = 2;
    for (int s = 0; s < steps; ++s) {
      const int rank = 32 * s + 8 * (narrow ? q & 1 : q);
      auto load_b = [&](int g, u32x4 (&wf)[FN]) __attribute__((always_inline)) {
#pragma unroll
        for (int fn = 0; fn < FN; ++fn) {
          const int n = col0 + 16 * fn + c;
          // past the ranks: zeros, as T has them
          wf[fn] = rank < rb ? *(const u32x4 *)(B + (int64_t)g * bstride +
                                                2 * ((int64_t)(n < N ? n : N - 1) * rb + rank))
                             : u32x4{0u, 0u, 0u, 0u};
        }
      };
      auto load_t = [&](int f0, Raw8<TCU_ELEM_F32> (&t)[kGroup]) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
          const int m = row0 + 16 * (f0 + i) + c;
          t[i] = load8<TCU_ELEM_F32>(
              (const unsigned char *)(T + (int64_t)(m < M ? m : M - 1) * rp + rank), 8);
        }
      };
      int held = -1;
      u32x4 wf[FN];
#pragma unroll
      for (int fn = 0; fn < FN; ++fn) wf[fn] = u32x4{0u, 0u, 0u, 0u};
      Raw8<TCU_ELEM_F32> t[kGroup];
      load_t(0, t);
#pragma unroll
      for (int f0 = 0; f0 < FM; f0 += kGroup) {
        u32x4 w[kGroup][kWords];
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
          float v[8];
          unpack8<TCU_ELEM_F32>(t[i], v);
          words(v, ELEM == TCU_ELEM_F16 ? ex[f0 + i] : 0, w[i]);
          if (narrow) {
            // lanes of the upper ranks' places take the second word, and of a
            // third word's product nothing
            const u32x4 none = {0u, 0u, 0u, 0u};
            w[i][0] = q < 2 ? w[i][0] : w[i][1];
            if constexpr (kWords == 3) w[i][1] = q < 2 ? w[i][2] : none;
          }
        }
        if (f0 + kGroup < FM) load_t(f0 + kGroup, t);
        // rows whose adapter is still to come, 16 bits a block
        unsigned left = 0u;
#pragma unroll
        for (int i = 0; i < kGroup; ++i)
          left |= (unsigned)(__ballot(id[f0 + i] >= 0) & 0xffffu) << (16 * i);
        auto lead = [&]() __attribute__((always_inline)) {
          const int at = __builtin_ctz(left);
          return __builtin_amdgcn_readlane(at < 16 ? id[f0] : id[f0 + 1], at & 15);
        };
        if (left == 0u) continue;
        int g = lead();
        if (g != held) load_b(g, wf);
        while (true) {
          unsigned mine = 0u;
#pragma unroll
          for (int i = 0; i < kGroup; ++i)
            mine |= (unsigned)(__ballot(id[f0 + i] == g) & 0xffffu) << (16 * i);
          left &= ~mine;
          // the next adapter's B is on its way under this one's products
          const int next = left != 0u ? lead() : g;
          u32x4 wn[FN];
          if (left != 0u) load_b(next, wn);
#pragma unroll
          for (int i = 0; i < kGroup; ++i) {
            if ((mine >> (16 * i) & 0xffffu) == 0u) continue;
            const bool own = id[f0 + i] == g;
#pragma unroll
            for (int fn = 0; fn < FN; ++fn) {
              f32x4 d = mfma_k32(DT, wf[fn], w[i][0], f32x4{0.f, 0.f, 0.f, 0.f});
              if (kWords == 3 || !narrow) d = mfma_k32(DT, wf[fn], w[i][1], d);
              if constexpr (kWords == 3)
                if (!narrow) d = mfma_k32(DT, wf[fn], w[i][2], d);
              f32x4 v = bitcast<f32x4>(acc[fn][f0 + i]);
#pragma unroll
              for (int e = 0; e < 4; ++e)
                v[e] = own ? v[e] + (ELEM == TCU_ELEM_F16 ? ldexpf(d[e], ex[f0 + i]) : d[e]) : v[e];
              acc[fn][f0 + i] = bitcast<Acc>(v);
            }
          }
          if (left == 0u) break;
          g = next;
#pragma unroll
          for (int fn = 0; fn < FN; ++fn) wf[fn] = wn[fn];
        }
        held = g;
      }
    }
  }
};

// B of every adapter with rows of rp ranks, zeros from rank r on (ranks that are
// no multiple of 8).
__global__ __launch_bounds__(256) void pad_ranks_kernel(const unsigned short *__restrict__ B,
                                                        unsigned short *__restrict__ out,
                                                        int64_t rows, int r, int rp) {
  const int64_t total = rows * rp;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total;
       i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / rp;
    const int j = (int)(i - row * rp);
    out[i] = j < r ? B[row * r + j] : (unsigned short)0;
  }
}

// out (cols x rows) of every adapter = in (rows x cols), 16-bit values, in `tiles`
// tiles of 4096: 32 along the shorter side, the rank's, 128 along the other, or 16
// and 256 where the shorter one has no more (27 adapters of 5966 x 16: gradients and
// input's gradient 69.4 us, 75.2 with the wider tile half empty).
struct Transpose {
  const unsigned short *in;
  unsigned short *out;
  int64_t rows, cols, tiles;
};
__host__ __device__ constexpr int64_t tiles_of(int64_t rows, int64_t cols) {
  return rows < cols ? rows <= 16 ? (cols + 255) / 256 : (rows + 31) / 32 * ((cols + 127) / 128)
         : cols <= 16 ? (rows + 255) / 256
                      : (rows + 127) / 128 * ((cols + 31) / 32);
}
template <int kR, int kC>
__device__ __forceinline__ void transpose_tiles(const Transpose &a, int64_t t, int64_t step,
                                                unsigned short *tile) {
  const unsigned tc = (unsigned)((a.cols + kC - 1) / kC), per = (unsigned)tiles_of(a.rows, a.cols);
  const int rows = (int)a.rows, cols = (int)a.cols;
  for (; t < a.tiles; t += step) {
    const int64_t g = t / per, base = g * a.rows * a.cols;
    const unsigned in_g = (unsigned)(t - g * per);
    const int r0 = in_g / tc * kR, c0 = in_g % tc * kC;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = threadIdx.x + 1024 * i, y = e / kC, x = e % kC;
      if (r0 + y < rows && c0 + x < cols)
        tile[y * (kC + 2) + x] = a.in[base + (int64_t)(r0 + y) * cols + c0 + x];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int e = threadIdx.x + 1024 * i, y = e / kR, x = e % kR;
      if (c0 + y < cols && r0 + x < rows)
        a.out[base + (int64_t)(c0 + y) * rows + r0 + x] = tile[x * (kC + 2) + y];
    }
    __syncthreads();
  }
}

// What the gradients need first, in one launch: one or two transposes and (order
// not null) the rows' order.
__global__ __launch_bounds__(kGroupThreads) void prepare_kernel(Transpose t0, Transpose t1,
                                                                const int *__restrict__ ids,
                                                                int *__restrict__ start,
                                                                int *__restrict__ order, int M,
                                                                int G) {
  __shared__ unsigned short tile[256 * 18];   // the largest of the four
  const int groups = order ? G : 0;
  if ((int)blockIdx.x < groups) {
    group_rows(ids, start, order, M, G, blockIdx.x);
    return;
  }
  const int64_t t = (int)blockIdx.x - groups, step = (int)gridDim.x - groups;
  auto transpose = [&](const Transpose &a) {
    if (a.rows < a.cols) {
      if (a.rows <= 16)
        transpose_tiles<16, 256>(a, t, step, tile);
      else
        transpose_tiles<32, 128>(a, t, step, tile);
    } else if (a.cols <= 16) {
      transpose_tiles<256, 16>(a, t, step, tile);
    } else {
      transpose_tiles<128, 32>(a, t, step, tile);
    }
  };
  transpose(t0);
  transpose(t1);
}

// ---------------------------------------------------------------------------
// D_g(j, c) = sum over g's rows of T[m][j] X[m][c], the rows in the order of
// group_kernel cut into chunks.  A workgroup takes one chunk, 128 columns, 16 or 32
// ranks and every `beside`th adapter,
// its 4 waves every fourth group of 4 rows: binary32 matrix products over 4 rows,
// a lane holding 8 columns of one of them (16 bytes), value e of the 16 lanes
// being columns e, 8 + e, .. of product e.  An adapter whose rows lie in one
// chunk is written at once; the parts of the others (those a chunk begins with,
// and those it ends with) go to scratch and are added by finish_kernel in the
// order of the chunks.  X and dY of 8192 x 4096, rank 16: 37 us, 3.7 TB/s.
// ---------------------------------------------------------------------------
struct Factor {
  const unsigned char *X;
  const float *T;
  float *D, *parts;      // parts: chunk, first or last, then as one of D
  int64_t ldx, dj, dc;   // D_g(j, c) at D + g r C + j dj + c dc
  int C;
};
constexpr int kFactorCols = 128;

template <int ELEM, int kBlocks>
__global__ __launch_bounds__(256) void factor_kernel(Factor f0, Factor f1,
                                                     const int *__restrict__ order,
                                                     const int *__restrict__ start, int r, int rp,
                                                     int G, int chunk, int cols0) {
  // (a lane's place c + 17 q: the reads below go across the lanes)
  __shared__ f32x4 sums[4][8][68];
  const bool second = (int)blockIdx.x >= cols0;
  const Factor f = second ? f1 : f0;
  const int c0 = ((int)blockIdx.x - (second ? cols0 : 0)) * kFactorCols;
  const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = lane & 15, q = lane >> 4;
  const int begin = blockIdx.y * chunk, count = start[G];
  const int end = begin + chunk < count ? begin + chunk : count;
  const int col = c0 + 8 * c, valid = f.C - col;
  const int64_t rc = (int64_t)r * f.C;
  // this workgroup's ranks, and its adapters with rows in the chunk: every beside'th
  const int rank_blocks = rp / (16 * kBlocks), beside = gridDim.z / rank_blocks;
  const int zg = blockIdx.z / rank_blocks, j0 = (blockIdx.z - zg * rank_blocks) * (16 * kBlocks);
  for (int g0 = zg; g0 < G; g0 += 64 * beside) {
    const int gl = g0 + lane * beside;
    const int b0 = gl < G ? start[gl] : 0, b1 = gl < G ? start[gl + 1] : 0;
    unsigned long long here = __ballot(b0 < b1 && b0 < end && b1 > begin);
    while (here != 0) {
      const int from = __builtin_ctzll(here);
      here &= here - 1;
      const int g = g0 + from * beside;
      const int s0 = __builtin_amdgcn_readlane(b0, from), s1 = __builtin_amdgcn_readlane(b1, from);
      const int at = s0 > begin ? s0 : begin, to = s1 < end ? s1 : end;
      float *const out = s0 >= begin && s1 <= end
                             ? f.D + g * rc
                             : f.parts + (2 * (int64_t)blockIdx.y + (s0 >= begin)) * rc;
      f32x4 acc[kBlocks][8];
#pragma unroll
      for (int b = 0; b < kBlocks; ++b)
#pragma unroll
        for (int e = 0; e < 8; ++e) acc[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
      // kU groups of 4 rows, their loads in flight together; past the run's end
      // (not `whole`) zeros
      constexpr int kU = 4;
      auto rows = [&](int m0, auto whole) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole)::value;
        Raw8<ELEM> xr[kU];
        float t[kU][kBlocks];
        int m[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const int i = m0 + 16 * u + q;
          m[u] = order[kWhole || i < to ? i : to - 1];
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          const bool in = kWhole || m0 + 16 * u + q < to;
          xr[u] = load8<ELEM>(f.X + 2 * ((int64_t)m[u] * f.ldx + col),
                              kWhole ? 8 : in ? valid : 0);
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
            t[u][b] = in ? f.T[(int64_t)m[u] * rp + j0 + 16 * b + c] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < kU; ++u) {
          float x[8];
          unpack8<ELEM>(xr[u], x);
#pragma unroll
          for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 8; ++e)
              acc[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(t[u][b], x[e], acc[b][e], 0, 0, 0);
        }
      };
      int m0 = at + 4 * w;
      if (c0 + kFactorCols <= f.C)
        for (; m0 + 16 * (kU - 1) + 4 <= to; m0 += 16 * kU) rows(m0, std::true_type{});
      for (; m0 < to; m0 += 16 * kU) rows(m0, std::false_type{});
      // The waves' sums, 16 ranks at a time: a lane holds ranks 4 q .. of column
      // 8 c + e, and stores four ranks of a column, its neighbours what lies beside
      // them: the next columns (dc = 1) or the column's other ranks (dj = 1; with
      // the ranks a stride apart 300 rows of 20 adapters, K = N = 2048, rank 64 took
      // 34.7 us, 19.7 so).
#pragma unroll
      for (int b = 0; b < kBlocks; ++b) {
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[w][e][c + 17 * q] = acc[b][e];
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = threadIdx.x + 256 * h;
          const int x = f.dc == 1 ? 64 * h + lane : at >> 2, p = f.dc == 1 ? w : at & 3;
          const int from = (x >> 3) + 17 * p;
          f32x4 v = sums[0][x & 7][from];
#pragma unroll
          for (int u = 1; u < 4; ++u) v += sums[u][x & 7][from];
          const int cc = c0 + x, j = j0 + 16 * b + 4 * p;
          if (cc >= f.C) continue;
          float *const o = out + j * f.dj + cc * f.dc;
          if (f.dj == 1 && (r & 3) == 0) {
            if (j < r) *(f32x4 *)o = v;
          } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
              if (j + k < r) o[k * f.dj] = v[k];
          }
        }
      }
    }
  }
}

// Adapters without rows: zeros.  Adapters whose rows lie in several chunks: the
// sum of their parts, V (one value or four) at a time.
template <typename V>
__device__ __forceinline__ void finish(const Factor &f, const int *__restrict__ start, int64_t rc,
                                       int G, int chunk) {
  for (int g = blockIdx.z; g < G; g += gridDim.z) {
    const int s0 = start[g], s1 = start[g + 1];
    const int first = s0 / chunk, last = s1 > s0 ? (s1 - 1) / chunk : first;
    if (s1 > s0 && first == last) continue;
    const int64_t n = rc * 4 / (int64_t)sizeof(V);
    V *const D = (V *)(f.D + g * rc);
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n;
         i += (int64_t)gridDim.x * 256) {
      V v = V{};
      if (s1 > s0) {
        const V *p = (const V *)(f.parts + 2 * (int64_t)first * rc) + i;
        v = p[n];
        p += 2 * n;
        int k = first + 1;
        for (; k + 4 <= last + 1; k += 4, p += 8 * n) {
          const V u0 = p[0], u1 = p[2 * n], u2 = p[4 * n], u3 = p[6 * n];
          v = v + u0 + u1 + u2 + u3;
        }
        for (; k <= last; ++k, p += 2 * n) v += p[0];
      }
      D[i] = v;
    }
  }
}
__global__ __launch_bounds__(256) void finish_kernel(Factor f0, Factor f1,
                                                     const int *__restrict__ start, int r, int G,
                                                     int chunk) {
  const Factor f = blockIdx.y == 0 ? f0 : f1;
  const int64_t rc = (int64_t)r * f.C;
  if ((rc & 3) == 0)
    finish<f32x4>(f, start, rc, G, chunk);
  else
    finish<float>(f, start, rc, G, chunk);
}

// Ranks of a workgroup of factor_kernel.
constexpr int factor_ranks(int64_t rp) { return rp == 16 ? 16 : 32; }

// Rows of a chunk: enough workgroups of 128 columns for the chip, and parts (2 r
// rows of binary32 a chunk) that stay small beside what is read (4000 rows, K = N
// = 2048, rank 64: factors and join 52 + 14 us with 128 rows, 39 + 13 with 256).
// All rows at most, so that it fits the kernels' int.
int64_t factor_groups(int64_t K, int64_t N, int64_t r) {
  const int64_t strips = (K + kFactorCols - 1) / kFactorCols + (N + kFactorCols - 1) / kFactorCols;
  return strips * (rank_pad(r) / factor_ranks(rank_pad(r)));
}
int64_t least_chunk(int64_t r) { return (4 * r + 63) / 64 * 64; }
int chunk_rows(int64_t M, int64_t K, int64_t N, int64_t r) {
  const int64_t least = least_chunk(r);
  const int64_t rows = (M * factor_groups(K, N, r) / 1024 + 63) / 64 * 64;
  const int64_t all = M < least ? least : M;
  return (int)(rows < least ? least : rows < all ? rows : all);
}
// Chunks of M rows or fewer at most: a chunk has `least` rows, and 64 / 65 of a 1024th
// of the rows' share (rounded down before it is rounded up).
int64_t most_chunks(int64_t M, int64_t K, int64_t N, int64_t r) {
  const int64_t groups = factor_groups(K, N, r);
  const int64_t a = M / least_chunk(r), b = groups > 0 ? 1040 / groups : 0;
  return (a < b ? a : b) + 1;
}

// Scratch: T of X and of dY, the rows in their adapters' order, the adapters
// transposed or with padded ranks, the parts of the factors' gradients.  No smaller
// than that of fewer rows: a program keeps one for its largest batch.
struct Scratch {
  unsigned char *at, *bt, *padded;
  float *t, *dt, *parts_a, *parts_b;
  int *start, *order;
  void *few;
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
  s.t = (float *)take(M * rank_pad(r) * 4);
  s.dt = (float *)take(M * rank_pad(r) * 4);
  s.start = (int *)take((G + 1) * 4);
  s.order = (int *)take(M * 4);
  s.at = take(G * r * K * 2);
  s.bt = take(G * r * N * 2);
  const int64_t chunks = most_chunks(M, K, N, r);
  // padded ranks and the gradients' parts are not of the same call
  const int64_t pad = round256(G * (N > K ? N : K) * rank_pad(r) * 2);
  const int64_t pa = round256(2 * chunks * r * K * 4), pb = round256(2 * chunks * r * N * 4);
  s.padded = take(pad > pa + pb ? pad : pa + pb);
  s.parts_a = (float *)s.padded;
  s.parts_b = (float *)(s.padded + pa);
  const int64_t fa = few_work_bytes(M, K, N, r), fb = few_work_bytes(M, N, K, r);
  s.few = take(fa > fb ? fa : fb);
  s.bytes = at;
  return s;
}

unsigned grid_for(int64_t n) { return (unsigned)(n < 1 ? 1 : n < (1 << 16) ? n : 1 << 16); }

hipError_t group(const int32_t *ids, const Scratch &s, int64_t M, int64_t G, hipStream_t stream) {
  hipLaunchKernelGGL(group_kernel, dim3((unsigned)G), dim3(kGroupThreads), 0, stream, ids, s.start,
                     s.order, (int)M, (int)G);
  return hipGetLastError();
}

constexpr int64_t kWidePieces = 512;

// T of one product, or of two (n1.X not null); order null: found by the kernel.
template <int ELEM>
hipError_t narrow(const Narrow &n0, const Narrow &n1, const float *alpha, const int32_t *ids,
                  const int *order, const int *start, int64_t M, int64_t r, int64_t G,
                  hipStream_t stream) {
  const int rp = (int)rank_pad(r);
  auto go = [&](auto blocks, auto held, auto rows) {
    constexpr int kBlocks = decltype(blocks)::value, kR = decltype(rows)::value;
    // pieces: every adapter's last one may be short
    const int64_t most = (M + 16 * kR - 1) / (16 * kR) + G - 1;
    // a launch counts its work items in 32 bits
    constexpr int64_t kMost = 1 << 22;
    const int64_t pieces = most < M ? most : M;
    for (int64_t first = 0;
         first < pieces && (first == 0 || hipPeekAtLastError() == hipSuccess); first += kMost)
      hipLaunchKernelGGL((narrow_kernel<ELEM, kBlocks, decltype(held)::value, kR>),
                         dim3((unsigned)(pieces - first < kMost ? pieces - first : kMost),
                              n1.X ? 2 : 1, rp / (16 * kBlocks)),
                         dim3(kNarrowThreads), 0, stream, n0, n1, alpha, ids, order, start, (int)M,
                         (int)r, rp, (int)G, (int)first);
  };
  typedef std::integral_constant<int, 1> One;
  typedef std::integral_constant<int, 2> Two;
  // Pieces of 32 rows read F half as often; of 16 rows they are more, for the chip
  // to be full and an adapter's last one to waste less (us of a call, 16 / 32 rows: 6000 x
  // 1000 x 300 rank 64 40.6 / 32.5, 8192 x 8192 x 8192 rank 32 872 / 867, 8000 x
  // 256 x 256 rank 16 25.0 / 23.7; below 512 pieces 4000 x 5000 x 512 rank 32
  // 60.4 / 63.0).
  const int64_t all = (M / 16 + G) * (n1.X ? 2 : 1) * (rp > 32 ? rp / 32 : 1);
  const bool wide = all > kWidePieces && n0.K >= 64;
  auto by_rows = [&](auto blocks, auto held) {
    if (wide)
      go(blocks, held, Two{});
    else
      go(blocks, held, One{});
  };
  auto by_order = [&](auto blocks) {
    if (order)
      by_rows(blocks, std::integral_constant<int, 0>{});
    else if (M <= 4 * kNarrowThreads)
      by_rows(blocks, std::integral_constant<int, 4>{});
    else
      by_rows(blocks, std::integral_constant<int, kScanHeld>{});
  };
  if (rp == 16)
    by_order(One{});
  else
    by_order(Two{});
  return hipGetLastError();
}

Transpose transpose_of(const void *in, void *out, int64_t G, int64_t rows, int64_t cols) {
  return Transpose{(const unsigned short *)in, (unsigned short *)out, rows, cols,
                   G * tiles_of(rows, cols)};
}

// ids null: the transposes alone.
hipError_t prepare(const Transpose &t0, const Transpose &t1, const int32_t *ids, const Scratch &s,
                   int64_t M, int64_t G, hipStream_t stream) {
  const int64_t tiles = t0.tiles > t1.tiles ? t0.tiles : t1.tiles;
  const int64_t blocks = (ids ? G : 0) + (tiles < 2048 ? tiles : 2048);
  if (blocks == 0) return hipSuccess;
  hipLaunchKernelGGL(prepare_kernel, dim3((unsigned)blocks), dim3(kGroupThreads), 0, stream, t0, t1,
                     ids, s.start, ids ? s.order : nullptr, (int)M, (int)G);
  return hipGetLastError();
}

// The narrow product's launch beside a product of few tiles: one number for every size (us
// of the kernel, 65 to 512 rows, rank 16 / 64: K = 512 4.0 / 4.2, 2048 4.8 / 5.8, 4096
// 6.4 / 8, 8192 9.5 / 12.7).  It is on both sides of the choice wherever T is apart.
constexpr double kNarrowUs = 7.5;

template <int ELEM, int DT, int OUT, bool kQ8>
hipError_t project(const AdapterArgs &a, const Scratch &s, hipStream_t stream, int num_cus) {
  typedef AdapterTail<ELEM, OUT, kQ8> Tail;
  const RectArgs p{kQ8 ? a.Xq : a.X, kQ8 ? a.ldxq : a.ldx, a.W, a.ldw, a.Y, a.ldy,
                   a.M, a.K, a.N, false};
  const int64_t rp = rank_pad(a.r), rb = (a.r + 7) / 8 * 8;
  auto narrow_of = [&]() {
    const bool ordered = a.M > kScanRows || a.G > kScanAdapters;
    const hipError_t e = ordered ? group(a.ids, s, a.M, a.G, stream) : hipSuccess;
    if (e != hipSuccess) return e;
    const Narrow n{(const unsigned char *)a.X, (const unsigned char *)a.A, s.t, a.ldx, (int)a.K};
    return narrow<ELEM>(n, Narrow{}, a.alpha, a.ids, ordered ? s.order : nullptr, s.start, a.M, a.r,
                        a.G, stream);
  };
  hipError_t e = hipSuccess;
  if (few_ok(DT, a)) {
    // Past one block of rows by the models of both sides' times.
    const int64_t cus = knob(TCU_KNOB_PP_GRID) > 0 ? knob(TCU_KNOB_PP_GRID) : num_cus;
    const bool dma = ring_dma_ok<DT>(p);
    double t_us = few_narrow_us(a, kQ8);
    const bool apart = t_us > kNarrowUs;
    if (apart) t_us = kNarrowUs;
    if (a.M <= kFewBlock ||
        (gemm_path() == GemmPath::kAuto &&
         few_us(a, kQ8) + t_us <
             choose_ring<DT, Tail>(p, dma, GemmPath::kAuto, cus).us + kNarrowUs)) {
      AdapterArgs b = a;
      b.work = s.few;
      if (apart) e = narrow_of();
      return e != hipSuccess ? e : launch_few(DT, b, apart ? s.t : nullptr, (int)rp, stream);
    }
  }
  const void *B = a.B;
  if (a.G > 0) {
    if (rb != a.r) {
      const int64_t rows = a.G * a.N;
      hipLaunchKernelGGL(pad_ranks_kernel, dim3(grid_for((rows * rb + 255) / 256)), dim3(256), 0,
                         stream, (const unsigned short *)a.B, (unsigned short *)s.padded, rows,
                         (int)a.r, (int)rb);
      e = hipGetLastError();
      if (e != hipSuccess) return e;
      B = s.padded;
    }
    e = narrow_of();
    if (e != hipSuccess) return e;
  }
  const Tail tail{s.t,   a.xscale,       a.wscale, (const unsigned char *)B,
                  a.ids, a.N * rb * 2, (int)rp,  (int)rb, (int)a.G};
  return launch_dt<DT>(p, stream, num_cus, tail);
}

hipError_t project_dt(int dtype, const AdapterArgs &a, const Scratch &s, hipStream_t stream,
                      int num_cus) {
  switch (dtype) {
    case TCU_F16_F32:
      return project<TCU_ELEM_F16, TCU_F16_F32, TCU_F16_F32, false>(a, s, stream, num_cus);
    case TCU_BF16_F32:
      return project<TCU_ELEM_BF16, TCU_BF16_F32, TCU_BF16_F32, false>(a, s, stream, num_cus);
    case TCU_BF16_BF16:
      return project<TCU_ELEM_BF16, TCU_BF16_BF16, TCU_BF16_BF16, false>(a, s, stream, num_cus);
    case TCU_I8_I32:
      return project<TCU_ELEM_BF16, TCU_I8_I32, TCU_BF16_BF16, true>(a, s, stream, num_cus);
  }
  return hipErrorInvalidValue;
}

template <int ELEM>
hipError_t grad_go(const AdapterGradArgs &a, hipStream_t stream) {
  const Scratch s = scratch(a.work, a.M, a.K, a.N, a.r, a.G);
  const int rp = (int)rank_pad(a.r);
  // (no rows: their order is then found empty, whatever ids is)
  hipError_t e = prepare(transpose_of(a.B, s.bt, a.G, a.N, a.r), Transpose{},
                         a.M > 0 ? a.ids : (const int32_t *)s.order, s, a.M, a.G, stream);
  if (e != hipSuccess) return e;
  const unsigned char *X = (const unsigned char *)a.X, *dY = (const unsigned char *)a.dY;
  const int chunk = chunk_rows(a.M, a.K, a.N, a.r);
  const Factor fa{X, s.dt, a.dA, s.parts_a, a.ldx, a.K, 1, (int)a.K};
  const Factor fb{dY, s.t, a.dB, s.parts_b, a.lddy, 1, a.r, (int)a.N};
  if (a.M > 0) {
    e = narrow<ELEM>(Narrow{X, (const unsigned char *)a.A, s.t, a.ldx, (int)a.K},
                     Narrow{dY, s.bt, s.dt, a.lddy, (int)a.N}, a.alpha, a.ids, s.order, s.start,
                     a.M, a.r, a.G, stream);
    if (e != hipSuccess) return e;
    const int ca = (int)((a.K + kFactorCols - 1) / kFactorCols);
    const int cb = (int)((a.N + kFactorCols - 1) / kFactorCols);
    // a chunk's adapters side by side, about as many workgroups as it has adapters, and
    // up to one for each while the chip has room (645 rows of 4, K = 192, N = 1408, rank
    // 32, with the input's gradient: 44.3 us, 48.7 with one)
    const int rank_blocks = rp / factor_ranks(rp);
    const int64_t chunks = (a.M + chunk - 1) / chunk, one = (ca + cb) * chunks * rank_blocks;
    int64_t beside = a.G / chunks + 1;
    if (beside * one < 512) beside = 512 / one < a.G ? 512 / one : a.G;
    const dim3 grid(ca + cb, (unsigned)chunks, (unsigned)(beside < 16 ? beside : 16) * rank_blocks);
    if (rp == 16)
      hipLaunchKernelGGL((factor_kernel<ELEM, 1>), grid, dim3(256), 0, stream, fa, fb,
                         s.order, s.start, (int)a.r, rp, (int)a.G, chunk, ca);
    else
      hipLaunchKernelGGL((factor_kernel<ELEM, 2>), grid, dim3(256), 0, stream, fa, fb,
                         s.order, s.start, (int)a.r, rp, (int)a.G, chunk, ca);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const int64_t most = (a.r * (a.K > a.N ? a.K : a.N) + 1023) / 1024;
  hipLaunchKernelGGL(finish_kernel, dim3((unsigned)(most < 512 ? most : 512), 2,
                                         (unsigned)(a.G < 1024 ? a.G : 1024)),
                     dim3(256), 0, stream, fa, fb, s.start, (int)a.r, (int)a.G, chunk);
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
  const Scratch s = scratch(a.work, a.M, a.K, a.N, a.r, a.G);
  AdapterArgs b = a;
  const hipError_t e = prepare(transpose_of(a.B, s.at, a.G, a.K, a.r),
                               transpose_of(a.A, s.bt, a.G, a.r, a.N), nullptr, s, a.M, a.G, stream);
  if (e != hipSuccess) return e;
  b.A = s.at;
  b.B = s.bt;
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

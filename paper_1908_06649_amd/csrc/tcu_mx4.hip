// Matrices to 4 bits and back (tcu_mx4_quant, tcu_mx4_dequant).
//
//   e = floor(log2 max|x|) - 2 over a block of 32,  code = x / 2^e to nearest even on
//   0, 1/2, 1, 3/2, 2, 3, 4, 6, clamped to 6;  scale byte e + 127
//
// Both are bound by memory: x is read once, also where it is written along its rows
// and along its columns (8192 x 8192 bf16, us from memory / where x is still in the last cache:
// along the rows 30.6 / 25.7, both ways 45.8 / 34.8, 4.5 / 5.9 TB/s, back 37.7 / 30.8; a copy
// from memory 5.0 TB/s).  Along the rows a lane holds eight values, four lanes a block, 16 a group of
// 128 with its word of four scales; a workgroup takes 8 rows of 512 columns.  Along the
// columns a tile of 128 x 128 goes through LDS, where a lane takes 16 rows of two columns.
#include <algorithm>

#include "tcu_mx4_dev.h"

namespace tcu {
namespace {

// The tile of a workgroup.  Workgroups go round the 8 XCDs: where rows of x begin inside
// lines, neighbouring tiles share lines, and an XCD takes a run of tiles (`runs`), in bands
// of kBand rows of them and column by column, so that these lines meet in its L2; where
// rows are whole lines, in order (us from memory, in order / in runs: 8191 x 8191 bf16 along
// the rows 57.4 / 35.7, both ways 65.5 / 49.1; 8192 x 8192 30.8 / 34.0 and 45.8 / 46.0.  Back, whose
// stores are these rows, 48.9 / 46.0 and smaller ones slower: always in order).
template <int kBand>
__device__ __forceinline__ void place_tile(bool runs, unsigned row_tiles, unsigned col_tiles,
                                           int64_t &row, int64_t &col) {
  unsigned v = blockIdx.x;
  if (!runs) {
    row = v / col_tiles;
    col = v % col_tiles;
    return;
  }
  const unsigned body = gridDim.x & ~7u;
  if (v < body) v = (v & 7) * (body >> 3) + (v >> 3);
  const unsigned band = v / (kBand * col_tiles), in_band = v - band * kBand * col_tiles;
  const unsigned rows = min((unsigned)kBand, row_tiles - kBand * band);
  row = kBand * band + in_band % rows;
  col = in_band / rows;
}
// Whether rows of pitch ld bytes from p on begin inside lines.
bool inside_lines(const void *p, int64_t ld) {
  return (((uintptr_t)p | (uintptr_t)ld) & 127) != 0;
}

// ------------------------------------------------------------- along the rows
// Two rows a wave (us, two / eight, bf16: 64 x 4096 2.6 / 4.1, 1024 x 4096 3.4 / 4.4, 8192 x 8192
// 24.8 / 29.7; back 2.9 / 5.2, 4.8 / 6.3, 29.8 / 31.3).
constexpr int kMine = 2, kRowTile = 4 * kMine, kColTile = 512;

template <int ELEM>
__global__ __launch_bounds__(256) void quant_rows_kernel(Mx4QuantArgs a, unsigned col_tiles,
                                                         bool runs) {
  constexpr int ES = elem_bytes<ELEM>;
  __shared__ unsigned words[4][kRowTile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int64_t r0, c0;
  place_tile<4>(runs, (unsigned)((a.rows + kRowTile - 1) / kRowTile), col_tiles, r0, c0);
  r0 *= kRowTile;
  c0 *= kColTile;
  const int64_t col = c0 + lane * 8;
  const int64_t groups = mx4_groups(a.cols);
  const int valid = (int)min((int64_t)8, max((int64_t)0, a.cols - col));
  Raw8<ELEM> raw[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int64_t r = r0 + i * 4 + wave;
    raw[i] = Raw8<ELEM>{};
    if (r < a.rows && valid > 0)
      raw[i] = load8<ELEM>((const unsigned char *)a.x + (r * a.ldx + col) * ES, valid);
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int64_t r = r0 + i * 4 + wave;
    float x[8];
    unpack8<ELEM>(raw[i], x);
    unsigned m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = umax(m, abs_bits(x[e]));
    m = quad_max(m);
    const unsigned byte = scale_byte(m);
    const unsigned c = codes8(x, byte, __any(scale_low(m)));
    if (r < a.rows && col < groups * 128) *(unsigned *)(a.q + r * a.ldq + (col >> 1)) = c;
    const unsigned word = quads_or(byte << (8 * ((lane >> 2) & 3)));
    if ((lane & 15) == 0) words[lane >> 4][i * 4 + wave] = word;
  }
  __syncthreads();
  if (threadIdx.x < 4 * kRowTile) {
    const int g = threadIdx.x / kRowTile, i = threadIdx.x % kRowTile;
    const int64_t r = r0 + i, group = c0 / 128 + g;
    if (r < a.rows && group < groups) a.s[group * a.lds + r] = words[g][i];
  }
}

// --------------------------------------------------- along the columns, or both
constexpr int kTile = 128;

// A tile in LDS as it is stored, rows of 128 values and one bank more, so that the rows'
// vectors are written, and pairs of columns read, over all banks.  The columns' codes are
// 80 bytes apart (8 lanes' vectors over all banks).
template <int ELEM>
constexpr int kTilePitch = kTile *elem_bytes<ELEM> + 4;
constexpr int kCodePitch = 80;

template <int ELEM, bool kRows>
__global__ __launch_bounds__(512) void quant_both_kernel(Mx4QuantArgs a, unsigned col_tiles,
                                                         bool runs) {
  constexpr int ES = elem_bytes<ELEM>, kPitch = kTilePitch<ELEM>;
  __shared__ __attribute__((aligned(16))) unsigned char tile[kTile * kPitch];
  __shared__ unsigned words[kTile];
  __shared__ __attribute__((aligned(16))) unsigned char codes[kTile * kCodePitch];
  __shared__ unsigned char bytes[kTile * 4];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int64_t r0, c0;
  place_tile<2>(runs, (unsigned)((a.rows + kTile - 1) / kTile), col_tiles, r0, c0);
  r0 *= kTile;
  c0 *= kTile;
  {
    // 16 lanes a row, 32 rows at a time
    const int64_t col = c0 + (t & 15) * 8;
    const int valid = (int)min((int64_t)8, max((int64_t)0, a.cols - col));
    Raw8<ELEM> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int64_t r = r0 + i * 32 + (t >> 4);
      raw[i] = Raw8<ELEM>{};
      if (r < a.rows && valid > 0)
        raw[i] = load8<ELEM>((const unsigned char *)a.x + (r * a.ldx + col) * ES, valid);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = i * 32 + (t >> 4);
      unsigned *p = (unsigned *)(tile + row * kPitch + (t & 15) * 8 * ES);
#pragma unroll
      for (int d = 0; d < 2 * ES; ++d) p[d] = raw[i].v[d >> 2][d & 3];
      if constexpr (kRows) {
        float x[8];
        unpack8<ELEM>(raw[i], x);
        unsigned m = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = umax(m, abs_bits(x[e]));
        m = quad_max(m);
        const unsigned byte = scale_byte(m);
        const unsigned c = codes8(x, byte, __any(scale_low(m)));
        if (r0 + row < a.rows) *(unsigned *)(a.q + (r0 + row) * a.ldq + c0 / 2 + (t & 15) * 4) = c;
        const unsigned word = quads_or(byte << (8 * ((t >> 2) & 3)));
        if ((t & 15) == 0) words[row] = word;
      }
    }
  }
  __syncthreads();
  if constexpr (kRows) {
    if (t < kTile && r0 + t < a.rows) a.s[c0 / 128 * a.lds + r0 + t] = words[t];
  }
  // Two waves to 32 rows, each half of the columns: a lane takes 16 rows (the upper half
  // of a wave the second 16) of two columns.
  {
    const int block = wave >> 1, pair = (wave & 1) * 32 + (lane & 31), upper = lane >> 5;
    const unsigned char *p = tile + (32 * block + 16 * upper) * kPitch + pair * 2 * ES;
    unsigned m0 = 0, m1 = 0;
    float x0[16], x1[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if constexpr (ELEM == TCU_ELEM_F32) {
        x0[i] = ((const float *)(p + i * kPitch))[0];
        x1[i] = ((const float *)(p + i * kPitch))[1];
      } else {
        const unsigned v = *(const unsigned *)(p + i * kPitch);
        if constexpr (ELEM == TCU_ELEM_F16) {
          x0[i] = (float)bitcast<_Float16>((unsigned short)(v & 0xffffu));
          x1[i] = (float)bitcast<_Float16>((unsigned short)(v >> 16));
        } else {
          x0[i] = bf16_to_f32(v & 0xffffu);
          x1[i] = bitcast<float>(v & 0xffff0000u);
        }
      }
      m0 = umax(m0, abs_bits(x0[i]));
      m1 = umax(m1, abs_bits(x1[i]));
    }
    m0 = umax(m0, __shfl_xor(m0, 32));
    m1 = umax(m1, __shfl_xor(m1, 32));
    const unsigned b0 = scale_byte(m0), b1 = scale_byte(m1);
    const bool low = __any(scale_low(m0) || scale_low(m1));
    u32x2 q0, q1;
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      float y0[8], y1[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y0[e] = x0[8 * d + e];
        y1[e] = x1[8 * d + e];
      }
      q0[d] = codes8(y0, b0, low);
      q1[d] = codes8(y1, b1, low);
    }
    *(u32x2 *)(codes + (2 * pair) * kCodePitch + block * 16 + upper * 8) = q0;
    *(u32x2 *)(codes + (2 * pair + 1) * kCodePitch + block * 16 + upper * 8) = q1;
    if (upper == 0) {
      bytes[(2 * pair) * 4 + block] = (unsigned char)b0;
      bytes[(2 * pair + 1) * 4 + block] = (unsigned char)b1;
    }
  }
  __syncthreads();
  {
    const int64_t c = c0 + (t >> 2);
    if (c < a.cols)
      *(u32x4 *)(a.qt + c * a.ldqt + r0 / 2 + (t & 3) * 16) =
          *(const u32x4 *)(codes + (t >> 2) * kCodePitch + (t & 3) * 16);
  }
  if (t < kTile && c0 + t < a.cols)
    a.ts[r0 / 128 * a.ldts + c0 + t] = *(const unsigned *)(bytes + t * 4);
}

// ----------------------------------------------------------------------- back
// A lane's values: 16 bytes of the output.
template <int ELEM>
constexpr int kBackValues = 16 / elem_bytes<ELEM>;

template <int ELEM>
__global__ __launch_bounds__(256) void dequant_kernel(Mx4DequantArgs a, unsigned col_tiles) {
  constexpr int ES = elem_bytes<ELEM>, V = kBackValues<ELEM>;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)(blockIdx.x / col_tiles) * kRowTile;
  const int64_t col = (int64_t)(blockIdx.x % col_tiles) * (64 * V) + lane * V;
  const int valid = (int)min((int64_t)V, a.cols - col);
  if (valid <= 0) return;
  unsigned c[kMine], byte[kMine];
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int64_t r = min(r0 + i * 4 + wave, a.rows - 1);
    const unsigned char *q = a.q + r * a.ldq + (col >> 1);
    c[i] = V == 8 ? *(const unsigned *)q : (unsigned)*(const unsigned short *)q;
    byte[i] = (a.s[(col >> 7) * a.lds + r] >> (8 * ((col >> 5) & 3))) & 255u;
  }
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int64_t r = r0 + i * 4 + wave;
    // a scale of 2^-127 is no normal number: the value is formed 2^32 times larger
    const bool low = byte[i] < 32u;
    const float scale = byte[i] == 255u ? __builtin_nanf("")
                                        : bitcast<float>((low ? byte[i] + 32u : byte[i]) << 23);
    const float down = low ? 0x1p-32f : 1.f;
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e >= V) {
        x[e] = 0.f;
        continue;
      }
      const unsigned k = (c[i] >> (4 * e)) & 15u, mag = k & 7u;
      // e2m1: exponent field 0 has steps of a half, then 2^(field - 1) (1 + m / 2)
      const float v = mag < 2u ? 0.5f * (float)mag
                               : bitcast<float>(((mag >> 1) + 126u) << 23 | (mag & 1u) << 22);
      x[e] = bitcast<float>(bitcast<unsigned>(v) | (k & 8u) << 28) * scale * down;
    }
    if (r >= a.rows) continue;
    unsigned char *y = (unsigned char *)a.y + (r * a.ldy + col) * ES;
    if (valid == V)
      store16_any(y, pack8<ELEM>(x).v[0]);
    else
      store8<ELEM>(y, x, valid);
  }
}

// Threads of a launch count in 32 bits: more tiles of rows than that are launched in turn.
template <typename F>
hipError_t by_rows(int64_t rows, int64_t row_tile, int64_t col_tiles, F launch) {
  if (col_tiles == 0) return hipSuccess;
  const int64_t most = std::max<int64_t>(1, ((int64_t)1 << 22) / col_tiles);
  for (int64_t r = 0; r < rows; r += most * row_tile) {
    const int64_t n = std::min(rows - r, most * row_tile);
    launch(r, n, (unsigned)((n + row_tile - 1) / row_tile * col_tiles));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <int ELEM>
hipError_t quant(const Mx4QuantArgs &a, hipStream_t stream) {
  const int width = a.qt ? kTile : kColTile;
  const int64_t col_tiles = (a.cols + width - 1) / width;
  return by_rows(a.rows, a.qt ? kTile : kRowTile, col_tiles, [&](int64_t r, int64_t n, unsigned blocks) {
    Mx4QuantArgs p = a;
    p.x = (const unsigned char *)a.x + r * a.ldx * elem_bytes<ELEM>;
    const bool runs = inside_lines(p.x, a.ldx * elem_bytes<ELEM>);
    p.rows = n;
    if (a.q) {
      p.q += r * a.ldq;
      p.s += r;
    }
    if (a.qt) {
      p.qt += r / 2;
      p.ts += r / 128 * a.ldts;
    }
    if (a.qt && a.q)
      quant_both_kernel<ELEM, true><<<blocks, 512, 0, stream>>>(p, (unsigned)col_tiles, runs);
    else if (a.qt)
      quant_both_kernel<ELEM, false><<<blocks, 512, 0, stream>>>(p, (unsigned)col_tiles, runs);
    else
      quant_rows_kernel<ELEM><<<blocks, 256, 0, stream>>>(p, (unsigned)col_tiles, runs);
  });
}

template <int ELEM>
hipError_t dequant(const Mx4DequantArgs &a, hipStream_t stream) {
  constexpr int kWidth = 64 * kBackValues<ELEM>;
  const int64_t col_tiles = (a.cols + kWidth - 1) / kWidth;
  return by_rows(a.rows, kRowTile, col_tiles, [&](int64_t r, int64_t n, unsigned blocks) {
    Mx4DequantArgs p = a;
    p.q += r * a.ldq;
    p.s += r;
    p.y = (unsigned char *)a.y + r * a.ldy * elem_bytes<ELEM>;
    p.rows = n;
    dequant_kernel<ELEM><<<blocks, 256, 0, stream>>>(p, (unsigned)col_tiles);
  });
}

}  // namespace

hipError_t launch_mx4_quant(int elem, const Mx4QuantArgs &a, hipStream_t stream) {
  switch (elem) {
    case TCU_ELEM_F32: return quant<TCU_ELEM_F32>(a, stream);
    case TCU_ELEM_F16: return quant<TCU_ELEM_F16>(a, stream);
    default: return quant<TCU_ELEM_BF16>(a, stream);
  }
}

hipError_t launch_mx4_dequant(int elem, const Mx4DequantArgs &a, hipStream_t stream) {
  switch (elem) {
    case TCU_ELEM_F32: return dequant<TCU_ELEM_F32>(a, stream);
    case TCU_ELEM_F16: return dequant<TCU_ELEM_F16>(a, stream);
    default: return dequant<TCU_ELEM_BF16>(a, stream);
  }
}

}  // namespace tcu

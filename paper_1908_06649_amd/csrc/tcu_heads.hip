// Norms of queries and keys for each head with the position's rotation in the same
// pass, and their gradients (tcu_qk_norm, tcu_qk_norm_grad).
//
//   n = x rstd,  rstd = 1 / sqrt(mean(x^2) + eps),  v = n w,  y = R v
//   dv = R^T dy,  g = dv w,  dx = rstd (g - n mean(g n)),  dw = sum dv n
//
// R turns pairs of a token's elements by its position's angles.  Both are bound by
// memory: every value is read once, held in registers and written once.
//   * A head is L lanes', a power of two; a lane holds V pairs as two runs of V
//     elements: where the pairs are half the rotated part apart the runs are, and where
//     they are adjacent both runs hold whole pairs.  V is 8, whole vectors: where a part is
//     no whole number of them its last slot begins earlier, and what it shares with the slot
//     before it is left out of the sums and stored twice with the same value.  Heads
//     whose parts are shorter than two vectors have V = 1, and kP slots a lane if they
//     need more than 64.
//   * A wave takes a few tokens, or a part of one token's heads where tokens are few, and as
//     many heads at once as fit, queries and keys in one sequence; the angles are formed
//     once a token, one lane each, in binary64 (a far position's angle has no digits left
//     in binary32), and shared through LDS.
//   * The weights' gradients are summed in registers over a workgroup's tokens, and the
//     workgroups' parts by a second launch, in their order.
// 16384 tokens of 72 heads of 128 bf16 124 us, 4.9 TB/s; gradients of 8192 tokens of 40 heads 54
// + 4.8 us, 4.7 TB/s; a copy 5.0.
#include <algorithm>

#include "tcu_elem.h"
#include "tcu_heads.h"

namespace tcu {
namespace {

constexpr int kWaves = 4;

// V elements as stored, at any element-aligned address: one, or whole vectors.
template <int ELEM, int V>
struct Run {
  static_assert(V == 1 || V == 8);
  static constexpr int kBytes = V * elem_bytes<ELEM>, kWords = kBytes < 4 ? 1 : kBytes / 4;
  unsigned w[kWords];
};
template <int ELEM, int V>
__device__ __forceinline__ Run<ELEM, V> load_run(const unsigned char *p) {
  Run<ELEM, V> r;
  constexpr int B = Run<ELEM, V>::kBytes;
  if constexpr (B >= 16) {
#pragma unroll
    for (int i = 0; i < B / 16; ++i) {
      const u32x4 v = load16_any(p + 16 * i);
#pragma unroll
      for (int d = 0; d < 4; ++d) r.w[4 * i + d] = v[d];
    }
  } else if constexpr (B == 4) {
    r.w[0] = load4_any(p);
  } else {
    r.w[0] = *(const unsigned short *)p;
  }
  return r;
}
template <int ELEM, int V>
__device__ __forceinline__ void unpack(const Run<ELEM, V> &r, float (&x)[V]) {
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if constexpr (ELEM == TCU_ELEM_F32) {
      x[e] = bitcast<float>(r.w[e]);
    } else {
      const unsigned half = (r.w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
      if constexpr (ELEM == TCU_ELEM_F16)
        x[e] = (float)bitcast<_Float16>((unsigned short)half);
      else
        x[e] = bf16_to_f32(half);
    }
  }
}

template <int ELEM, int V>
__device__ __forceinline__ void store_run(unsigned char *p, const float (&x)[V]) {
  if constexpr (V == 1) {
    f32_to_elem<ELEM>(p, x[0]);
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x[e];
    const Raw8<ELEM> r = pack8<ELEM>(v);
#pragma unroll
    for (int i = 0; i < elem_bytes<ELEM> / 2; ++i) store16_any(p + 16 * i, r.v[i]);
  }
}

// Slot j's two runs, and whether they are rotated.  An odd head's last slot has no second
// run (V = 1); the first `skip` values of a run are another slot's too (V = 8).
struct Slot {
  int lo, hi, skip_lo, skip_hi, at;   // at: the first pair's angle
  bool in, two, turned;
};
template <int V>
__device__ __forceinline__ Slot slot_of(int j, int dim, int rot, bool adjacent) {
  Slot s;
  const int turned = (rot / 2 + V - 1) / V, rest = (dim - rot + 2 * V - 1) / (2 * V);
  s.turned = j < turned;
  s.in = j < turned + rest;
  s.skip_lo = s.skip_hi = 0;
  if (s.turned && !adjacent) {
    s.at = V > 1 ? min(V * j, rot / 2 - V) : j;
    s.lo = s.at;
    s.hi = s.lo + rot / 2;
    s.skip_lo = s.skip_hi = V * j - s.at;
  } else {
    // 2 V neighbouring elements
    const int first = s.turned ? 2 * V * j : rot + 2 * V * (j - turned);
    s.lo = V > 1 ? min(first, (s.turned ? rot : dim) - 2 * V) : first;
    s.hi = s.lo + V;
    s.at = s.lo / 2;
    s.skip_lo = min(first - s.lo, V);
    s.skip_hi = first - s.lo - s.skip_lo;
  }
  s.two = s.hi < dim;
  return s;
}

// One wave's tables: cos and sin of its token's angles.
constexpr int kAngles = TCU_MAX_HEAD_DIM / 2;

// cos and sin of pos * freq.  The product and its share of a turn are formed with their
// rounding errors, so that the angle is right to binary32 at any position.
__device__ __forceinline__ void angle_of(int pos, float freq, float &c, float &s) {
  constexpr double kTurn = 0.15915494309189535, kTurnLow = -9.8393380152725e-18;   // 1 / 2 pi
  const double p = (double)pos, f = (double)freq;
  const double a = p * f, a_low = __builtin_fma(p, f, -a);
  const double t = a * kTurn;
  double r = t - __builtin_rint(t);
  r += __builtin_fma(a, kTurn, -t) + (a * kTurnLow + a_low * kTurn);
  sincospif(2.f * (float)r, &s, &c);
}

// Turns a lane's pairs by their angles (back: by the negative ones).
template <int V>
__device__ __forceinline__ void turn(float (&lo)[V], float (&hi)[V], const float (&c)[V],
                                     const float (&s)[V], bool adjacent, float sign) {
  if (V == 1 || !adjacent) {
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float a = lo[e], b = hi[e], si = sign * s[e];
      lo[e] = a * c[e] - b * si;
      hi[e] = a * si + b * c[e];
    }
  } else if constexpr (V > 1) {
#pragma unroll
    for (int e = 0; e < V / 2; ++e) {
      float a = lo[2 * e], b = lo[2 * e + 1], si = sign * s[e];
      lo[2 * e] = a * c[e] - b * si;
      lo[2 * e + 1] = a * si + b * c[e];
      a = hi[2 * e], b = hi[2 * e + 1], si = sign * s[V / 2 + e];
      hi[2 * e] = a * c[V / 2 + e] - b * si;
      hi[2 * e + 1] = a * si + b * c[V / 2 + e];
    }
  }
}

// The sum over L lanes, a power of two, for each of them.  (L is the same for all lanes of
// a launch: the steps not taken are branches.)
template <int kCtrl>
__device__ __forceinline__ float add_dpp(float v) {
  return v + bitcast<float>(__builtin_amdgcn_mov_dpp(bitcast<int>(v), kCtrl, 0xf, 0xf, true));
}
__device__ __forceinline__ float group_sum(float v, int L) {
  if (L > 1) v = add_dpp<0xB1>(v);    // lanes 1 0 3 2 of a quad
  if (L > 2) v = add_dpp<0x4E>(v);    // lanes 2 3 0 1
  if (L > 4) v = add_dpp<0x141>(v);   // 8 lanes mirrored: the other quad
  if (L > 8) v = add_dpp<0x140>(v);   // 16 lanes mirrored: the other eight
  if (L > 16) v += __shfl_xor(v, 16);
  if (L > 32) v += __shfl_xor(v, 32);
  return v;
}

// (without an eps a head of zeros has none to divide by: 0, not NaN)
__device__ __forceinline__ float rstd_of(float sum_sq, int dim, float eps) {
  const float v = sum_sq / (float)dim + eps;
  return v == 0.f ? 0.f : 1.f / sqrtf(v);
}

// A wave's task: `tokens` tokens, or one token's part of `heads` heads, of `parts` (tokens =
// 1).  The next task is `step` such groups of tokens and `rest` parts further.  A wave's
// next heads are at_once further: skip_tokens tokens and skip_heads heads.
struct Tasks {
  int64_t step;
  int tokens, parts, heads, rest, skip_tokens, skip_heads;
};

// A wave's pairs of one lane: slots lane % L + 64 i (kP > 1: L is 64).  The next heads'
// values are on their way while a wave's heads are worked on.  kShared: slots may share
// values.  Four waves on a SIMD, gradients two: five and three, for 16-bit types, spill (52
// sizes 23 % slower in the mean, 59 sizes 9 %).
template <int ELEM, int V, int kP, bool kGrad, bool kShared>
__global__ __launch_bounds__(64 * kWaves, kP > 1 ? 1 : kGrad ? 2 : 4) void heads_kernel(
    QkNormArgs a, int L, Tasks by) {
  constexpr int ES = elem_bytes<ELEM>;
  // tables of angles, or the gradient's sums: kWaves x 64 / L x 2 dim values, dim at most
  // 2 V kP L
  constexpr int kTables = kWaves * 2 * kAngles, kSums = kGrad ? kWaves * 256 * V * kP : 0;
  __shared__ __attribute__((aligned(16))) float lds[kTables > kSums ? kTables : kSums];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j0 = lane & (L - 1), sub = lane / L;
  const int H = a.heads[0] + a.heads[1], half = a.rot / 2;
  float *const cosines = lds + wave * 2 * kAngles, *const sines = cosines + kAngles;

  Slot slot[kP];
#pragma unroll
  for (int i = 0; i < kP; ++i) slot[i] = slot_of<V>(j0 + 64 * i, a.dim, a.rot, a.adjacent);
  // whether a value is this slot's alone to add
  auto own = [&](int i, int r, int e) {
    return !kShared || e >= (r ? slot[i].skip_hi : slot[i].skip_lo);
  };
  float dw[2][kP][2][V];
  if constexpr (kGrad) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[s][i][0][e] = dw[s][i][1][e] = 0.f;
  }

  typedef Run<ELEM, V> R;
  R rx[kP][2], rd[kGrad ? kP : 1][2];
  // a head's values of x and of the gradient (lanes without one: zeros)
  auto fetch = [&](int64_t token, int h, bool live) {
    const int which = h >= a.heads[0] ? 1 : 0;
    const int64_t hh = which ? h - a.heads[0] : h;
    const Heads hx = which ? a.x[1] : a.x[0];
    const unsigned char *px = (const unsigned char *)hx.p + (token * hx.ld + hh * hx.hd) * ES;
    const Heads hd = which ? a.dy[1] : a.dy[0];
    const unsigned char *pd = (const unsigned char *)hd.p + (token * hd.ld + hh * hd.hd) * ES;
#pragma unroll
    for (int i = 0; i < kP; ++i) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        rx[i][r] = R{};
        if constexpr (kGrad) rd[i][r] = R{};
      }
      if (live && slot[i].in) {
        rx[i][0] = load_run<ELEM, V>(px + slot[i].lo * ES);
        if constexpr (kGrad) rd[i][0] = load_run<ELEM, V>(pd + slot[i].lo * ES);
        if (slot[i].two) {
          rx[i][1] = load_run<ELEM, V>(px + slot[i].hi * ES);
          if constexpr (kGrad) rd[i][1] = load_run<ELEM, V>(pd + slot[i].hi * ES);
        }
      }
    }
  };

  // the task: its first token, how many, and its heads' end; the lane's first head
  const int first = blockIdx.x * kWaves + wave;
  int64_t group = first / by.parts;
  int part = first - (int)group * by.parts;
  // (of several tokens: the lane's first head in any task)
  const int tok0 = by.tokens > 1 ? sub / H : 0, head0 = by.tokens > 1 ? sub - tok0 * H : sub;
  int64_t token = group * by.tokens;
  int h = part * by.heads + head0;   // the lane's head, of token + tok
  int tok = tok0, h_end = min(H, (part + 1) * by.heads);
  int count = (int)min((int64_t)by.tokens, a.tokens - token);
  // angle `lane` of a task's tokens, whose position is loaded a task ahead
  const int angle_tok = half > 0 ? lane / half : 0, angle_at = lane - angle_tok * half;
  const float freq0 = half > 0 ? a.freq[angle_at] : 0.f;
  int pos = 0;
  auto fetch_pos = [&](int64_t token, int count) {
    if (angle_tok < count) pos = a.pos[token + angle_tok];
  };
  if (token < a.tokens) {
    if (half > 0) fetch_pos(token, count);
    fetch(token + tok, h, tok < count && h < h_end);
  }
  while (token < a.tokens) {
    part += by.rest;
    const bool carry = part >= by.parts;
    if (carry) part -= by.parts;
    group += by.step + carry;
    const int64_t next_token = group * by.tokens;
    const int next_h = part * by.heads + head0, next_end = min(H, (part + 1) * by.heads);
    const int next_count = (int)min((int64_t)by.tokens, a.tokens - next_token);
    if (half > 0) {
      for (int i = lane; i < count * half; i += 64) {
        if (i == lane) {
          angle_of(pos, freq0, cosines[i], sines[i]);
        } else {
          const int t = i / half;
          angle_of(a.pos[token + t], a.freq[i - t * half], cosines[i], sines[i]);
        }
      }
      // the wave's own values: in order, once they are written
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (next_token < a.tokens) fetch_pos(next_token, next_count);
    }

    while (true) {
      const bool live = tok < count && h < h_end;
      const int which = live && h >= a.heads[0] ? 1 : 0;
      const int64_t hh = which ? h - a.heads[0] : h;
      const int64_t at_token = token + tok;
      const int table = live ? tok * half : 0;
      // the next heads: of this task, or the next one's first
      h += by.skip_heads;
      tok += by.skip_tokens;
      if (by.tokens > 1 && h >= H) {
        h -= H;
        ++tok;
      }
      const bool more = __any(tok < count && h < h_end);
      // (the weights are in the caches)
      const unsigned char *pw = (const unsigned char *)(which ? a.w[1] : a.w[0]);
      R rw[kP][2];
#pragma unroll
      for (int i = 0; i < kP; ++i) {
        rw[i][0] = rw[i][1] = R{};
        if (live && slot[i].in) {
          rw[i][0] = load_run<ELEM, V>(pw + slot[i].lo * ES);
          if (slot[i].two) rw[i][1] = load_run<ELEM, V>(pw + slot[i].hi * ES);
        }
      }
      float x[kP][2][V], w[kP][2][V], d[kP][2][V];
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < kP; ++i) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          unpack<ELEM, V>(rx[i][r], x[i][r]);
          unpack<ELEM, V>(rw[i][r], w[i][r]);
          if constexpr (kGrad) unpack<ELEM, V>(rd[i][r], d[i][r]);
#pragma unroll
          for (int e = 0; e < V; ++e)
            sq += own(i, r, e) ? x[i][r][e] * x[i][r][e] : 0.f;
        }
      }
      // (in place, nobody's outputs are another's inputs)
      if (more)
        fetch(token + tok, h, tok < count && h < h_end);
      else if (next_token < a.tokens)
        fetch(next_token + tok0, next_h, tok0 < next_count && next_h < next_end);
      // (read by every lane at once, also by those that turn nothing)
      float c[kP][V], s[kP][V];
#pragma unroll
      for (int i = 0; i < kP; ++i) {
        const int at = table + (slot[i].turned ? slot[i].at : 0);
        if constexpr (V == 8 && !kShared) {
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const f32x4 cv = *(const f32x4 *)(cosines + at + 4 * k);
            const f32x4 sv = *(const f32x4 *)(sines + at + 4 * k);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              c[i][4 * k + e] = cv[e];
              s[i][4 * k + e] = sv[e];
            }
          }
        } else {
#pragma unroll
          for (int e = 0; e < V; ++e) {
            c[i][e] = cosines[at + e];
            s[i][e] = sines[at + e];
          }
        }
      }
      const float rstd = rstd_of(group_sum(sq, L), a.dim, a.eps);
      const Heads hy = which ? a.y[1] : a.y[0];
      unsigned char *py = (unsigned char *)hy.p + (at_token * hy.ld + hh * hy.hd) * ES;
      if constexpr (!kGrad) {
#pragma unroll
        for (int i = 0; i < kP; ++i) {
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][r][e] = x[i][r][e] * rstd * w[i][r][e];
          if (slot[i].turned) turn<V>(x[i][0], x[i][1], c[i], s[i], a.adjacent, 1.f);
        }
      } else {
        // (no head's values in the other weights' sums, also where they are not finite)
        const bool any_q = __any(live && !which), any_k = __any(which);
        float gn = 0.f;
#pragma unroll
        for (int i = 0; i < kP; ++i) {
          if (slot[i].turned) turn<V>(d[i][0], d[i][1], c[i], s[i], a.adjacent, -1.f);
#pragma unroll
          for (int r = 0; r < 2; ++r) {
            float t[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
              x[i][r][e] *= rstd;
              t[e] = d[i][r][e] * x[i][r][e];
              d[i][r][e] *= w[i][r][e];
              gn += own(i, r, e) ? d[i][r][e] * x[i][r][e] : 0.f;
            }
            if (!any_k) {
#pragma unroll
              for (int e = 0; e < V; ++e) dw[0][i][r][e] += t[e];
            } else if (!any_q) {
#pragma unroll
              for (int e = 0; e < V; ++e) dw[1][i][r][e] += t[e];
            } else {
#pragma unroll
              for (int e = 0; e < V; ++e) {
                dw[0][i][r][e] += which ? 0.f : t[e];
                dw[1][i][r][e] += which ? t[e] : 0.f;
              }
            }
          }
        }
        const float mean = group_sum(gn, L) / (float)a.dim;
#pragma unroll
        for (int i = 0; i < kP; ++i)
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) x[i][r][e] = rstd * (d[i][r][e] - x[i][r][e] * mean);
      }
#pragma unroll
      for (int i = 0; i < kP; ++i) {
        if (live && slot[i].in) {
          store_run<ELEM, V>(py + slot[i].lo * ES, x[i][0]);
          if (slot[i].two) store_run<ELEM, V>(py + slot[i].hi * ES, x[i][1]);
        }
      }
      if (!more) break;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // the angles are read
    token = next_token;
    count = next_count;
    h = next_h;
    h_end = next_end;
    tok = tok0;
  }

  if constexpr (kGrad) {
    // every lane's sums to LDS as they are, heads' rows one after the other: few instructions
    // (a kernel of few tokens waits for each of its own code's lines)
    const int rows = 64 / L;
    float *const mine = lds + (wave * rows + sub) * 2 * a.dim;
    __syncthreads();   // the tables are read
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const int at = r ? slot[i].hi : slot[i].lo;
          if (!slot[i].in || (r == 1 && !slot[i].two)) continue;
          if constexpr (V == 8 && !kShared) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const float *v = dw[s][i][r] + 4 * k;
              *(f32x4 *)(mine + s * a.dim + at + 4 * k) = f32x4{v[0], v[1], v[2], v[3]};
            }
          } else {
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (own(i, r, e)) mine[s * a.dim + at + e] = dw[s][i][r][e];
          }
        }
    __syncthreads();
    // the rows in `segs` pieces, a thread a column of one, and the pieces in their order
    const int cols = 2 * a.dim, all = kWaves * rows;
    const int segs = max(1, 64 * kWaves / cols), each = (all + segs - 1) / segs;
    const int seg = (int)threadIdx.x / cols, col = (int)threadIdx.x - seg * cols;
    float v = 0.f;
    if (segs > 1) {
      if (seg < segs) {
#pragma unroll 8
        for (int k = seg * each; k < min(all, (seg + 1) * each); ++k) v += lds[k * cols + col];
      }
      __syncthreads();   // the rows are read
      lds[threadIdx.x] = v;
      __syncthreads();
      if (seg == 0) {
        v = 0.f;
        for (int k = 0; k < segs; ++k) v += lds[k * cols + col];
        a.parts[(int64_t)blockIdx.x * cols + col] = v;
      }
      return;
    }
    for (int i = threadIdx.x; i < cols; i += 64 * kWaves) {
      v = 0.f;
#pragma unroll 8
      for (int k = 0; k < all; ++k) v += lds[k * cols + i];
      a.parts[(int64_t)blockIdx.x * cols + i] = v;
    }
  }
}

// dw: the parts' sums, 64 threads to a column, each in their order.
__global__ __launch_bounds__(1024) void head_dw_kernel(QkNormArgs a, int parts) {
  __shared__ float sums[64][17];
  const int col = threadIdx.x & 15, seg = threadIdx.x >> 4;
  const int i = blockIdx.x * 16 + col;
  float v = 0.f;
  if (i < 2 * a.dim) {
#pragma unroll 4
    for (int p = seg; p < parts; p += 64) v += a.parts[(int64_t)p * 2 * a.dim + i];
  }
  sums[seg][col] = v;
  __syncthreads();
  if (seg == 0 && i < 2 * a.dim) {
    v = 0.f;
#pragma unroll
    for (int s = 0; s < 64; ++s) v += sums[s][col];
    const int s = i >= a.dim;
    float *dw = s ? a.dw[1] : a.dw[0];
    if (dw) dw[i - s * a.dim] = v;
  }
}

int slots_of(const QkNormArgs &a, int V) {
  return (a.rot / 2 + V - 1) / V + (a.dim - a.rot + 2 * V - 1) / (2 * V);
}

template <int ELEM, int V, int kP, bool kGrad, bool kShared>
hipError_t launch(const QkNormArgs &a, hipStream_t stream, int num_cus) {
  const int slots = slots_of(a, V);
  int L = 1;
  while (L < slots && L < 64) L <<= 1;
  const int H = a.heads[0] + a.heads[1], at_once = 64 / L, half = a.rot / 2;
  const int rounds = (H + at_once - 1) / at_once;
  // waves for the whole chip: a token's heads are several waves' where tokens are few, and a
  // wave takes several tokens where they are many and rounds and angles are then fuller
  const int64_t waves = (int64_t)num_cus * (kGrad ? 8 : 16);
  Tasks by{0, 1, 1, rounds * at_once, 0, 0, at_once};
  if (a.tokens < waves) {
    by.parts = (int)std::min<int64_t>(rounds, waves / a.tokens);
    by.heads = (rounds + by.parts - 1) / by.parts * at_once;
    by.parts = (H + by.heads - 1) / by.heads;
  } else {
    // instructions of a round, of 64 angles and of a task, about, times the tasks of a wave:
    // between their mean and the most that one has.  More tokens only where that saves a
    // twentieth (us, bf16, one token / the rule: 20000 tokens of 18 heads of 64 26.8 / 20.0, of
    // 80, 40 of them turned, 40.4 / 31.1; 16 heads of 128 28.4, four tokens 31.9; rounded tasks
    // counted / the mean alone, 6000 tokens of 3 heads of 64 5.0 / 7.1, of 20 10.1 / 11.8).
    double least = 1e300;
    for (int n = 1; n <= 8 && n * half <= kAngles; ++n) {
      const int r = (n * H + at_once - 1) / at_once, angles = (n * half + 63) / 64;
      const int64_t groups = (a.tokens + n - 1) / n, most = (groups + waves - 1) / waves;
      const double mean = std::max(1.0, (double)groups / waves);
      const double each = 0.5 * (most + mean) * (r * 250.0 + angles * 150.0 + 100.0);
      if (each < 0.95 * least) {
        least = each;
        by.tokens = n;
      }
    }
    if (by.tokens > 1) {
      by.heads = H;
      by.skip_tokens = at_once / H;
      by.skip_heads = at_once % H;
    }
  }
  const int64_t groups = (a.tokens + by.tokens - 1) / by.tokens;
  const int64_t tasks = groups * by.parts;
  int64_t blocks = (tasks + kWaves - 1) / kWaves;
  blocks = std::min<int64_t>(blocks, kGrad ? kHeadParts : 8 * (int64_t)num_cus);
  by.step = blocks * kWaves / by.parts;
  by.rest = (int)(blocks * kWaves % by.parts);
  heads_kernel<ELEM, V, kP, kGrad, kShared><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(a, L, by);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !kGrad) return e;
  head_dw_kernel<<<(unsigned)((2 * a.dim + 15) / 16), 1024, 0, stream>>>(a, (int)blocks);
  return hipGetLastError();
}

// Whole vectors where each part of a head has room for a slot (us, 2000 tokens of 9 heads of
// 100 elements, 50 of them turned, by vectors / by pairs: 6.7 / 9.7, gradients
// 15.4 / 20.1).
template <int ELEM, bool kGrad>
hipError_t pick(const QkNormArgs &a, hipStream_t stream, int num_cus) {
  const int rest = a.dim - a.rot;
  if (a.rot % 16 == 0 && rest % 16 == 0)
    return launch<ELEM, 8, 1, kGrad, false>(a, stream, num_cus);
  if ((a.rot == 0 || a.rot >= 16) && (rest == 0 || rest >= 16) && slots_of(a, 8) <= 64)
    return launch<ELEM, 8, 1, kGrad, true>(a, stream, num_cus);
  if (slots_of(a, 1) <= 64) return launch<ELEM, 1, 1, kGrad, false>(a, stream, num_cus);
  return launch<ELEM, 1, 8, kGrad, false>(a, stream, num_cus);
}

__global__ void zero_dw_kernel(QkNormArgs a) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= a.dim) return;
#pragma unroll
  for (int s = 0; s < 2; ++s)
    if (a.dw[s]) a.dw[s][i] = 0.f;
}

}  // namespace

hipError_t launch_qk_norm(int elem, const QkNormArgs &a, hipStream_t stream, int num_cus) {
  switch (elem) {
    case TCU_ELEM_F32: return pick<TCU_ELEM_F32, false>(a, stream, num_cus);
    case TCU_ELEM_F16: return pick<TCU_ELEM_F16, false>(a, stream, num_cus);
    default: return pick<TCU_ELEM_BF16, false>(a, stream, num_cus);
  }
}

hipError_t launch_qk_norm_grad(int elem, const QkNormArgs &a, hipStream_t stream, int num_cus) {
  if (a.tokens == 0) {
    zero_dw_kernel<<<(unsigned)((a.dim + 255) / 256), 256, 0, stream>>>(a);
    return hipGetLastError();
  }
  switch (elem) {
    case TCU_ELEM_F32: return pick<TCU_ELEM_F32, true>(a, stream, num_cus);
    case TCU_ELEM_F16: return pick<TCU_ELEM_F16, true>(a, stream, num_cus);
    default: return pick<TCU_ELEM_BF16, true>(a, stream, num_cus);
  }
}

}  // namespace tcu

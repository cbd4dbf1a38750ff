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
//     they are adjacent both runs hold whole pairs.  V is 8 where the sizes allow whole
//     vectors, down to 1 for any size; heads that need more than 64 lanes of one pair
//     have kP pairs a lane.
//   * A wave takes a token and as many of its heads at once as fit, queries and keys in
//     one sequence; the angles are formed once a token, one lane each, in binary64 (a
//     far position's angle has no digits left in binary32), and shared through LDS.
//   * The weights' gradients are summed in registers over a workgroup's tokens, and the
//     workgroups' parts by a second launch, in their order.
#include <algorithm>

#include "tcu_elem.h"
#include "tcu_heads.h"

namespace tcu {
namespace {

constexpr int kWaves = 4;

// V elements as stored, at any element-aligned address.
template <int ELEM, int V>
__device__ __forceinline__ void load_run(const unsigned char *p, float (&x)[V]) {
  constexpr int ES = elem_bytes<ELEM>;
  if constexpr (V == 8) {
    const Raw8<ELEM> r = load8<ELEM>(p, 8);
    unpack8<ELEM>(r, x);
  } else if constexpr (V * ES >= 4) {
    unsigned w[V * ES / 4];
    if constexpr (V * ES == 16) {
      const u32x4 v = load16_any(p);
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = v[i];
    } else if constexpr (V * ES == 8) {
      typedef u32x2 u32x2_any __attribute__((aligned(1)));
      const u32x2 v = *(const u32x2_any *)p;
      w[0] = v[0];
      w[1] = v[1];
    } else {
      w[0] = load4_any(p);
    }
#pragma unroll
    for (int e = 0; e < V; ++e) {
      if constexpr (ELEM == TCU_ELEM_F32) {
        x[e] = bitcast<float>(w[e]);
      } else {
        const unsigned half = (w[e >> 1] >> (16 * (e & 1))) & 0xffffu;
        if constexpr (ELEM == TCU_ELEM_F16)
          x[e] = (float)bitcast<_Float16>((unsigned short)half);
        else
          x[e] = bf16_to_f32(half);
      }
    }
  } else {
    x[0] = elem_to_f32<ELEM>(p);
  }
}

template <int ELEM, int V>
__device__ __forceinline__ void store_run(unsigned char *p, const float (&x)[V]) {
  constexpr int ES = elem_bytes<ELEM>;
  if constexpr (V == 1) {
    f32_to_elem<ELEM>(p, x[0]);
  } else {
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = e < V ? x[e] : 0.f;
    const Raw8<ELEM> r = pack8<ELEM>(v);
    if constexpr (V == 8) {
#pragma unroll
      for (int i = 0; i < ES / 2; ++i) store16_any(p + 16 * i, r.v[i]);
    } else if constexpr (V * ES == 16) {
      store16_any(p, r.v[0]);
    } else if constexpr (V * ES == 8) {
      typedef u32x2 u32x2_any __attribute__((aligned(1)));
      *(u32x2_any *)p = u32x2{r.v[0][0], r.v[0][1]};
    } else {
      store4_any(p, r.v[0][0]);
    }
  }
}

// Slot j's two runs, and whether they are rotated.  An odd head's last slot has no
// second run (one pair a slot).
struct Slot {
  int lo, hi;
  bool in, two, turned;
};
template <int V>
__device__ __forceinline__ Slot slot_of(int j, int dim, int rot, bool adjacent) {
  Slot s;
  const int turned = rot / (2 * V);
  s.turned = j < turned;
  if (s.turned) {
    s.lo = adjacent ? 2 * V * j : V * j;
    s.hi = adjacent ? s.lo + V : s.lo + rot / 2;
  } else {
    s.lo = rot + 2 * V * (j - turned);
    s.hi = s.lo + V;
  }
  s.in = s.lo < dim;
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

__device__ __forceinline__ float group_sum(float v, int L) {
  for (int m = 1; m < L; m <<= 1) v += __shfl_xor(v, m);
  return v;
}

// (without an eps a head of zeros has none to divide by: 0, not NaN)
__device__ __forceinline__ float rstd_of(float sum_sq, int dim, float eps) {
  const float v = sum_sq / (float)dim + eps;
  return v == 0.f ? 0.f : 1.f / sqrtf(v);
}

// A token's pairs of one lane: slots lane % L + 64 i (kP > 1: L is 64).
template <int ELEM, int V, int kP, bool kGrad>
__global__ __launch_bounds__(64 * kWaves) void heads_kernel(QkNormArgs a, int L, int64_t token_tasks,
                                                          int head_tasks, int heads_per_task) {
  constexpr int ES = elem_bytes<ELEM>;
  __shared__ float tables[kWaves][2][kAngles];
  __shared__ float sums[kGrad ? kWaves : 1][2][kGrad ? TCU_MAX_HEAD_DIM : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int j0 = lane & (L - 1), sub = lane / L, at_once = 64 / L;
  const int H = a.heads[0] + a.heads[1];

  Slot slot[kP];
#pragma unroll
  for (int i = 0; i < kP; ++i) slot[i] = slot_of<V>(j0 + 64 * i, a.dim, a.rot, a.adjacent);
  float dw[2][kP][2][V];
  if constexpr (kGrad) {
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int e = 0; e < V; ++e) dw[s][i][0][e] = dw[s][i][1][e] = 0.f;
  }

  const int64_t tasks = token_tasks * head_tasks;
  for (int64_t task = (int64_t)blockIdx.x * kWaves + wave; task < tasks;
       task += (int64_t)gridDim.x * kWaves) {
    const int64_t token = task / head_tasks;
    const int h0 = (int)(task - token * head_tasks) * heads_per_task;
    const int h1 = min(H, h0 + heads_per_task);
    float c[kP][V], s[kP][V];
    if (a.rot > 0) {
      const int pos = a.pos[token];
      for (int i = lane; i < a.rot / 2; i += 64)
        angle_of(pos, a.freq[i], tables[wave][0][i], tables[wave][1][i]);
      // the wave's own values: in order, once they are written
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int i = 0; i < kP; ++i)
#pragma unroll
      for (int e = 0; e < V; ++e) {
        const int at = (j0 + 64 * i) * V + e;
        c[i][e] = slot[i].turned ? tables[wave][0][at] : 1.f;
        s[i][e] = slot[i].turned ? tables[wave][1][at] : 0.f;
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // read before the next token's are written

    for (int hb = h0; hb < h1; hb += at_once) {
      const int h = hb + sub;
      const bool live = h < h1;
      const int which = h >= a.heads[0] && live ? 1 : 0;
      const int64_t hh = which ? h - a.heads[0] : h;
      const Heads hx = which ? a.x[1] : a.x[0];
      const unsigned char *px = (const unsigned char *)hx.p + (token * hx.ld + hh * hx.hd) * ES;
      const unsigned char *pw = (const unsigned char *)(which ? a.w[1] : a.w[0]);
      float x[kP][2][V], w[kP][2][V], d[kP][2][V];
      float sq = 0.f;
#pragma unroll
      for (int i = 0; i < kP; ++i) {
#pragma unroll
        for (int e = 0; e < V; ++e) x[i][0][e] = x[i][1][e] = w[i][0][e] = w[i][1][e] = 0.f;
        if (live && slot[i].in) {
          load_run<ELEM, V>(px + slot[i].lo * ES, x[i][0]);
          load_run<ELEM, V>(pw + slot[i].lo * ES, w[i][0]);
          if (slot[i].two) {
            load_run<ELEM, V>(px + slot[i].hi * ES, x[i][1]);
            load_run<ELEM, V>(pw + slot[i].hi * ES, w[i][1]);
          }
        }
        if constexpr (kGrad) {
#pragma unroll
          for (int e = 0; e < V; ++e) d[i][0][e] = d[i][1][e] = 0.f;
          const Heads hd = which ? a.dy[1] : a.dy[0];
          const unsigned char *pd = (const unsigned char *)hd.p + (token * hd.ld + hh * hd.hd) * ES;
          if (live && slot[i].in) {
            load_run<ELEM, V>(pd + slot[i].lo * ES, d[i][0]);
            if (slot[i].two) load_run<ELEM, V>(pd + slot[i].hi * ES, d[i][1]);
          }
        }
#pragma unroll
        for (int e = 0; e < V; ++e) sq += x[i][0][e] * x[i][0][e] + x[i][1][e] * x[i][1][e];
      }
      const float rstd = rstd_of(group_sum(sq, L), a.dim, a.eps);
      const Heads hy = which ? a.y[1] : a.y[0];
      unsigned char *py = (unsigned char *)hy.p + (token * hy.ld + hh * hy.hd) * ES;
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
        float gn = 0.f;
#pragma unroll
        for (int i = 0; i < kP; ++i) {
          if (slot[i].turned) turn<V>(d[i][0], d[i][1], c[i], s[i], a.adjacent, -1.f);
#pragma unroll
          for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int e = 0; e < V; ++e) {
              x[i][r][e] *= rstd;
              const float t = d[i][r][e] * x[i][r][e];
              dw[0][i][r][e] += which ? 0.f : t;
              dw[1][i][r][e] += which ? t : 0.f;
              d[i][r][e] *= w[i][r][e];
              gn += d[i][r][e] * x[i][r][e];
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
    }
  }

  if constexpr (kGrad) {
    // the wave's lanes of one slot, then the waves
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
      for (int i = 0; i < kP; ++i)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
          for (int e = 0; e < V; ++e) {
            float v = dw[s][i][r][e];
            for (int m = L; m < 64; m <<= 1) v += __shfl_xor(v, m);
            const int at = (r ? slot[i].hi : slot[i].lo) + e;
            if (sub == 0 && (r ? slot[i].two : slot[i].in)) sums[wave][s][at] = v;
          }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.dim; i += 64 * kWaves) {
      const int s = i >= a.dim, at = i - s * a.dim;
      float v = 0.f;
#pragma unroll
      for (int k = 0; k < kWaves; ++k) v += sums[k][s][at];
      a.parts[(int64_t)blockIdx.x * 2 * a.dim + i] = v;
    }
  }
}

// dw: the parts' sums, 16 threads to a column, each in their order.
__global__ __launch_bounds__(256) void head_dw_kernel(QkNormArgs a, int parts) {
  __shared__ float sums[16][17];
  const int col = threadIdx.x & 15, seg = threadIdx.x >> 4;
  const int i = blockIdx.x * 16 + col;
  float v = 0.f;
  if (i < 2 * a.dim)
    for (int p = seg; p < parts; p += 16) v += a.parts[(int64_t)p * 2 * a.dim + i];
  sums[seg][col] = v;
  __syncthreads();
  if (seg == 0 && i < 2 * a.dim) {
    v = 0.f;
#pragma unroll
    for (int s = 0; s < 16; ++s) v += sums[s][col];
    const int s = i >= a.dim;
    float *dw = s ? a.dw[1] : a.dw[0];
    if (dw) dw[i - s * a.dim] = v;
  }
}

template <int ELEM, int V, int kP, bool kGrad>
hipError_t launch(const QkNormArgs &a, hipStream_t stream, int num_cus) {
  const int slots = (a.dim + 2 * V - 1) / (2 * V);
  int L = 1;
  while (L < slots && L < 64) L <<= 1;
  const int H = a.heads[0] + a.heads[1], at_once = 64 / L;
  const int rounds = (H + at_once - 1) / at_once;
  // waves for the whole chip: a token's heads are several waves' where tokens are few
  const int64_t waves = (int64_t)num_cus * (kGrad ? 8 : 16);
  const int head_tasks =
      (int)std::max<int64_t>(1, std::min<int64_t>(rounds, waves / std::max<int64_t>(a.tokens, 1)));
  const int per_task = (rounds + head_tasks - 1) / head_tasks * at_once;
  const int tasks_h = (H + per_task - 1) / per_task;
  const int64_t tasks = a.tokens * tasks_h;
  int64_t blocks = (tasks + kWaves - 1) / kWaves;
  blocks = std::min<int64_t>(blocks, kGrad ? kHeadParts : 8 * (int64_t)num_cus);
  heads_kernel<ELEM, V, kP, kGrad><<<(unsigned)blocks, 64 * kWaves, 0, stream>>>(
      a, L, a.tokens, tasks_h, per_task);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !kGrad) return e;
  head_dw_kernel<<<(unsigned)((2 * a.dim + 15) / 16), 256, 0, stream>>>(a, (int)blocks);
  return hipGetLastError();
}

// The widest runs that a head's rotated and other parts are whole numbers of.
template <int ELEM, bool kGrad>
hipError_t pick(const QkNormArgs &a, hipStream_t stream, int num_cus) {
  const int rest = a.dim - a.rot;
  const auto fits = [&](int v) { return a.rot % (2 * v) == 0 && rest % (2 * v) == 0; };
  if (fits(8)) return launch<ELEM, 8, 1, kGrad>(a, stream, num_cus);
  if (fits(4) && a.dim <= 512) return launch<ELEM, 4, 1, kGrad>(a, stream, num_cus);
  if (fits(2) && a.dim <= 256) return launch<ELEM, 2, 1, kGrad>(a, stream, num_cus);
  if (a.dim <= 128) return launch<ELEM, 1, 1, kGrad>(a, stream, num_cus);
  return launch<ELEM, 1, 8, kGrad>(a, stream, num_cus);
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

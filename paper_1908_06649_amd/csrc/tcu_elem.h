// Element access of the layer operators: 16-bit and binary32 values to binary32
// and back, eight at a time at any element-aligned address.
#pragma once

#include "tcu_device.h"

namespace tcu {

template <int ELEM>
constexpr int elem_bytes = ELEM == TCU_ELEM_F32 ? 4 : 2;

// Eight elements as stored: 16 bytes, or 32 of binary32.
template <int ELEM>
struct Raw8 {
  u32x4 v[elem_bytes<ELEM> / 2];
};

template <int ELEM>
__device__ __forceinline__ float elem_to_f32(const unsigned char *p) {
  if constexpr (ELEM == TCU_ELEM_F32) return *(const float *)p;
  else if constexpr (ELEM == TCU_ELEM_F16) return (float)*(const _Float16 *)p;
  else return bf16_to_f32(*(const unsigned short *)p);
}

template <int ELEM>
__device__ __forceinline__ void f32_to_elem(unsigned char *p, float x) {
  if constexpr (ELEM == TCU_ELEM_F32) *(float *)p = x;
  else if constexpr (ELEM == TCU_ELEM_F16) *(_Float16 *)p = (_Float16)x;
  else *(unsigned short *)p = (unsigned short)(pack_bf16x2(x, 0.f) & 0xffffu);
}

// The first `valid` (1..8) of eight elements at p; the others are zero and
// are not read.
template <int ELEM>
__device__ __forceinline__ Raw8<ELEM> load8(const unsigned char *p, int valid) {
  constexpr int ES = elem_bytes<ELEM>, EPC = 16 / ES;
  Raw8<ELEM> r;
#pragma unroll
  for (int i = 0; i < 8 / EPC; ++i)
    r.v[i] = valid >= 8 ? load16_any(p + 16 * i) : u32x4{0u, 0u, 0u, 0u};
  if (valid < 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e < valid) {
        const unsigned x = ES == 2 ? (unsigned)((const unsigned short *)p)[e]
                                   : ((const unsigned *)p)[e];
        r.v[e / EPC][(e % EPC) * ES / 4] |= ES == 2 ? x << (16 * (e & 1)) : x;
      }
    }
  }
  return r;
}

template <int ELEM>
__device__ __forceinline__ void unpack8(const Raw8<ELEM> &r, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    if constexpr (ELEM == TCU_ELEM_F32) {
      x[e] = bitcast<float>(r.v[e >> 2][e & 3]);
    } else {
      const unsigned half = (r.v[0][e >> 1] >> (16 * (e & 1))) & 0xffffu;
      if constexpr (ELEM == TCU_ELEM_F16)
        x[e] = (float)bitcast<_Float16>((unsigned short)half);
      else
        x[e] = bf16_to_f32(half);
    }
  }
}

template <int ELEM>
__device__ __forceinline__ Raw8<ELEM> pack8(const float (&x)[8]) {
  Raw8<ELEM> r;
  if constexpr (ELEM == TCU_ELEM_F32) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e >> 2][e & 3] = bitcast<unsigned>(x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (ELEM == TCU_ELEM_F16) {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        r.v[0][e] = bitcast<unsigned>(f16x2{(_Float16)x[2 * e], (_Float16)x[2 * e + 1]});
      } else {
        r.v[0][e] = pack_bf16x2(x[2 * e], x[2 * e + 1]);
      }
    }
  }
  return r;
}

// Store the first `valid` (1..8) of eight elements at p.
template <int ELEM>
__device__ __forceinline__ void store8(unsigned char *p, const float (&x)[8], int valid) {
  constexpr int ES = elem_bytes<ELEM>;
  if (valid >= 8) {
    const Raw8<ELEM> r = pack8<ELEM>(x);
#pragma unroll
    for (int i = 0; i < ES / 2; ++i) store16_any(p + 16 * i, r.v[i]);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (e < valid) f32_to_elem<ELEM>(p + e * ES, x[e]);
  }
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m);
  return v;
}
__device__ __forceinline__ unsigned wave_max(unsigned v) {
#pragma unroll
  for (int m = 32; m > 0; m >>= 1) {
    const unsigned o = __shfl_xor(v, m);
    v = o > v ? o : v;
  }
  return v;
}

}  // namespace tcu

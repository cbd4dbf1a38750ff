// Device side of the 4-bit format (OCP microscaling: e2m1 values, a power-of-two
// scale for every block of 32 along the contracted index).
#pragma once

#include "tcu_elem.h"
#include "tcu_mx4.h"

namespace tcu {

constexpr unsigned kNotFinite = 0x7f800000u;

__device__ __forceinline__ unsigned abs_bits(float v) { return bitcast<unsigned>(v) & 0x7fffffffu; }
__device__ __forceinline__ unsigned umax(unsigned a, unsigned b) { return a > b ? a : b; }

// The scale byte of a block whose largest magnitude has these bits: the exponent of
// the largest power of two in it less that of the codes' largest (2), so that it lies
// in [4, 8) scales; 255 for a block with a value that is not finite.
__device__ __forceinline__ unsigned scale_byte(unsigned max_bits) {
  const unsigned e = max_bits >> 23;
  return max_bits >= kNotFinite ? 255u : e > 2u ? e - 2u : 0u;
}

// Eight values of a block as codes, the first in the lowest bits: rounded to nearest
// even and clamped to 6.  Values near binary32's smallest are brought up together
// with their scale first (the conversion takes normal numbers).
__device__ __forceinline__ unsigned codes8(const float (&x)[8], unsigned byte) {
  if (byte == 255u) return 0u;
  const bool low = byte < 32u;
  const float scale = bitcast<float>((low ? byte + 32u : byte) << 23);
  unsigned c = 0;
  if (__builtin_expect(low, 0)) {
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0] * 0x1p32f, x[1] * 0x1p32f, scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2] * 0x1p32f, x[3] * 0x1p32f, scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4] * 0x1p32f, x[5] * 0x1p32f, scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6] * 0x1p32f, x[7] * 0x1p32f, scale, 3);
  }
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], scale, 2);
  return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], scale, 3);
}

// Lanes of a quad, and of a row of 16 lanes, exchanged in registers.
template <int kCtrl>
__device__ __forceinline__ unsigned dpp(unsigned v) {
  return (unsigned)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xf, 0xf, true);
}
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  v = umax(v, dpp<0xB1>(v));   // lanes 1 0 3 2
  return umax(v, dpp<0x4E>(v));   // lanes 2 3 0 1
}
// The or over lanes of one position of the four quads of 16 lanes.
__device__ __forceinline__ unsigned quads_or(unsigned v) {
  v |= dpp<0x124>(v);   // a row of 16 turned by 4
  return v | dpp<0x128>(v);   // and by 8
}

}  // namespace tcu

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

// Whether a lane's block needs the slow conversion: its values or its scale may lie below
// binary32's normal numbers, which the conversion takes.
__device__ __forceinline__ bool scale_low(unsigned max_bits) {
  return max_bits != 0u && max_bits < 34u << 23;
}

// Eight values of a block as codes, the first in the lowest bits: rounded to nearest
// even and clamped to 6.  kLow: values are brought up by 2^32 together with their scale.
template <bool kLow>
__device__ __forceinline__ unsigned codes8(const float (&x)[8], unsigned byte) {
  const float up = kLow && byte < 32u ? 0x1p32f : 1.f;
  const unsigned e = kLow && byte < 32u ? byte + 32u : byte;
  const float scale = bitcast<float>((e > 1u ? e : 1u) << 23);   // (a block of zeros: any)
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = kLow ? x[i] * up : x[i];
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], scale, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], scale, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], scale, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], scale, 3);
  return byte == 255u ? 0u : c;
}
// any_low: whether any lane of the wave has a low block (uniform).
__device__ __forceinline__ unsigned codes8(const float (&x)[8], unsigned byte, bool any_low) {
  return __builtin_expect(any_low, 0) ? codes8<true>(x, byte) : codes8<false>(x, byte);
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

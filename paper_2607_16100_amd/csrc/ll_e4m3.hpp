// 8-bit values with a power-of-two scale a block (include/llblock.h).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "ll_num.hpp"

namespace llc {

constexpr uint32_t kBlock = 128;  // LL_BLOCK

// Bits of the magnitude of a finite value; 0 for the others, which no scale counts.
__device__ __forceinline__ uint32_t finite_bits(float v) {
  const uint32_t b = (uint32_t)__float_as_int(v) & 0x7FFFFFFFu;
  return b < 0x7F800000u ? b : 0u;
}

// Maximum over each aligned group of 16 lanes, in every lane.
template <int kCtrl>
__device__ __forceinline__ uint32_t dpp_u32(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, kCtrl, 0xF, 0xF, true);
}
__device__ __forceinline__ uint32_t max16(uint32_t v) {
  v = max(v, dpp_u32<0xB1>(v));
  v = max(v, dpp_u32<0x4E>(v));
  v = max(v, dpp_u32<0x141>(v));
  return max(v, dpp_u32<0x140>(v));
}

// The scale (exponent + 127) of a block whose largest magnitude has these bits:
// the least power of two with the magnitude at most 1.75 * 2^top of it, 448 =
// 1.75 * 2^8 for e4m3 and 57344 = 1.75 * 2^15 for e5m2.  Magnitudes up to
// 2^(top - 125) have the least scale, 2^-126, whose inverse is a binary32 number.
template <int kTop>
__device__ __forceinline__ uint32_t scale_of(uint32_t bits) {
  const int s = (int)(bits >> 23) - kTop + ((bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(s, 1);
}
__device__ __forceinline__ float scale_value(uint32_t s) { return __int_as_float((int)(s << 23)); }
__device__ __forceinline__ float scale_inverse(uint32_t s) { return __int_as_float((int)((254u - s) << 23)); }

// a and b, scaled to at most 448, rounded to e4m3 in the low 16 bits; what is
// not finite becomes no number.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b) {
  a = fabsf(a) < __builtin_inff() ? a : __int_as_float(0x7FC00000);
  b = fabsf(b) < __builtin_inff() ? b : __int_as_float(0x7FC00000);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false) & 0xFFFFu;
}

// Four values, scaled to at most 448 or no numbers, in a word.
__device__ __forceinline__ uint32_t pack_e4m3(float a, float b, float c, float d) {
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
}

}  // namespace llc

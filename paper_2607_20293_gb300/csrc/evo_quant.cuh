// The 8-bit format of the caches: e4m3 codes with one power-of-two scale per
// group of values (32 values of a unit's cache, the row of one head in a paged
// memory).  The scale is 2^k for the least integer k >= -126 with
// amax <= 448 * 2^k (448 = 1.75 * 2^8 is the largest code), held as the byte
// k + 127; a code is x * 2^-k rounded to nearest even.  Scaling by a power of
// two is exact, so a stored value is off by the one rounding of the code (half
// a step: 2^-4 of the value, or 2^-10 * 2^k among the subnormal codes), the
// same on every path, and a value that is read back is exact in bf16 as well (its
// subnormals have steps of 2^-133; codes of the two smallest scales go to 2^-135).
// A group that holds a NaN or an infinity gets scale byte 255 and reads back
// as NaN.
#pragma once

#include <cstdint>

#include "evo_internal.h"

namespace evo {

constexpr uint32_t SCALE_NAN = 255;

// the scale byte for a group whose largest magnitude has these fp32 bits
__device__ __forceinline__ uint32_t scale_byte(uint32_t amax_bits) {
  if (amax_bits >= 0x7f800000u) return SCALE_NAN;
  const int k = (int)(amax_bits >> 23) - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(k, 1);
}

// 2^k of a scale byte (NaN for 255)
__device__ __forceinline__ float scale_value(uint32_t byte) {
  return __uint_as_float(byte == SCALE_NAN ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}

// 2^-k of a byte that scale_byte gave (1 .. 247)
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// largest magnitude as fp32 bits: unsigned order puts infinities above every
// finite value and NaN above those
__device__ __forceinline__ uint32_t amax_bits(uint32_t a, float x) { return max(a, __float_as_uint(x) & 0x7fffffffu); }

// maximum over groups of G consecutive lanes
template <int G>
__device__ __forceinline__ uint32_t group_umax(uint32_t v) {
#pragma unroll
  for (int o = G / 2; o > 0; o >>= 1) v = max(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// four codes of x * 2^-k, the first in the lowest byte
__device__ __forceinline__ uint32_t quantise4(float4 x, uint32_t byte) {
  if (byte == SCALE_NAN) return 0x7f7f7f7fu;
  const float i = scale_inverse(byte);
  uint16_t lo, hi;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(lo) : "f"(x.y * i), "f"(x.x * i));
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(hi) : "f"(x.w * i), "f"(x.z * i));
  return (uint32_t)lo | (uint32_t)hi << 16;
}

// the values of four codes, without their scale
__device__ __forceinline__ float4 codes4(uint32_t c) {
  uint32_t lo, hi;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(lo) : "h"((uint16_t)(c & 0xffffu)));
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(hi) : "h"((uint16_t)(c >> 16)));
  float4 v;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(v.x), "=f"(v.y) : "r"(lo));
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %2;\n cvt.f32.f16 %0, a;\n cvt.f32.f16 %1, b;\n}" : "=f"(v.z), "=f"(v.w) : "r"(hi));
  return v;
}

}  // namespace evo

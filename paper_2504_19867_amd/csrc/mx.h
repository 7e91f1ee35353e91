// Power-of-two block scales and the small formats under them (device code).
//
// A block of entries shares a scale 2^(b - 127), b one byte (E8M0).  b is the smallest with which the block's largest magnitude does not
// pass the format's largest value (E4M3: 448 = 1.75 2^8, E2M1: 6 = 1.5 2^2), and at least 1 (2^-126: the factors formed here are normal
// fp32 numbers).  Multiplying by such a scale or its inverse is exact, so that a code is its entry rounded once.
#pragma once

#include "internal.h"

namespace spd {

constexpr uint32_t MX_NAN_SCALE = 255;             // E8M0 NaN: the whole block is

// b for a block whose largest finite magnitude has the fp32 bits `m`.  emax, top: exponent and mantissa bits of the format's largest value.
template <int EMAX, uint32_t TOP>
__device__ inline uint32_t scale_byte(uint32_t m) {
  const int b = (int)(m >> 23) - EMAX + ((m & 0x7fffff) > TOP ? 1 : 0);
  return (uint32_t)max(b, 1);
}
__device__ inline uint32_t scale_byte_e4m3(uint32_t m) { return scale_byte<8, 0x600000>(m); }
__device__ inline uint32_t scale_byte_e2m1(uint32_t m) { return scale_byte<2, 0x400000>(m); }
// 2^(b - 127) and its inverse
__device__ inline float scale_of(uint32_t b) { return __builtin_bit_cast(float, b << 23); }
__device__ inline float inverse_scale_of(uint32_t b) { return __builtin_bit_cast(float, (254 - b) << 23); }
// the magnitude's bits of an entry that counts for its block's scale: infinities and NaN do not
__device__ inline uint32_t finite_magnitude(float x) {
  const uint32_t m = __builtin_bit_cast(uint32_t, x) & 0x7fffffff;
  return m < 0x7f800000 ? m : 0;
}
// Four entries (under their block's scale, magnitudes up to 448) as E4M3 codes, nearest even; infinities and NaN become NaN.
__device__ inline uint32_t e4m3_codes(float a, float b, float c, float d) {
  int pk = 0;
  pk = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, pk, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, pk, true);
}

}  // namespace spd

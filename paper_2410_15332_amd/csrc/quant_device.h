// Device helpers of the 8-bit operands: the scale of a group and the rounding to e4m3.
#pragma once

#include "device_common.h"

namespace epic {

// Order-preserving bits of |v|, 0 for infinities and NaN: a group's scale comes from its
// finite values.
__device__ __forceinline__ uint32_t finite_abs(float v) {
  const uint32_t a = __float_as_uint(v) & 0x7FFFFFFFu;
  return a < 0x7F800000u ? a : 0u;
}

// e8m0 byte t + 127 of the smallest t with top <= 448 * 2^t = 1.75 * 2^(t + 8), at least
// -127; t = 0 for a group of zeros.  Adding 0x1FFFFF carries into the exponent exactly
// where the fraction is above 1.75; the largest float gives 247.
__device__ __forceinline__ int scale_byte(uint32_t top) {
  const int e = int((top + 0x1FFFFFu) >> 23) - 8;
  return top == 0 ? 127 : max(e, 0);
}

// Four values over 2^(byte - 127), rounded to nearest even e4m3, in memory order.  Every
// finite one is at most 448 then; infinities, which e4m3 does not have, become NaN like NaN.
__device__ __forceinline__ uint32_t pack_e4m3x4(float a, float b, float c, float d, int byte) {
  const int t = 127 - byte;
  auto in = [&](float v) {
    return __builtin_amdgcn_ldexpf((__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? __uint_as_float(0x7FC00000u) : v, t);
  };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), r, true));
}

// The same for values without infinities, in two instructions: the conversion divides by a
// power of two itself.
__device__ __forceinline__ uint32_t pack_finite_e4m3x4(float a, float b, float c, float d, int byte) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  const float s = __uint_as_float(uint32_t(byte) << 23);
  i16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(i16x2{0, 0}, a, b, s, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, c, d, s, true));
}

// Largest of the 16 lanes of a DPP row, in all of them.
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xF, 0xF, false)));   // row_ror:8
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xF, 0xF, false)));
  v = max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xF, 0xF, false)));
  return max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xF, 0xF, false)));
}

// ... of 32 lanes.
__device__ __forceinline__ uint32_t half_max(uint32_t v) {
  v = row16_max(v);
  return max(v, uint32_t(__shfl_xor(int(v), 16)));
}

}  // namespace epic

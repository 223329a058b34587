// Device helpers of the 8-bit GEMM kernels.
#pragma once

#include "device_common.h"
#include "gemm_device.h"

namespace epic {

typedef int i32x8 __attribute__((ext_vector_type(8)));         // MFMA operand: 32 e4m3 values of a lane

// acc += (a * 2^(byte a_sel of sa - 127)) (b * 2^(byte 0 of sb - 127)), 32 x 32 x 64: lane l has
// 32 of the 64 values of row l % 32 of either operand, and that row's scale; column l % 32
// of the result belongs to b.  Which values of K a lane has does not matter as long as
// both operands agree.
template <int SEL_A, int SEL_B>
__device__ __forceinline__ f32x16 mfma8(const i32x8& a, const i32x8& b, const f32x16& c, int sa, int sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 0, 0, SEL_A, sa, SEL_B, sb);
}

// 32 bytes of an operand row from two 16-byte chunks in LDS.
__device__ __forceinline__ i32x8 read32(const char* p, int c0, int c1) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 lo = *reinterpret_cast<const i32x4*>(p + c0), hi = *reinterpret_cast<const i32x4*>(p + c1);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

}  // namespace epic

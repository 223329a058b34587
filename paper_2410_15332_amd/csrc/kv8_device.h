// Device helpers of the 8-bit cache: one wavefront holds the K and V of a (block, KV head).
//
// Lane l = r + 16 a (r < 16, a < 4) holds, for each 64 dims j, 16 bytes of K (token r, dims
// 64 j + 16 a ..) and 16 bytes of V (dims 64 j + 16 t + r of tokens 4 a ..): four dwords t of
// four tokens.  Both are byte 1024 j + 16 l of the slab, so loads are 1 KB runs, and both
// are matrix operands as they are: K's bytes are two k-steps of A for 16 tokens, V's dword t
// is A (transposed V) for dims 16 t .. of the tokens whose probabilities the lane holds.
#pragma once

#include "kv8.h"
#include "quant_device.h"

namespace epic {

typedef __bf16 bf16x2r __attribute__((ext_vector_type(2)));

// Two e4m3 of a dword (its low or high half) as a packed bf16 pair, times a power of two: exact.
template <bool HI>
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(int(w), scale, HI));
}

// Loads and stores of bytes that nothing reads again soon.
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ uint4 load16(const void* p) { return __builtin_bit_cast(uint4, __builtin_nontemporal_load(static_cast<const u32x4*>(p))); }
__device__ __forceinline__ uint2 load8(const void* p) { return __builtin_bit_cast(uint2, __builtin_nontemporal_load(static_cast<const u32x2*>(p))); }
__device__ __forceinline__ void store16(void* p, const uint4& x) { __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), static_cast<u32x4*>(p)); }

// |bits| of the pairs of a dword, and the larger of two such dwords, half by half.
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pair_abs(uint32_t w) { return w & 0x7FFF7FFFu; }
__device__ __forceinline__ uint32_t pair_max(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}
// Largest of the 16 lanes of a DPP row, half by half, in all of them.
__device__ __forceinline__ uint32_t row16_pair_max(uint32_t v) {
  v = pair_max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x128, 0xF, 0xF, false)));   // row_ror:8
  v = pair_max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x124, 0xF, 0xF, false)));
  v = pair_max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x122, 0xF, 0xF, false)));
  return pair_max(v, uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x121, 0xF, 0xF, false)));
}

// Scale byte of a row from the largest |bits| of its bf16 values: that of the 8-bit operands, or NaN.
__device__ __forceinline__ int kv8_byte(uint32_t top16) {
  return top16 >= 0x7F80u ? kKv8Nan : scale_byte(top16 << 16);
}

// Two bf16 pairs over 2^(byte - 127) as four e4m3, for finite values.
__device__ __forceinline__ uint32_t round4(uint32_t lo, uint32_t hi, int byte) {
  return pack_e4m3x4(__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u), __uint_as_float(hi << 16),
                     __uint_as_float(hi & 0xFFFF0000u), byte);
}

// Rows in the K arrangement: x[2 j], x[2 j + 1] are the 16 bf16 of dims 64 j + 16 a .. of token r.
template <int J>
__device__ __forceinline__ uint32_t row_top(const uint4 (&x)[2 * J]) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < 2 * J; ++i)
    m = pair_max(m, pair_max(pair_max(pair_abs(x[i].x), pair_abs(x[i].y)), pair_max(pair_abs(x[i].z), pair_abs(x[i].w))));
  m = pair_max(m, uint32_t(__shfl_xor(int(m), 16)));
  m = pair_max(m, uint32_t(__shfl_xor(int(m), 32)));
  return max(m & 0xFFFFu, m >> 16);
}
__device__ __forceinline__ uint4 round16(const uint4& p, const uint4& q, int byte) {
  return make_uint4(round4(p.x, p.y, byte), round4(p.z, p.w, byte), round4(q.x, q.y, byte), round4(q.z, q.w, byte));
}
constexpr uint32_t kNanBytes = 0x7F7F7F7Fu;   // K of a NaN token: its scores are NaN, whatever its scale

}  // namespace epic

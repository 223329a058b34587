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
__device__ __forceinline__ uint4 load16(const void* p) {
  return __builtin_bit_cast(uint4, __builtin_nontemporal_load(static_cast<const u32x4*>(p)));
}
__device__ __forceinline__ uint2 load8(const void* p) {
  return __builtin_bit_cast(uint2, __builtin_nontemporal_load(static_cast<const u32x2*>(p)));
}
__device__ __forceinline__ void store16(void* p, const uint4& x) {
  __builtin_nontemporal_store(__builtin_bit_cast(u32x4, x), static_cast<u32x4*>(p));
}

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

// Two bf16 pairs over 2^(byte - 127) as four e4m3, for finite values: the conversion divides by a power of two itself.
__device__ __forceinline__ uint32_t round4(uint32_t lo, uint32_t hi, int byte) {
  typedef short i16x2 __attribute__((ext_vector_type(2)));
  const float s = __uint_as_float(uint32_t(byte) << 23);
  const i16x2 r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(i16x2{0, 0}, __builtin_bit_cast(bf16x2r, lo), s, false);
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2r, hi), s, true));
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

// The rows of S that a block receives, rounded, as its wavefront holds a block; zero rows elsewhere.
template <int J>
struct Kv8Fresh {
  uint4 k[J], v[J];
  int kb;                                     // scale byte of K of token r
  uint32_t ks, vs;                            // scale bytes of K and V of tokens 4 a ..
  uint32_t tokens;                            // bit s: token s is a row of S
};

constexpr int kTurnLd = 68;                   // bytes of a token's 64 dims in LDS
template <int J>
constexpr int kTurnInts = J * 16 * kTurnLd / 4;

// row: of token r, or -1.  V rows come like K's, 16 dims of a token a lane; their e4m3 bytes change places
// through `turn`, LDS of this wavefront alone.
template <int D>
__device__ __forceinline__ Kv8Fresh<D / 64> kv8_fresh(int row, const uint16_t* k_s, const uint16_t* v_s, int hkv, int g,
                                                      int lane, uint32_t* turn) {
  constexpr int J = D / 64;
  const int r = lane & 15, a = lane >> 4;
  Kv8Fresh<J> f;
  f.tokens = uint32_t(__ballot(row >= 0)) & 0xFFFFu;
  uint4 x[2 * J], y[2 * J];
#pragma unroll
  for (int i = 0; i < 2 * J; ++i) x[i] = y[i] = make_uint4(0, 0, 0, 0);
  if (f.tokens != 0) {
    const size_t from = (size_t(max(row, 0)) * hkv + g) * D + 16 * a;
#pragma unroll
    for (int i = 0; i < 2 * J; ++i) {
      x[i] = *reinterpret_cast<const uint4*>(k_s + from + 64 * (i >> 1) + 8 * (i & 1));
      y[i] = *reinterpret_cast<const uint4*>(v_s + from + 64 * (i >> 1) + 8 * (i & 1));
    }
    const uint32_t keep = row >= 0 ? 0xFFFFFFFFu : 0u;
#pragma unroll
    for (int i = 0; i < 2 * J; ++i) {
      x[i] = make_uint4(x[i].x & keep, x[i].y & keep, x[i].z & keep, x[i].w & keep);
      y[i] = make_uint4(y[i].x & keep, y[i].y & keep, y[i].z & keep, y[i].w & keep);
    }
  }
  int kb = kv8_byte(row_top<J>(x)), vb = kv8_byte(row_top<J>(y));
  if (kb == kKv8Nan || vb == kKv8Nan) kb = vb = kKv8Nan;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    f.k[j] = round16(x[2 * j], x[2 * j + 1], kb);
    uint4 q = round16(y[2 * j], y[2 * j + 1], vb);
    if (kb == kKv8Nan) {
      f.k[j] = make_uint4(kNanBytes, kNanBytes, kNanBytes, kNanBytes);
      q = make_uint4(0, 0, 0, 0);
    }
    uint32_t* to = turn + (j * 16 * kTurnLd + r * kTurnLd + 16 * a) / 4;
    to[0] = q.x, to[1] = q.y, to[2] = q.z, to[3] = q.w;
  }
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();            // one wavefront: its LDS accesses run in order
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  f.kb = kb;
  f.ks = f.vs = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f.ks |= uint32_t(__shfl(kb, 4 * a + i)) << (8 * i);
    f.vs |= uint32_t(__shfl(vb, 4 * a + i)) << (8 * i);
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const uint8_t* from = reinterpret_cast<const uint8_t*>(turn) + j * 16 * kTurnLd;
    uint32_t w[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      w[t] = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) w[t] |= uint32_t(from[(4 * a + i) * kTurnLd + 16 * t + r]) << (8 * i);
    }
    f.v[j] = make_uint4(w[0], w[1], w[2], w[3]);
  }
  return f;
}

// Bytes i of a dword, for the bits i of the four.
__device__ __forceinline__ uint32_t byte_mask(uint32_t four) { return (four * 0x00204081u & 0x01010101u) * 255u; }

__device__ __forceinline__ uint4 merge(const uint4& old, const uint4& x, uint32_t mask) {
  return make_uint4((old.x & ~mask) | (x.x & mask), (old.y & ~mask) | (x.y & mask), (old.z & ~mask) | (x.z & mask),
                    (old.w & ~mask) | (x.w & mask));
}

// The bytes of the rows of S into their block, and no others: what the block holds beside them may be read meanwhile.
template <int D>
__device__ __forceinline__ void kv8_store_fresh(const Kv8Fresh<D / 64>& f, const epic_kv8_cache& c, size_t block_head,
                                                int lane) {
  constexpr int J = D / 64;
  const int r = lane & 15, a = lane >> 4;
  const size_t to = block_head * 16 * D;
  uint8_t* s = c.scale + block_head * kKv8Scales;
  if (f.tokens >> r & 1) {
#pragma unroll
    for (int j = 0; j < J; ++j) *reinterpret_cast<uint4*>(c.k + to + 1024 * j + 16 * lane) = f.k[j];
    if (a == 0) s[r] = uint8_t(f.kb);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (!(f.tokens >> (4 * a + i) & 1)) continue;
    uint8_t* v = c.v + to + 16 * lane + i;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      v[1024 * j] = uint8_t(f.v[j].x >> (8 * i));
      v[1024 * j + 4] = uint8_t(f.v[j].y >> (8 * i));
      v[1024 * j + 8] = uint8_t(f.v[j].z >> (8 * i));
      v[1024 * j + 12] = uint8_t(f.v[j].w >> (8 * i));
    }
    if (r == 0) s[16 + 4 * a + i] = uint8_t(f.vs >> (8 * i));
  }
}

// The rows of S over what their block's source holds (kb: of token r, vs: of tokens 4 a ..).
template <int D>
__device__ __forceinline__ void kv8_merge(const Kv8Fresh<D / 64>& f, uint4 (&kq)[D / 64], uint4 (&vq)[D / 64], int& kb,
                                          uint32_t& vs, int lane) {
  const bool fresh = f.tokens >> (lane & 15) & 1;
  const uint32_t mask = byte_mask(f.tokens >> (4 * (lane >> 4)) & 15u);
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    kq[j] = fresh ? f.k[j] : kq[j];
    vq[j] = merge(vq[j], f.v[j], mask);
  }
  kb = fresh ? f.kb : kb;
  vs = (vs & ~mask) | (f.vs & mask);
}

// A whole block.
template <int D>
__device__ __forceinline__ void kv8_store_block(const uint4 (&kq)[D / 64], const uint4 (&vq)[D / 64], int kb, uint32_t vs,
                                                const epic_kv8_cache& c, size_t block_head, int lane) {
  const size_t to = block_head * 16 * D;
  uint8_t* s = c.scale + block_head * kKv8Scales;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    *reinterpret_cast<uint4*>(c.k + to + 1024 * j + 16 * lane) = kq[j];
    *reinterpret_cast<uint4*>(c.v + to + 1024 * j + 16 * lane) = vq[j];
  }
  if (lane < 16) s[lane] = uint8_t(kb);
  if ((lane & 15) == 0) *reinterpret_cast<uint32_t*>(s + 16 + 4 * (lane >> 4)) = vs;
}

// What a wavefront reads of a block.
template <int D>
__device__ __forceinline__ void kv8_load_block(const epic_kv8_cache& c, size_t block_head, int lane, uint4 (&kq)[D / 64],
                                               uint4 (&vq)[D / 64], int& kb, uint32_t& vs) {
  const uint8_t* s = c.scale + block_head * kKv8Scales;
  kb = s[lane & 15];
  vs = *reinterpret_cast<const uint32_t*>(s + 16 + 4 * (lane >> 4));
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    kq[j] = *reinterpret_cast<const uint4*>(c.k + block_head * 16 * D + 1024 * j + 16 * lane);
    vq[j] = *reinterpret_cast<const uint4*>(c.v + block_head * 16 * D + 1024 * j + 16 * lane);
  }
}

// Rows of zeros.
template <int D>
__device__ __forceinline__ void kv8_no_block(uint4 (&kq)[D / 64], uint4 (&vq)[D / 64], int& kb, uint32_t& vs) {
  kb = 127;
  vs = 0x7F7F7F7Fu;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) kq[j] = vq[j] = make_uint4(0, 0, 0, 0);
}

// The link write of one (private block i, KV head) by one wavefront: what its source block holds, zero rows without
// one, then its rows of S.  A block that is its own source only receives its rows.
template <int D>
__device__ __forceinline__ void kv8_write_private(const Kv8Rows& w, const epic_kv8_cache& c, int i, int hkv, int g, int lane,
                                                  uint32_t* turn) {
  const int dst = w.block[i], src = w.src[i], row = w.rows[i * 16 + (lane & 15)];
  const size_t to = size_t(dst) * hkv + g;
  if (src == dst) {
    kv8_store_fresh<D>(kv8_fresh<D>(row, w.k_s, w.v_s, hkv, g, lane, turn), c, to, lane);
    return;
  }
  uint4 kq[D / 64], vq[D / 64];
  int kb;
  uint32_t vs;
  kv8_load_block<D>(c, size_t(max(src, 0)) * hkv + g, lane, kq, vq, kb, vs);
  const Kv8Fresh<D / 64> f = kv8_fresh<D>(row, w.k_s, w.v_s, hkv, g, lane, turn);
  if (src < 0) kv8_no_block<D>(kq, vq, kb, vs);            // (here: before, it would wait for the loads)
  kv8_merge<D>(f, kq, vq, kb, vs, lane);
  kv8_store_block<D>(kq, vq, kb, vs, c, to, lane);
}

}  // namespace epic

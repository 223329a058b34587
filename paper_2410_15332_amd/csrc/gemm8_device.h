// Device helpers of the 8-bit GEMM kernels.
#pragma once

#include "device_common.h"
#include "gemm8.h"
#include "gemm_device.h"
#include "quant_device.h"

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

__device__ __forceinline__ float silu(float x) { return x * __builtin_amdgcn_rcpf(1.0f + fast_exp2(-x * kLog2e)); }

// 32 bytes of an operand row from two 16-byte chunks in LDS.
__device__ __forceinline__ i32x8 read32(const char* p, int c0, int c1) {
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 lo = *reinterpret_cast<const i32x4*>(p + c0), hi = *reinterpret_cast<const i32x4*>(p + c1);
  return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A quantised result's scale jumps where its group's largest |y| crosses 1.75 * 2^e, and the
// matrix cores leave y about 5e-5 off (gemm8.h): one group in 17000 would get the
// neighbouring scale, and another one by another route.  So where the largest, with bits
// top, is within 2^-12 of a border (one group in 1400), that one result is computed again in
// 64 bits, by all wavefronts of the workgroup, and decides.  Of 1.5 million groups none then
// differs from float64's (87 before).  This is no guarantee: sums whose large products cancel
// are farther off than the window is wide, and a result that is not the largest before it is
// computed again, but would be after, is not looked at.  A result costs some
// 4 us where it holds up its workgroup, with and without: 20560 x 28672 x 4096 1884 us and 1803, 100 rows 32.7
// and 32.1, 32 rows 30.9 and 30.1; 736 rows 96-101 and 93-96.  In one tile some 1 us each: 736 times the
// same row, next to a border, 272 where others take 89.
__device__ __forceinline__ bool near_border(uint32_t top) {
  return abs(int(top & 0x7FFFFFu) - 0x600000) <= 3584;   // 1.75 * 2^23 * 2^-12
}

// Results to compute again, at most MOST, in LDS.
template <int NW, int MOST>
struct Border {
  int count;
  int at[MOST][2];                                      // row, column
  double part[MOST][NW][2];                             // gate and up: sums of a wavefront's share of K

  __device__ __forceinline__ int add(int m, int c) {
    const int h = atomicAdd(&count, 1);
    at[h][0] = m;
    at[h][1] = c;
    return h;
  }

  // After a barrier: the sums, 1 KB of K after another dealt to the wavefronts.  Products of
  // two e4m3 values are exact in 32 bits.
  __device__ __forceinline__ void compute(const Gemm8Args& g, int n, int wv, int lane) {
    const int ffn = g.N >> 1, ks = g.K >> 7, ld = (g.M + 3) & ~3;
#pragma unroll 1
    for (int h = 0; h < n; ++h) {
      const int m = __builtin_amdgcn_readfirstlane(at[h][0]), c = __builtin_amdgcn_readfirstlane(at[h][1]);
      const uint8_t *pa = g.A + size_t(m) * g.K, *pg = g.W + size_t(c) * g.K, *pu = g.W + size_t(ffn + c) * g.K;
      double x = 0.0, y = 0.0;
      for (int k = wv * 1024 + lane * 16; k < g.K; k += NW * 1024) {
        const uint4 va = *reinterpret_cast<const uint4*>(pa + k), vg = *reinterpret_cast<const uint4*>(pg + k),
                    vu = *reinterpret_cast<const uint4*>(pu + k);
        const int t = int(g.sa[size_t(k >> 7) * ld + m]) - 254;
        const int tg = g.sw[(c >> 7) * ks + (k >> 7)], tu = g.sw[((ffn + c) >> 7) * ks + (k >> 7)];
        const uint32_t a[4] = {va.x, va.y, va.z, va.w}, b[4] = {vg.x, vg.y, vg.z, vg.w}, d[4] = {vu.x, vu.y, vu.z, vu.w};
        double sg = 0.0, su = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const auto a0 = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8(a[i], true);
          const auto b0 = __builtin_amdgcn_cvt_pk_f32_fp8(b[i], false), b1 = __builtin_amdgcn_cvt_pk_f32_fp8(b[i], true);
          const auto d0 = __builtin_amdgcn_cvt_pk_f32_fp8(d[i], false), d1 = __builtin_amdgcn_cvt_pk_f32_fp8(d[i], true);
          sg += double(a0[0] * b0[0]) + double(a0[1] * b0[1]) + double(a1[0] * b1[0]) + double(a1[1] * b1[1]);
          su += double(a0[0] * d0[0]) + double(a0[1] * d0[1]) + double(a1[0] * d1[0]) + double(a1[1] * d1[1]);
        }
        x += ldexp(sg, t + tg);
        y += ldexp(su, t + tu);
      }
#pragma unroll
      for (int i = 1; i < 64; i *= 2) {
        x += __shfl_xor(x, i);
        y += __shfl_xor(y, i);
      }
      if (lane == 0) part[h][wv][0] = x, part[h][wv][1] = y;
    }
  }

  // After another barrier: the scale's byte of the group whose largest, result h, has bits top.
  __device__ __forceinline__ int byte(int h, uint32_t top) const {
    double x = 0.0, y = 0.0;
#pragma unroll
    for (int i = 0; i < NW; ++i) x += part[h][i][0], y += part[h][i][1];
    const float border = __uint_as_float((top & 0x7F800000u) | 0x600000u);
    return max(int(top >> 23) - 8 + (fabs(x / (1.0 + exp(-x)) * y) > double(border) ? 1 : 0), 0);
  }
};

// The scale's byte of a group of row m in 32 lanes, four results (from column n on) each, the
// largest with bits top.  Called by the whole workgroup; live: the row is one of the result's.
// The list's count is 0, and everyone's to see.
template <int NW, int MOST>
__device__ __forceinline__ int group_byte(Border<NW, MOST>& list, const Gemm8Args& g, uint32_t top, const float4& v, int m, int n,
                                          bool live) {
  const int lane = threadIdx.x & 63;
  const bool near = live && near_border(top);
  int h = -1;
  if (__any(near)) {                                    // the first of the half's lanes that has it
    const int e = finite_abs(v.x) == top ? 0 : finite_abs(v.y) == top ? 1 : finite_abs(v.z) == top ? 2 : 3;
    const bool has = finite_abs(v.x) == top || finite_abs(v.y) == top || finite_abs(v.z) == top || finite_abs(v.w) == top;
    const uint32_t lanes = uint32_t(__ballot(near && has) >> (lane & 32));
    const int first = (lane & 32) + __ffs(lanes) - 1;
    if (near && lane == first) h = list.add(m, n + e);
    h = __shfl(h, near ? first : lane);
  }
  barrier_lds();
  const int count = list.count;
  if (count > 0) {
    list.compute(g, count, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane);
    barrier_lds();
    if (near) return list.byte(h, top);
  }
  return scale_byte(top);
}

}  // namespace epic

// Rounding rows, weights and the residual stream's norm to e4m3 with e8m0 scales.
//
// For a group of 128 values y: t = the smallest integer with max |y| <= 448 * 2^t, and
// q = e4m3(y / 2^t), rounded once, to nearest even.  e4m3 has an exponent of its own, so
// a power of two costs no relative precision against max |y| / 448 (at most one of the
// lowest binades), the division is exact, and the matrix cores apply such scales
// themselves.  All three kernels read their input once and are bound by that.
#include <type_traits>

#include "quant.h"
#include "quant_device.h"

namespace epic {

namespace {

constexpr int kThreads = 256;

// Eight bf16 of a lane as floats.
__device__ __forceinline__ void widen(const uint4& p, float v[8]) {
  const uint32_t w[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ uint32_t top_of(const uint4& p) {
  float v[8];
  widen(p, v);
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, finite_abs(v[i]));
  return top;
}

__device__ __forceinline__ uint2 round8(const uint4& p, int byte) {
  float v[8];
  widen(p, v);
  return make_uint2(pack_e4m3x4(v[0], v[1], v[2], v[3], byte), pack_e4m3x4(v[4], v[5], v[6], v[7], byte));
}

// Rows as one run of m * k values: a thread takes a piece of 8 (16 lanes a group), so loads
// and stores are contiguous whatever k is.  20 560 x 4096: 49 us (253 MB, 5.1 TB/s: a copy
// on this card reaches 4.9); 32 x 4096: 3.1.  Four pieces per thread: 50 and 3.8.
__global__ __launch_bounds__(kThreads) void quant_rows_kernel(const uint4* __restrict__ x, uint2* __restrict__ q,
                                                              uint8_t* __restrict__ scale, int64_t pieces, int groups,
                                                              int ld) {
  const int64_t p = int64_t(blockIdx.x) * kThreads + threadIdx.x;
  const uint4 v = x[min(p, pieces - 1)];
  const int byte = scale_byte(row16_max(top_of(v)));
  if (p >= pieces) return;
  q[p] = round8(v, byte);
  if ((threadIdx.x & 15) == 0) {
    const uint32_t g = uint32_t(p >> 4), row = g / uint32_t(groups);
    scale[size_t(g - row * groups) * ld + row] = uint8_t(byte);
  }
}

// A 128 x 128 block per workgroup, 16 rows a step, kept in registers between the maximum
// and the rounding.  28 672 x 4096: 64 us (352 MB, 5.5 TB/s).
__global__ __launch_bounds__(kThreads) void quant_blocks_kernel(const uint16_t* __restrict__ x, uint8_t* __restrict__ q,
                                                                uint8_t* __restrict__ scale, int m, int k) {
  __shared__ uint32_t red[kThreads / 64];
  constexpr int STEPS = 8;
  const int row0 = blockIdx.y * kGroup + (threadIdx.x >> 4), col = blockIdx.x * kGroup + (threadIdx.x & 15) * 8;
  uint4 v[STEPS];
  uint32_t top = 0;
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
    v[s] = *reinterpret_cast<const uint4*>(x + size_t(min(row0 + s * 16, m - 1)) * k + col);
#pragma unroll
  for (int s = 0; s < STEPS; ++s) top = max(top, top_of(v[s]));   // rows past m repeat row m - 1, of this block too
  top = half_max(top);
  top = max(top, uint32_t(__shfl_xor(int(top), 32)));
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kThreads / 64; ++i) top = max(top, red[i]);
  const int byte = scale_byte(top);
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
    if (row0 + s * 16 < m) *reinterpret_cast<uint2*>(q + size_t(row0 + s * 16) * k + col) = round8(v[s], byte);
  if (threadIdx.x == 0) scale[size_t(blockIdx.y) * gridDim.x + blockIdx.x] = uint8_t(byte);
}

enum Addend { kNone, kDelta, kPlanes };

// One workgroup per row, the row in registers (KEEP float4 per thread) between the sum of
// squares and the rounding; 32 lanes hold a group.  512 threads: enough loads in flight for a
// single row, enough rows on a CU for many (us with 256 / 512 / 1024; 4096 wide with delta):
// 1 row 4.2 / 3.7 / 3.7, 736 rows 8.4 / 8.0 / 8.9, 20 560 rows 159 / 155 / 161 (927 MB, 6.0
// TB/s); 8192 wide, 20 560 rows 323 / 320 / 318.
template <int ADD, int KEEP>
__global__ __launch_bounds__(1024) void rmsnorm_fp8_kernel(const float* x, const uint16_t* __restrict__ delta, StreamSum s,
                                                           const uint16_t* __restrict__ w, int hidden, float eps,
                                                           float* x_out, uint8_t* __restrict__ q,
                                                           uint8_t* __restrict__ scale, int ld) {
  __shared__ float red[16];
  const int row = blockIdx.x, n4 = hidden / 4, T = blockDim.x;
  const float4* xr = reinterpret_cast<const float4*>(x + size_t(row) * hidden);
  float4 v[KEEP];
  uint2 wv[KEEP], dv[KEEP];
#pragma unroll
  for (int j = 0; j < KEEP; ++j) {
    const int i = min(int(threadIdx.x) + j * T, n4 - 1);
    v[j] = xr[i];
    if constexpr (ADD == kDelta) dv[j] = *reinterpret_cast<const uint2*>(delta + size_t(row) * hidden + 4 * i);
    wv[j] = *reinterpret_cast<const uint2*>(w + 4 * i);
  }
  if constexpr (ADD != kNone) {
#pragma unroll
    for (int j = 0; j < KEEP; ++j) {
      float4 a;
      if constexpr (ADD == kDelta)
        a = make_float4(__uint_as_float(dv[j].x << 16), __uint_as_float(dv[j].x & 0xFFFF0000u),
                        __uint_as_float(dv[j].y << 16), __uint_as_float(dv[j].y & 0xFFFF0000u));
      else
        a = s.sum4(row, 4 * min(int(threadIdx.x) + j * T, n4 - 1));
      v[j] = make_float4(v[j].x + a.x, v[j].y + a.y, v[j].z + a.z, v[j].w + a.w);
    }
  }
  float ss = 0.0f;
#pragma unroll
  for (int j = 0; j < KEEP; ++j) {
    const int i = threadIdx.x + j * T;
    const float sq = v[j].x * v[j].x + v[j].y * v[j].y + v[j].z * v[j].z + v[j].w * v[j].w;
    ss += i < n4 ? sq : 0.0f;
    if (x_out != nullptr && i < n4) reinterpret_cast<float4*>(x_out + size_t(row) * hidden)[i] = v[j];
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = ss;
  __syncthreads();
  float total = 0.0f;
  for (int i = 0; i < T / 64; ++i) total += red[i];
  const float inv = 1.0f / sqrtf(total / float(hidden) + eps);
#pragma unroll
  for (int j = 0; j < KEEP; ++j) {
    const int i = threadIdx.x + j * T;
    const float y0 = v[j].x * inv * bf16_to_f32(uint16_t(wv[j].x & 0xFFFFu));
    const float y1 = v[j].y * inv * bf16_to_f32(uint16_t(wv[j].x >> 16));
    const float y2 = v[j].z * inv * bf16_to_f32(uint16_t(wv[j].y & 0xFFFFu));
    const float y3 = v[j].w * inv * bf16_to_f32(uint16_t(wv[j].y >> 16));
    const uint32_t top = half_max(max(max(finite_abs(y0), finite_abs(y1)), max(finite_abs(y2), finite_abs(y3))));
    const int byte = scale_byte(top);
    if (i < n4) {                                       // a whole half wavefront or none: hidden % 128 == 0
      *reinterpret_cast<uint32_t*>(q + size_t(row) * hidden + 4 * i) = pack_e4m3x4(y0, y1, y2, y3, byte);
      if ((threadIdx.x & 31) == 0) scale[size_t(i >> 5) * ld + row] = uint8_t(byte);
    }
  }
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

}  // namespace

void launch_quant_rows(const uint16_t* x, int m, int k, uint8_t* q, uint8_t* scale, hipStream_t stream) {
  const int64_t pieces = int64_t(m) * k / 8;
  quant_rows_kernel<<<unsigned((pieces + kThreads - 1) / kThreads), kThreads, 0, stream>>>(
      reinterpret_cast<const uint4*>(x), reinterpret_cast<uint2*>(q), scale, pieces, k / kGroup, scale_ld(m));
}

void launch_quant_blocks(const uint16_t* x, int m, int k, uint8_t* q, uint8_t* scale, hipStream_t stream) {
  quant_blocks_kernel<<<dim3(k / kGroup, cdiv(m, kGroup)), kThreads, 0, stream>>>(x, q, scale, m, k);
}

void launch_rmsnorm_fp8(const float* x, const uint16_t* delta, const StreamSum& s, const uint16_t* w, int m, int hidden,
                        float eps, float* x_out, uint8_t* q, uint8_t* scale, hipStream_t stream) {
  const int n4 = hidden / 4;
  const int T = norm_threads(hidden);
  const int keep = cdiv(n4, T);
  const int ld = scale_ld(m);
  auto go = [&](auto kernel) { kernel<<<m, T, 0, stream>>>(x, delta, s, w, hidden, eps, x_out, q, scale, ld); };
  auto by_length = [&](auto add) {
    constexpr int ADD = decltype(add)::value;
    if (keep <= 1) go(rmsnorm_fp8_kernel<ADD, 1>);
    else if (keep <= 2) go(rmsnorm_fp8_kernel<ADD, 2>);
    else if (keep <= 4) go(rmsnorm_fp8_kernel<ADD, 4>);
    else go(rmsnorm_fp8_kernel<ADD, 8>);
  };
  if (s.partial != nullptr) by_length(std::integral_constant<int, kPlanes>{});
  else if (delta != nullptr) by_length(std::integral_constant<int, kDelta>{});
  else by_length(std::integral_constant<int, kNone>{});
}

}  // namespace epic

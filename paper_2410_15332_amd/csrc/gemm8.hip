// How 8-bit products are divided, and the pass that finishes those left in planes.
#include <algorithm>

#include "gemm8.h"
#include "quant.h"
#include "quant_device.h"

namespace epic {

namespace {

constexpr int kWorkers = 256;                           // one workgroup per CU

__device__ __forceinline__ float silu(float x) { return x * __builtin_amdgcn_rcpf(1.0f + fast_exp2(-x * kLog2e)); }

// Summed planes in bf16, or through SwiGLU (GLU): four columns per thread.
template <bool GLU>
__global__ __launch_bounds__(256) void finish_kernel(StreamSum s, uint16_t* __restrict__ out, int cols) {
  const int n4 = cols / 4;
  const int idx = blockIdx.x * 256 + threadIdx.x;
  const int m = idx / n4, n = (idx - m * n4) * 4;
  if (m >= s.M) return;
  float4 v = s.sum4(m, n);
  if constexpr (GLU) {
    const float4 u = s.sum4(m, cols + n);
    v = make_float4(silu(v.x) * u.x, silu(v.y) * u.y, silu(v.z) * u.z, silu(v.w) * u.w);
  }
  *reinterpret_cast<uint2*>(out + size_t(m) * cols + n) = make_uint2(pack_bf16x2(v.x, v.y), pack_bf16x2(v.z, v.w));
}

// SwiGLU of summed planes, quantised: four columns per thread, 32 lanes a group.
__global__ __launch_bounds__(256) void finish_quant_kernel(StreamSum s, uint8_t* __restrict__ out,
                                                           uint8_t* __restrict__ scale, int ffn, int ld) {
  const int n4 = ffn / 4;
  const int idx = blockIdx.x * 256 + threadIdx.x;
  const int m = idx / n4, n = (idx - m * n4) * 4;
  if (m >= s.M) return;                                 // whole half wavefronts: ffn % 128 == 0
  const float4 g = s.sum4(m, n), u = s.sum4(m, ffn + n);
  const float a = silu(g.x) * u.x, b = silu(g.y) * u.y, c = silu(g.z) * u.z, d = silu(g.w) * u.w;
  const int byte = scale_byte(half_max(max(max(finite_abs(a), finite_abs(b)), max(finite_abs(c), finite_abs(d)))));
  *reinterpret_cast<uint32_t*>(out + size_t(m) * ffn + n) = pack_e4m3x4(a, b, c, d, byte);
  if ((threadIdx.x & 31) == 0) scale[size_t(n >> 7) * ld + m] = uint8_t(byte);
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

}  // namespace

// Up to 128 rows: streamed.  Past that the cheaper of whole tiles and equal parts of K, by
// the time of the stages that the busiest CU runs and of what the planes move.
Gemm8Plan gemm8_plan(int M, int N, int K, int epi) {
  if (M <= 128 && gemm8_stream_fits(M, N, K)) return Gemm8Plan{true, 0, 0};
  const int ks = K / kGroup;
  Gemm8Plan best{};
  double best_time = 0.0;
  for (const int tm : {256, 128}) {
    const int64_t tiles = int64_t(cdiv(M, tm)) * cdiv(N, 256);
    const double stage = tm == 256 ? 1.1 : 0.75;
    for (int parts = 1; parts <= 32 && parts <= ks; ++parts) {
      if (parts > 1 && (tiles * parts > kWorkers || int64_t(parts) * M * N * 4 > int64_t(kPartial8Bytes) || ks / parts < 4))
        break;
      const double rounds = double((tiles * parts + kWorkers - 1) / kWorkers);
      double time = 6.0 + rounds * (cdiv(ks, parts) * stage + (tm == 256 ? 3.0 : 1.5));
      if (parts > 1) time += 4.0 + double(parts) * M * N * 8 * 0.25e-6;
      if (best.tm == 0 || time < best_time) best = Gemm8Plan{false, tm, parts == 1 ? 0 : parts}, best_time = time;
    }
  }
  return best;
}

StreamSum launch_gemm8_partial(const Gemm8Args& g, const Gemm8Plan& p, hipStream_t stream) {
  return p.stream ? launch_gemm8_stream(g, stream) : launch_gemm8_split(g, p.tm, std::max(p.parts, 1), stream);
}

void launch_gemm8_finish(const StreamSum& s, const Gemm8Args& g, int epi, hipStream_t stream) {
  const int cols = epi == kBf16Out ? g.N : g.N / 2;
  const int grid = cdiv(g.M * (cols / 4), 256);
  uint16_t* out = static_cast<uint16_t*>(g.out);
  if (epi == kBf16Out) finish_kernel<false><<<grid, 256, 0, stream>>>(s, out, cols);
  else if (epi == kGluOut) finish_kernel<true><<<grid, 256, 0, stream>>>(s, out, cols);
  else finish_quant_kernel<<<grid, 256, 0, stream>>>(s, static_cast<uint8_t*>(g.out), g.out_scale, cols, scale_ld(g.M));
}

void launch_gemm8(const Gemm8Args& g, int epi, hipStream_t stream) {
  const Gemm8Plan p = gemm8_plan(g.M, g.N, g.K, epi);
  if (p.stream || p.parts > 1) launch_gemm8_finish(launch_gemm8_partial(g, p, stream), g, epi, stream);
  else launch_gemm8_wide(g, epi, p.tm, stream);
}

}  // namespace epic

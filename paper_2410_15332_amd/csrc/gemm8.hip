// How 8-bit products are divided, and the pass that finishes those left in planes.
#include <algorithm>
#include <cmath>

#include "gemm8.h"
#include "gemm8_device.h"
#include "quant.h"
#include "quant_device.h"

namespace epic {

namespace {

constexpr int kWorkers = 256;                           // one workgroup per CU

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
__global__ __launch_bounds__(256) void finish_quant_kernel(StreamSum s, Gemm8Args args) {
  __shared__ Border<4, 8> list;
  if (threadIdx.x == 0) list.count = 0;
  barrier_lds();
  const int ffn = args.N / 2, ld = (args.M + 3) & ~3;
  const int n4 = ffn / 4;
  const int idx = blockIdx.x * 256 + threadIdx.x;
  const int m = idx / n4, n = (idx - m * n4) * 4;
  const bool live = m < s.M;                            // the same in a half wavefront: ffn % 128 == 0
  float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (live) {
    const float4 g = s.sum4(m, n), u = s.sum4(m, ffn + n);
    v = make_float4(silu(g.x) * u.x, silu(g.y) * u.y, silu(g.z) * u.z, silu(g.w) * u.w);
  }
  const uint32_t top = half_max(max(max(finite_abs(v.x), finite_abs(v.y)), max(finite_abs(v.z), finite_abs(v.w))));
  const int byte = group_byte(list, args, top, v, m, n, live);
  if (!live) return;
  *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(args.out) + size_t(m) * ffn + n) = pack_e4m3x4(v.x, v.y, v.z, v.w, byte);
  if ((threadIdx.x & 31) == 0) args.out_scale[size_t(n >> 7) * ld + m] = uint8_t(byte);
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

// Estimates in us, fitted to kernels replayed in a graph, that gemm8_plan chooses by.

// What reading the operands from memory takes at best.
double read_time(int M, int N, int K) { return (double(N) * K + double(M) * K) / 5.4e6; }

// A workgroup per 16 columns reads its rows of W and, from the caches, the rows of A: 30 bytes a
// ns.  1 row, N = K = 4096: 5.8 us (streamed 9.5); 16 rows, N 6144: 10.5 (11.8); but 32 rows,
// 6144: 15.2 (12.2), and 16 rows, N 1024, K 14336: 16 (11).
double few_time(int M, int N, int K, int epi) {
  const bool glu = epi == kGluOut;
  const double wgs = double(cdiv(glu ? N / 2 : N, 16));
  const double bytes = std::ceil(wgs / kWorkers) * 16.0 * K * ((glu ? 2 : 1) + M / 16.0);
  return 2.5 + std::max(bytes / 30e3, read_time(M, N, K)) + (epi == kGluQuantOut ? 3.0 : 0.0);
}

// Every worker has the same share of stages; the planes are added by a second launch.
double stream_time(int M, int N, int K) {
  const int tm = M <= 32 ? 32 : M <= 64 ? 64 : 128;
  return 7.0 + double(N / 64) * (K / kGroup) / kWorkers * (tm == 32 ? 0.38 : tm == 64 ? 0.47 : 0.6);
}

// Whole tiles of tm x tn, a workgroup each: what a CU can load paces a stage (64 x 256: two stages in
// flight do not cover the latency).  256 rows, N = K = 4096:
// 64 x 64 13.3 us, 64 x 128 16 (split 128-row tiles 17.5); 501 rows: 22.9 and 16.4 (21.8);
// SwiGLU of 100 rows, N 28672: 128 x 128 30 (streamed 41).
double narrow_time(int M, int N, int K, int tm, int tn) {
  const int tiles = cdiv(M, tm) * (N / tn);
  const double rounds = cdiv(tiles, kWorkers), busy = std::max(tiles / rounds / kWorkers - 0.6, 0.0);
  const double stage = (tm == 128 ? 0.56 : tn == 64 ? 0.24 : tn == 128 ? 0.35 : 0.66) * (1.0 + 0.5 * busy);
  const double run = rounds * (K / kGroup * stage) + (rounds - 1) * 4.0, read = read_time(M, N, K);
  return 4.5 + std::max(run, read) + 0.1 * std::min(run, read);
}

// 256-column tiles in equal parts of K: with more than half of the CUs at work a stage takes
// longer (power, and what they read), and what W takes from memory hides only in part.
// Planes: 2 us and 0.27 us a MB.  736 rows, K 14336, N 4096: 128-row tiles in 2 parts 62 us,
// 256 in 4 56, whole 78; 200 rows of gate|up, N 28672: whole 128-row tiles 40, 256 47.
double wide_time(int M, int N, int K, int tm, int parts) {
  const int work = cdiv(M, tm) * cdiv(N, 256) * parts;
  const double rounds = cdiv(work, kWorkers), busy = std::max(work / rounds / kWorkers - 0.5, 0.0);
  const double stage = tm == 256 ? 0.965 + busy : tm == 192 ? 0.82 + 0.7 * busy : 0.685 + 0.4 * busy;
  const double run = rounds * (cdiv(K / kGroup, parts) * stage + (tm == 256 ? 6.0 : tm == 192 ? 4.8 : 3.6)), read = read_time(M, N, K);
  return std::max(std::max(run, read) + 0.45 * std::min(run, read), 3.0 + tm / 32.0) + (parts > 1 ? 2.0 + 0.27e-6 * 4 * parts * M * N : 0.0);
}

}  // namespace

Gemm8Plan gemm8_plan(int M, int N, int K, int epi) {
  Gemm8Plan best{Gemm8Kind::kWhole, 256, 256, 1};
  double time = 1e30;                                   // whole tiles run every size
  auto consider = [&](const Gemm8Plan& p, double t) {
    if (t < time) best = p, time = t;
  };
  if (M <= 32 && int64_t(M) * N * 4 <= int64_t(kPartial8Bytes))   // one plane, where it is needed
    consider(Gemm8Plan{Gemm8Kind::kFew, 0, 0, 0}, few_time(M, N, K, epi));
  if (gemm8_stream_fits(M, N, K)) consider(Gemm8Plan{Gemm8Kind::kStream, 0, 0, 0}, stream_time(M, N, K));
  constexpr int kNarrow[][2] = {{64, 64}, {64, 128}, {128, 128}, {64, 256}};
  for (const auto& t : kNarrow)
    if (gemm8_narrow_fits(N, K, epi, t[0], t[1]))
      consider(Gemm8Plan{Gemm8Kind::kNarrow, t[0], t[1], 0}, narrow_time(M, N, K, t[0], t[1]));
  for (const int tm : {256, 192, 128})
    for (int parts = 1; parts <= 16; ++parts) {
      const int64_t work = int64_t(cdiv(M, tm)) * cdiv(N, 256) * parts;
      if (parts > 1 && (work > kWorkers || int64_t(parts) * M * N * 4 > int64_t(kPartial8Bytes) || K / kGroup / parts < 2))
        break;
      // whole Q|K|V tiles leave the link write to a launch of its own
      consider(Gemm8Plan{parts == 1 ? Gemm8Kind::kWhole : Gemm8Kind::kSplit, tm, 256, parts},
               wide_time(M, N, K, tm, parts) + (epi == kRopeOut && parts == 1 ? 3.0 : 0.0));
    }
  return best;
}

StreamSum launch_gemm8_partial(const Gemm8Args& g, const Gemm8Plan& p, hipStream_t stream) {
  if (p.kind == Gemm8Kind::kFew) return launch_gemm8_few_plane(g, stream);
  if (p.kind == Gemm8Kind::kStream) return launch_gemm8_stream(g, stream);
  return launch_gemm8_split(g, p.tm, p.parts, stream);
}

void launch_gemm8_finish(const StreamSum& s, const Gemm8Args& g, int epi, hipStream_t stream) {
  const int cols = epi == kBf16Out ? g.N : g.N / 2;
  const int grid = cdiv(g.M * (cols / 4), 256);
  uint16_t* out = static_cast<uint16_t*>(g.out);
  if (epi == kBf16Out) finish_kernel<false><<<grid, 256, 0, stream>>>(s, out, cols);
  else if (epi == kGluOut) finish_kernel<true><<<grid, 256, 0, stream>>>(s, out, cols);
  else finish_quant_kernel<<<grid, 256, 0, stream>>>(s, g);
}

void launch_gemm8(const Gemm8Args& g, int epi, hipStream_t stream) {
  const Gemm8Plan p = gemm8_plan(g.M, g.N, g.K, epi);
  if (p.kind == Gemm8Kind::kWhole) launch_gemm8_wide(g, epi, p.tm, stream);
  else if (p.kind == Gemm8Kind::kNarrow) launch_gemm8_narrow(g, epi, p.tm, p.tn, stream);
  else if (p.kind == Gemm8Kind::kFew && epi != kGluQuantOut) launch_gemm8_few(g, epi, stream);
  else launch_gemm8_finish(launch_gemm8_partial(g, p, stream), g, epi, stream);
}

}  // namespace epic

// 8-bit GEMMs of up to 32 rows: one launch, no partial sums in memory.
//
// With few rows and moderate weights what counts is latency: a streamed product
// (gemm8_stream.hip) costs a second launch that adds its planes.  Here a workgroup has 16
// columns (SwiGLU: of the gate, and the same of the up half) and all of K, dealt to its
// eight wavefronts in blocks of 128 in turn, so that at any time the workgroup reads runs of
// 1 KB of each row of W; the wavefronts' sums meet in LDS.  Nothing is staged: every byte of W
// is used once, so it goes from memory to the registers of the 16 x 16 x 128 instruction
// that multiplies it, four blocks ahead (six: slower); the rows come from the caches.  What
// bounds it is the latency of memory.  N 6144, K 4096: 1 row 7.8 us (25 MB, 3.2 TB/s), 8 rows 9.3
// (streamed 11.4 and 11.6); 32 rows 15.0 (12.2), as every workgroup reads all rows.
//
// A lane has row l % 16 of either operand and of a block the 16-byte chunks l / 16 and
// l / 16 + 4 (which values of K does not matter, as both operands agree): each load
// instruction reads runs of 64 bytes.  The result has column l % 16 = row of A, and rows 4 (l / 16)
// + 0 .. 3 = columns of C.
#include "gemm8.h"
#include "gemm8_device.h"

namespace epic {

namespace {

constexpr int kNW = 8, kAhead = 4;                      // wavefronts; blocks in flight per wavefront

// MT: tiles of 16 rows.  OUT: kBf16Out, kGluOut, or kFewPlane: fp32 [M][N] for a pass that does more.
constexpr int kFewPlane = 4;
template <int OUT, int MT>
__global__ __launch_bounds__(kNW * 64) void gemm8_few_kernel(Gemm8Args g) {
  constexpr bool GLU = OUT == kGluOut;
  constexpr int NT = GLU ? 2 : 1;                       // tiles of 16 columns
  __shared__ __attribute__((aligned(16))) float part[kNW][NT][MT][16][16];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int ks = g.K >> 7, ld = (g.M + 3) & ~3, ffn = g.N / 2;
  const int n0 = blockIdx.x * 16;
  const int row = lane & 15, chunk = (lane >> 4) * 16;

  const uint8_t *wp[NT], *swp[NT], *ap[MT], *sap[MT];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const int n = n0 + t * ffn;
    wp[t] = g.W + size_t(n + row) * g.K + chunk;
    swp[t] = g.sw + size_t(n >> 7) * ks;
  }
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    const int m = min(t * 16 + row, g.M - 1);
    ap[t] = g.A + size_t(m) * g.K + chunk;
    sap[t] = g.sa + m;
  }

  typedef int i32x4 __attribute__((ext_vector_type(4)));
  struct Block {
    i32x4 w[NT][2], a[MT][2];
    uint8_t sw[NT], sa[MT];
  } ring[kAhead];
  auto load = [&](Block& b, int k) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      b.w[t][0] = *reinterpret_cast<const i32x4*>(wp[t] + k * 128);
      b.w[t][1] = *reinterpret_cast<const i32x4*>(wp[t] + k * 128 + 64);
      b.sw[t] = swp[t][k];
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
      b.a[t][0] = *reinterpret_cast<const i32x4*>(ap[t] + k * 128);
      b.a[t][1] = *reinterpret_cast<const i32x4*>(ap[t] + k * 128 + 64);
      b.sa[t] = sap[t][size_t(k) * ld];
    }
  };
  f32x4 acc[NT][MT] = {};
  auto multiply = [&](const Block& b) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
      for (int u = 0; u < MT; ++u)
        acc[t][u] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
            __builtin_shufflevector(b.w[t][0], b.w[t][1], 0, 1, 2, 3, 4, 5, 6, 7),
            __builtin_shufflevector(b.a[u][0], b.a[u][1], 0, 1, 2, 3, 4, 5, 6, 7), acc[t][u], 0, 0, 0, int(b.sw[t]), 0,
            int(b.sa[u]));
  };

#pragma unroll
  for (int i = 0; i < kAhead; ++i)
    if (wv + i * kNW < ks) load(ring[i], wv + i * kNW);
  for (int k = wv; k < ks; k += kAhead * kNW) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (k + i * kNW < ks) multiply(ring[i]);
      if (k + (kAhead + i) * kNW < ks) load(ring[i], k + (kAhead + i) * kNW);
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int u = 0; u < MT; ++u)
      *reinterpret_cast<f32x4*>(&part[wv][t][u][row][(lane >> 4) * 4]) = acc[t][u];
  __syncthreads();
  // two neighbouring columns of a row per thread
  const int r = tid >> 3, c = (tid & 7) * 2;
  if (r >= MT * 16 || r >= g.M) return;
  float x[NT][2];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    x[t][0] = x[t][1] = 0.0f;
#pragma unroll
    for (int w = 0; w < kNW; ++w) {
      const float2 v = *reinterpret_cast<const float2*>(&part[w][t][r >> 4][r & 15][c]);
      x[t][0] += v.x;
      x[t][1] += v.y;
    }
  }
  if constexpr (OUT == kFewPlane) {
    *reinterpret_cast<float2*>(g.partial + size_t(r) * g.N + n0 + c) = make_float2(x[0][0], x[0][1]);
  } else if constexpr (GLU) {
    reinterpret_cast<uint32_t*>(g.out)[(size_t(r) * ffn + n0 + c) / 2] =
        pack_bf16x2(silu(x[0][0]) * x[NT - 1][0], silu(x[0][1]) * x[NT - 1][1]);
  } else {
    reinterpret_cast<uint32_t*>(g.out)[(size_t(r) * g.N + n0 + c) / 2] = pack_bf16x2(x[0][0], x[0][1]);
  }
}

template <int OUT>
void launch_out(const Gemm8Args& g, hipStream_t stream) {
  const int grid = (OUT == kGluOut ? g.N / 2 : g.N) / 16;
  if (g.M <= 16) gemm8_few_kernel<OUT, 1><<<grid, kNW * 64, 0, stream>>>(g);
  else gemm8_few_kernel<OUT, 2><<<grid, kNW * 64, 0, stream>>>(g);
}

}  // namespace

void launch_gemm8_few(const Gemm8Args& g, int epi, hipStream_t stream) {
  if (epi == kGluOut) launch_out<kGluOut>(g, stream);
  else launch_out<kBf16Out>(g, stream);
}

StreamSum launch_gemm8_few_plane(const Gemm8Args& g, hipStream_t stream) {
  launch_out<kFewPlane>(g, stream);
  StreamSum s{};
  s.partial = g.partial;
  s.M = g.M, s.N = g.N, s.fixed = 1;
  return s;
}

}  // namespace epic

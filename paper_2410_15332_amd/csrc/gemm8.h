// Products of 8-bit rows and weights (host side): C[M x N] = A[M x K] . W[N x K]^T, both
// e4m3 with a power-of-two scale per 128 of K (and per 128 rows of W).  Shapes are
// validated by the entry points.
//
// Sums are fp32, but the matrix cores form an 8-bit dot product of eight neighbouring values
// first, and drop what lies more than 13 bits below the exponent of its largest product
// (so for every 8-bit instruction; measured).  That leaves 1.5e-5 to 4e-5 of the results' norm with
// operands of independent signs, far below the 2^-4 that the operands were rounded by, and a hundredth
// of what rounding to bf16 costs: hence results are bf16 or e4m3, and none is fp32; the scales of the
// quantised ones are decided in 64 bits next to their borders (gemm8_device.h).  Large products
// that cancel within their eight take the small ones beside them along: 448 w - 448 w in every eight
// leaves results 1e-2 to 1.6e-2 of their norm off.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "stream_sum.h"

namespace epic {

enum Gemm8Epilogue { kBf16Out = 0, kGluOut = 1, kGluQuantOut = 2, kRopeOut = 3 };

struct Gemm8Args {
  const uint8_t* A;     // [M][K] e4m3
  const uint8_t* sa;    // [K / 128][scale_ld(M)] e8m0
  const uint8_t* W;     // [N][K] e4m3 (SwiGLU: N / 2 gate rows, then N / 2 up rows)
  const uint8_t* sw;    // [N / 128][K / 128] e8m0
  void* out;            // bf16 [M][N] (kBf16Out) or [M][N / 2] (kGluOut), e4m3 [M][N / 2] (kGluQuantOut)
  uint8_t* out_scale;   // [N / 256][scale_ld(M)] e8m0 (kGluQuantOut)
  float* partial;       // planes of partial sums, kPartial8Bytes
  int M, N, K;
  // kRopeOut (the fused Q|K|V projection): columns are heads of head_dim, hq query heads, then
  // hkv key heads, then hkv value heads; q and k heads are rotated by the rotary table cs
  // [M][head_dim / 2] (cos, sin) of each row; bf16 q [M][hq][D], k / v [M][hkv][D].
  uint16_t *q, *k, *v;
  const float2* cs;
  int hq, hkv, head_dim;
};
// Requirements: K % 128 == 0, N % 128 == 0 (SwiGLU: N % 256 == 0); M * K, N * K and the
// bytes of an output below 2^31.

constexpr size_t kPartial8Bytes = size_t(64) << 20;

// How a product runs: up to 32 rows in one launch (kFew), weights streamed past a short row
// set (kStream), whole tiles of 64 or 128 rows and columns (kNarrow), or 256-column tiles of
// 128, 192 or 256 rows, whole (kWhole) or in equal parts of K (kSplit).  kStream and kSplit leave
// partial sums in planes.
enum class Gemm8Kind { kFew, kStream, kNarrow, kWhole, kSplit };
struct Gemm8Plan {
  Gemm8Kind kind;
  int tm, tn, parts;
};
Gemm8Plan gemm8_plan(int M, int N, int K, int epi);
void launch_gemm8(const Gemm8Args& g, int epi, hipStream_t stream);
// Partial sums only, for a consumer that adds them up (stream_sum.h); the planes are in g.partial.
StreamSum launch_gemm8_partial(const Gemm8Args& g, const Gemm8Plan& p, hipStream_t stream);
// The pass that adds the planes and runs the epilogue.
void launch_gemm8_finish(const StreamSum& s, const Gemm8Args& g, int epi, hipStream_t stream);

// of gemm8_few.hip, gemm8_stream.hip and gemm8_wide.hip
void launch_gemm8_few(const Gemm8Args& g, int epi, hipStream_t stream);       // not kGluQuantOut
StreamSum launch_gemm8_few_plane(const Gemm8Args& g, hipStream_t stream);     // one fp32 plane
StreamSum launch_gemm8_stream(const Gemm8Args& g, hipStream_t stream);
bool gemm8_narrow_fits(int N, int K, int epi, int tm, int tn);
void launch_gemm8_narrow(const Gemm8Args& g, int epi, int tm, int tn, hipStream_t stream);
bool gemm8_stream_fits(int M, int N, int K);
StreamSum gemm8_stream_sum(int M, int N, int K);   // how its tiles are dealt, without the planes' address
StreamSum launch_gemm8_split(const Gemm8Args& g, int tm, int parts, hipStream_t stream);
void launch_gemm8_wide(const Gemm8Args& g, int epi, int tm, hipStream_t stream);

}  // namespace epic

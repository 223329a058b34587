// Entry points of the 8-bit operators: argument validation on the host, then kernel
// launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "gemm8.h"
#include "quant.h"
#include "status.h"

using namespace epic;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

epic_status hip_status(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(EPIC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return EPIC_OK;
}

// The sizes of a product (epilogue: Gemm8Epilogue).
epic_status check_gemm_sizes(int epilogue, int32_t m, int32_t n, int32_t k) {
  EPIC_CHECK_ARG(m >= 0 && n > 0 && k > 0, "m, n, k = %d, %d, %d", m, n, k);
  const int per = epilogue == kGluOut || epilogue == kGluQuantOut ? 2 * kGroup : kGroup;
  if (k % kGroup != 0 || n % per != 0)
    return fail(EPIC_ERR_UNSUPPORTED, "k %% %d == 0 and n %% %d == 0 required (k = %d, n = %d)", kGroup, per, k, n);
  // 31-bit byte offsets, of the fp32 partial sums of short row sets too (they fit the workspace)
  const int64_t rows = int64_t(m) + 256, lim = int64_t(1) << 31;
  if (rows * k >= lim || int64_t(n) * k >= lim || rows * n * 2 >= lim)
    return fail(EPIC_ERR_UNSUPPORTED, "operands of %d x %d x %d exceed the 2^31-byte limit", m, n, k);
  return EPIC_OK;
}

}  // namespace

extern "C" size_t epic_fp8_scale_bytes(int32_t m, int32_t k) {
  if (m < 0 || k <= 0 || k % kGroup != 0) return 0;
  return size_t(k / kGroup) * ((size_t(m) + 3) / 4 * 4);
}

extern "C" epic_status epic_quant_fp8(const uint16_t* x, int32_t m, int32_t k, int32_t block_rows, uint8_t* q,
                                      uint8_t* scale, void* stream) {
  clear_error();
  EPIC_CHECK_ARG(m >= 0 && k > 0, "m, k = %d, %d", m, k);
  EPIC_CHECK_ARG(block_rows == 1 || block_rows == kGroup, "block_rows %d (expected 1 or %d)", block_rows, kGroup);
  if (k % kGroup != 0) return fail(EPIC_ERR_UNSUPPORTED, "k %d must be a multiple of %d", k, kGroup);
  if (m > INT32_MAX - 4 || int64_t(m) * k / 8 > kMaxThreads || (block_rows == kGroup && m > 65535 * kGroup))
    return fail(EPIC_ERR_UNSUPPORTED, "%d x %d values are too many", m, k);
  if (m == 0) return EPIC_OK;
  EPIC_CHECK_ARG(x && q && scale, "NULL tensor argument");
  EPIC_CHECK_ARG(aligned(x, 16) && aligned(q, 16), "x and q must be 16-byte aligned");
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (block_rows == 1) launch_quant_rows(x, m, k, q, scale, s);
  else launch_quant_blocks(x, m, k, q, scale, s);
  return hip_status("quantisation launch");
}

extern "C" epic_status epic_rmsnorm_fp8(const float* x, const uint16_t* delta, const uint16_t* weight, int32_t m,
                                        int32_t hidden, float eps, float* x_out, uint8_t* q, uint8_t* scale,
                                        void* stream) {
  clear_error();
  EPIC_CHECK_ARG(m >= 0 && hidden > 0, "m, hidden = %d, %d", m, hidden);
  EPIC_CHECK_ARG(eps > 0.0f, "eps must be > 0");
  if (hidden % kGroup != 0 || hidden > kMaxNormHidden)
    return fail(EPIC_ERR_UNSUPPORTED, "hidden %d must be a multiple of %d, at most %d", hidden, kGroup, kMaxNormHidden);
  if (m > INT32_MAX - 4 || int64_t(m) * norm_threads(hidden) > kMaxThreads)
    return fail(EPIC_ERR_UNSUPPORTED, "%d rows of %d are too many", m, hidden);
  if (m == 0) return EPIC_OK;
  EPIC_CHECK_ARG(x && weight && q && scale, "NULL tensor argument");
  EPIC_CHECK_ARG(aligned(x, 16) && aligned(weight, 16) && aligned(q, 16) && aligned(delta, 16) && aligned(x_out, 16),
                 "tensors must be 16-byte aligned");
  launch_rmsnorm_fp8(x, delta, StreamSum{}, weight, m, hidden, eps, x_out, q, scale, static_cast<hipStream_t>(stream));
  return hip_status("norm launch");
}

extern "C" size_t epic_gemm_fp8_workspace_bytes(void) { return kPartial8Bytes; }

extern "C" epic_status epic_gemm_fp8(int32_t epilogue, const uint8_t* a, const uint8_t* a_scale, const uint8_t* w,
                                     const uint8_t* w_scale, int32_t m, int32_t n, int32_t k, void* out,
                                     uint8_t* out_scale, void* workspace, size_t workspace_bytes, void* stream) {
  clear_error();
  EPIC_CHECK_ARG(epilogue >= EPIC_FP8_BF16 && epilogue <= EPIC_FP8_SWIGLU_FP8, "unknown epilogue %d", epilogue);
  epic_status st = check_gemm_sizes(epilogue, m, n, k);
  if (st != EPIC_OK) return st;
  if (m == 0) return EPIC_OK;
  EPIC_CHECK_ARG(a && a_scale && w && w_scale && aligned(a, 16) && aligned(w, 16),
                 "operands must be non-NULL, a and w 16-byte aligned");
  EPIC_CHECK_ARG(aligned(a_scale, 4), "a_scale must be 4-byte aligned");
  EPIC_CHECK_ARG(out && aligned(out, 16), "out must be non-NULL and 16-byte aligned");
  if (epilogue == EPIC_FP8_SWIGLU_FP8)
    EPIC_CHECK_ARG(out_scale && aligned(out_scale, 4), "out_scale must be non-NULL and 4-byte aligned");
  if (workspace == nullptr || workspace_bytes < kPartial8Bytes)
    return fail(EPIC_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, kPartial8Bytes);
  EPIC_CHECK_ARG(aligned(workspace, 256), "workspace must be 256-byte aligned");
  Gemm8Args g{};
  g.A = a, g.sa = a_scale, g.W = w, g.sw = w_scale;
  g.M = m, g.N = n, g.K = k;
  g.out = out, g.out_scale = out_scale;
  g.partial = static_cast<float*>(workspace);
  launch_gemm8(g, epilogue, static_cast<hipStream_t>(stream));
  return hip_status("8-bit GEMM launch");
}

// The kernel that the plan has for a product of these sizes (epilogue: Gemm8Epilogue, kRopeOut too), or "" where they are
// not whole groups of 128.  It plans also what the entry points refuse for other reasons (SwiGLU of an odd number of
// blocks, operands of 2^31 bytes).  Host only and not in the public header: it is for tests, each of which is about one kernel.
extern "C" const char* epic_gemm_fp8_route_name(int32_t epilogue, int32_t m, int32_t n, int32_t k) {
  if (epilogue < kBf16Out || epilogue > kRopeOut || m <= 0 || n <= 0 || k <= 0 || n % kGroup != 0 || k % kGroup != 0)
    return "";
  const Gemm8Plan p = gemm8_plan(m, n, k, epilogue);
  if (p.kind == Gemm8Kind::kFew) return "few";
  if (p.kind == Gemm8Kind::kStream) return "stream";
  if (p.kind == Gemm8Kind::kNarrow)
    return p.tm == 128 ? "narrow128x128" : p.tn == 256 ? "narrow64x256" : p.tn == 128 ? "narrow64x128" : "narrow64x64";
  if (p.kind == Gemm8Kind::kSplit) return p.tm == 256 ? "split256" : p.tm == 192 ? "split192" : "split128";
  return p.tm == 256 ? "whole256" : p.tm == 192 ? "whole192" : "whole128";
}

// The fp32 planes [m][n] of partial sums that such a product has at most (few rows: one, where its consumer adds it), or -1
// for sizes that are refused.  For tests too.
extern "C" int32_t epic_gemm_fp8_planes(int32_t epilogue, int32_t m, int32_t n, int32_t k) {
  clear_error();
  if (epilogue < kBf16Out || epilogue > kRopeOut || m == 0 || check_gemm_sizes(epilogue, m, n, k) != EPIC_OK) return -1;
  const Gemm8Plan p = gemm8_plan(m, n, k, epilogue);
  if (p.kind == Gemm8Kind::kFew) return 1;
  if (p.kind == Gemm8Kind::kSplit) return p.parts;
  if (p.kind != Gemm8Kind::kStream) return 0;
  const StreamSum s = gemm8_stream_sum(m, n, k);
  int planes = 0;
  for (int tile = 0; tile < s.units / s.ks; ++tile) planes = std::max(planes, s.planes(tile));
  return planes;
}

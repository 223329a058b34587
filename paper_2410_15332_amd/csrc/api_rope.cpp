// Entry points of the head norm and rotation: frequencies on the host, argument validation,
// then one launch on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "plan_internal.h"
#include "qk_rope.h"
#include "status.h"

using namespace epic;

namespace {

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

epic_status validate_rope_cfg(const epic_rope_cfg* r) {
  EPIC_CHECK_ARG(r != nullptr, "rotation config is NULL");
  EPIC_CHECK_ARG(r->rot_dim >= 0 && r->rot_dim % 16 == 0, "rot_dim %d must be a multiple of 16", r->rot_dim);
  EPIC_CHECK_ARG(r->interleaved == 0 || r->interleaved == 1, "interleaved %d (expected 0 or 1)", r->interleaved);
  EPIC_CHECK_ARG(r->theta > 1.0f && std::isfinite(r->theta), "theta %g must be > 1", r->theta);
  EPIC_CHECK_ARG(r->factor >= 0.0f && std::isfinite(r->factor), "factor %g must be >= 0", r->factor);
  EPIC_CHECK_ARG(r->original_context >= 0, "original_context %d < 0", r->original_context);
  if (r->original_context > 0)
    EPIC_CHECK_ARG(r->low_turns >= 0.0f && r->high_turns > r->low_turns && std::isfinite(r->high_turns),
                   "low_turns %g, high_turns %g: 0 <= low < high required", r->low_turns, r->high_turns);
  EPIC_CHECK_ARG(r->amplitude >= 0.0f && std::isfinite(r->amplitude), "amplitude %g must be >= 0", r->amplitude);
  return EPIC_OK;
}

// Whether [a, a + n) and [b, b + m) have a byte in common.
bool overlap(const void* a, size_t n, const void* b, size_t m) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + m && y < x + n;
}

}  // namespace

extern "C" epic_status epic_rope_freqs(const epic_rope_cfg* rope, double* freqs) {
  clear_error();
  epic_status st = validate_rope_cfg(rope);
  if (st != EPIC_OK) return st;
  if (rope->rot_dim == 0) return EPIC_OK;
  EPIC_CHECK_ARG(freqs != nullptr, "freqs is NULL");
  const double factor = rope->factor > 0.0f ? double(rope->factor) : 1.0;
  const double two_pi = 6.283185307179586476925;
  for (int j = 0; j < rope->rot_dim / 2; ++j) {
    const double f = std::pow(double(rope->theta), -2.0 * j / rope->rot_dim);
    double keep = 0.0;                          // share of the frequency that is not divided
    if (rope->original_context > 0)
      keep = std::clamp((rope->original_context * f / two_pi - rope->low_turns) / (double(rope->high_turns) - rope->low_turns),
                        0.0, 1.0);
    freqs[j] = f * (keep + (1.0 - keep) / factor);
  }
  return EPIC_OK;
}

extern "C" epic_status epic_qk_norm_rope(const epic_attn_cfg* cfg, const epic_rope_cfg* rope, int32_t in_type,
                                         const void* qkv, int64_t ld, int32_t rows, const int32_t* pos,
                                         const double* freqs, const uint16_t* q_norm, const uint16_t* k_norm, float eps,
                                         uint16_t* q, uint16_t* k, uint16_t* v, void* stream) {
  clear_error();
  epic_status st = validate_attn_cfg(cfg);
  if (st != EPIC_OK) return st;
  st = validate_rope_cfg(rope);
  if (st != EPIC_OK) return st;
  const int d = cfg->head_dim, hq = cfg->num_q_heads, hkv = cfg->num_kv_heads;
  EPIC_CHECK_ARG(rope->rot_dim <= d, "rot_dim %d past the head dim %d", rope->rot_dim, d);
  EPIC_CHECK_ARG(in_type == EPIC_QKV_BF16 || in_type == EPIC_QKV_FP32, "unknown input type %d", in_type);
  EPIC_CHECK_ARG(rows >= 0, "rows %d < 0", rows);
  const int64_t cols = (int64_t(hq) + 2 * int64_t(hkv)) * d;
  const int elem = in_type == EPIC_QKV_FP32 ? 4 : 2;
  EPIC_CHECK_ARG(ld >= cols && ld * elem % 16 == 0, "row stride %lld: at least %lld, and a multiple of 16 bytes", (long long)ld,
                 (long long)cols);
  if (q_norm || k_norm) EPIC_CHECK_ARG(eps > 0.0f, "eps must be > 0");
  // grids, and byte counts below 2^63
  if (rows > kQkMaxRows || cols > (int64_t(1) << 26) || ld > (int64_t(1) << 36))
    return fail(EPIC_ERR_UNSUPPORTED, "%d rows of %lld values are too many", rows, (long long)cols);
  if (rows == 0) return EPIC_OK;
  EPIC_CHECK_ARG(qkv && pos && q && k && v, "NULL tensor argument");
  if (rope->rot_dim > 0) EPIC_CHECK_ARG(freqs && aligned(freqs, 8), "freqs NULL or unaligned");
  EPIC_CHECK_ARG(aligned(qkv, 16) && aligned(q, 16) && aligned(k, 16) && aligned(v, 16) && aligned(q_norm, 16) &&
                     aligned(k_norm, 16),
                 "tensors must be 16-byte aligned");
  const size_t in_bytes = (size_t(rows - 1) * ld + cols) * elem;
  const size_t q_bytes = size_t(rows) * hq * d * 2, kv_bytes = size_t(rows) * hkv * d * 2;
  EPIC_CHECK_ARG(!overlap(qkv, in_bytes, q, q_bytes) && !overlap(qkv, in_bytes, k, kv_bytes) &&
                     !overlap(qkv, in_bytes, v, kv_bytes) && !overlap(q, q_bytes, k, kv_bytes) &&
                     !overlap(q, q_bytes, v, kv_bytes) && !overlap(k, kv_bytes, v, kv_bytes),
                 "q, k, v and the input may not overlap");
  QkRopeArgs p{};
  p.qkv = qkv, p.pos = pos, p.freqs = freqs, p.q_norm = q_norm, p.k_norm = k_norm;
  p.q = q, p.k = k, p.v = v, p.ld = ld;
  p.rows = rows, p.hq = hq, p.hkv = hkv, p.rot = rope->rot_dim;
  p.eps = eps, p.amplitude = rope->amplitude > 0.0f ? rope->amplitude : 1.0f;
  launch_qk_rope(p, d, in_type == EPIC_QKV_FP32, rope->interleaved != 0, static_cast<hipStream_t>(stream));
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(EPIC_ERR_HIP, "norm and rotation launch: %s", hipGetErrorString(e));
  return EPIC_OK;
}

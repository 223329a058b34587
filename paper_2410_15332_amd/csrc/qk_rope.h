// Norm and rotation of the query and key heads of Q|K|V rows.  Host side of qk_rope.hip;
// arguments are validated by the callers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace epic {

struct QkRopeArgs {
  const void* qkv;                            // [rows][ld], bf16 or fp32: q heads, k heads, v heads
  const int32_t* pos;                         // [rows]
  const double* freqs;                        // [rot / 2], radians a position
  const uint16_t* q_norm;                     // [head dim], or null: not normed
  const uint16_t* k_norm;
  uint16_t *q, *k, *v;
  int64_t ld;
  int rows, hq, hkv, rot;
  float eps, amplitude;
};

// A workgroup of 256 threads a row: fewer than 2^32 threads.
constexpr int64_t kQkMaxRows = (int64_t(1) << 24) - 4;

void launch_qk_rope(const QkRopeArgs& p, int head_dim, bool fp32, bool interleaved, hipStream_t stream);

}  // namespace epic

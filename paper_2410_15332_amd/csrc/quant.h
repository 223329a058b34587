// 8-bit operands of the projections: e4m3 values with one power-of-two scale (an e8m0
// byte, 2^(byte - 127)) per group of 128 consecutive values of a row, or per 128 x 128
// block of a weight matrix.  Host side of quant.hip; sizes are validated by the callers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "stream_sum.h"

namespace epic {

constexpr int kGroup = 128;                             // values that share a scale
constexpr int kMaxNormHidden = 32768;                   // longest row of the 8-bit norm

// Row scales are [k / 128][scale_ld(m)]: a group's scales of all rows are contiguous, so a
// GEMM tile's come in one load per K stage; padded so that four rows are one aligned load.
inline int scale_ld(int m) { return (m + 3) & ~3; }

// Threads of a launch have to stay below 2^32: 8 values a thread, norm_threads() a row.
constexpr int64_t kMaxThreads = (int64_t(1) << 32) - 1024;
inline int norm_threads(int hidden) { return hidden > 4 * 8 * 512 ? 1024 : hidden >= 4 * 512 ? 512 : (hidden / 4 + 63) / 64 * 64; }

void launch_quant_rows(const uint16_t* x, int m, int k, uint8_t* q, uint8_t* scale, hipStream_t stream);
void launch_quant_blocks(const uint16_t* x, int m, int k, uint8_t* q, uint8_t* scale, hipStream_t stream);
// x + delta (bf16 [m][hidden]) or + the planes of s, where one is given, into x_out (where not
// null), and the RMSNorm of that into q, scale.  x_out may be x.
void launch_rmsnorm_fp8(const float* x, const uint16_t* delta, const StreamSum& s, const uint16_t* w, int m, int hidden,
                        float eps, float* x_out, uint8_t* q, uint8_t* scale, hipStream_t stream);

}  // namespace epic

// Norm and rotation of the query and key heads of Q|K|V rows, in one pass.
//
//   y = x / sqrt(mean(x^2) + eps) * w          per head, where a weight is given
//   (a, b) -> amplitude (a cos - b sin, b cos + a sin), angle pos * f_j,
// for the pairs j of the first `rot` dims: (j, j + rot / 2), or (2 j, 2 j + 1) interleaved; the
// other dims, and V, pass.  Statistics and products are fp32, the result is rounded once.
// Angles: pos * f_j in float64, in turns, less the nearest quarter turn; what is left is at
// most pi / 4 and goes to fp32 (off by 2^-25 of itself), where the Taylor polynomials of sine
// and cosine to x^9 and x^10 are off by 2e-9: below fp32's own rounding.
//
// What bounds it is reading and writing the rows once.  A head is D / 16 lanes of 16 values,
// two pieces of 8 each: both pieces of a lane's pairs, so a rotation stays in the lane.  A workgroup
// takes a row in passes of 256 threads, the next pass's loads ahead of this one's work; the row's
// angles (one per thread) are computed once, into LDS, while the first loads are in flight.
#include "device_common.h"
#include "qk_rope.h"

namespace epic {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64;

// (cos, sin) of pos * f.
__device__ __forceinline__ float2 turn_of(int pos, double f) {
  const double turns = double(pos) * (f * 0.15915494309189533577);     // 1 / 2 pi
  const double left = turns - rint(turns);                             // exact, -1/2 .. 1/2
  const double quarter = rint(4.0 * left);
  const float x = float((left - 0.25 * quarter) * 6.28318530717958647693), z = x * x;
  const float s = x * (1.0f + z * (-1.0f / 6 + z * (1.0f / 120 + z * (-1.0f / 5040 + z * (1.0f / 362880)))));
  const float c = 1.0f + z * (-0.5f + z * (1.0f / 24 + z * (-1.0f / 720 + z * (1.0f / 40320 + z * (-1.0f / 3628800)))));
  const int n = int(quarter) & 3;
  const float cn = n & 1 ? s : c, sn = n & 1 ? c : s;
  return make_float2(n == 1 || n == 2 ? -cn : cn, n >= 2 ? -sn : sn);
}

// Eight values of a row, as they lie.
template <bool F32>
struct Piece;
template <>
struct Piece<false> {
  uint4 w;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    w = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + at);
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(u[i] << 16);
      x[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  __device__ __forceinline__ uint4 bf16() const { return w; }
};
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}
template <>
struct Piece<true> {
  float4 a, b;
  __device__ __forceinline__ void load(const void* p, size_t at) {
    const float4* f = reinterpret_cast<const float4*>(static_cast<const float*>(p) + at);
    a = f[0], b = f[1];
  }
  __device__ __forceinline__ void get(float (&x)[8]) const {
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
  }
  __device__ __forceinline__ uint4 bf16() const {
    const float x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return pack8(x);
  }
};

template <int D, bool F32, bool INTER>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(QkRopeArgs p) {
  constexpr int L = D / 16;                   // lanes per head
  __shared__ float2 cs[kMaxPairs];
  const int heads = p.hq + 2 * p.hkv, row = blockIdx.x, step = kThreads / L * gridDim.y;
  const int l = threadIdx.x % L;
  // this lane's two pieces of 8 dims: the two sides of its pairs (half layout), or neighbours
  const int R = p.rot / 8;                    // rotated pieces, an even number
  const bool turned = l < R / 2;
  const int c0 = INTER || !turned ? 2 * l : l, c1 = INTER || !turned ? 2 * l + 1 : l + R / 2;

  int head = blockIdx.y * (kThreads / L) + threadIdx.x / L;
  Piece<F32> x[2];
  auto fetch = [&](int at) __attribute__((always_inline)) {
    const size_t from = size_t(row) * p.ld + size_t(min(at, heads - 1)) * D;
    x[0].load(p.qkv, from + 8 * c0);
    x[1].load(p.qkv, from + 8 * c1);
  };
  fetch(head);
  uint4 wq[2] = {}, wk[2] = {};
  if (p.q_norm) {
    wq[0] = *reinterpret_cast<const uint4*>(p.q_norm + 8 * c0);
    wq[1] = *reinterpret_cast<const uint4*>(p.q_norm + 8 * c1);
  }
  if (p.k_norm) {
    wk[0] = *reinterpret_cast<const uint4*>(p.k_norm + 8 * c0);
    wk[1] = *reinterpret_cast<const uint4*>(p.k_norm + 8 * c1);
  }
  if (int(threadIdx.x) < p.rot / 2) {
    const float2 t = turn_of(p.pos[row], p.freqs[threadIdx.x]);
    cs[threadIdx.x] = make_float2(p.amplitude * t.x, p.amplitude * t.y);
  }
  __syncthreads();
  for (;; head += step) {
    const Piece<F32> y0 = x[0], y1 = x[1];
    if (head + step < heads) fetch(head + step);
    const bool is_q = head < p.hq, is_v = head >= p.hq + p.hkv;
    float u[8], v[8];
    y0.get(u);
    y1.get(v);
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += u[i] * u[i] + v[i] * v[i];
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
    if (head >= heads) break;                 // after the exchange: all lanes of a head together
    uint4 r0 = y0.bf16(), r1 = y1.bf16();
    if (!is_v) {
      if ((is_q ? p.q_norm : p.k_norm) != nullptr) {
        const float inv = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
        float w0[8], w1[8];
        Piece<false>{is_q ? wq[0] : wk[0]}.get(w0);
        Piece<false>{is_q ? wq[1] : wk[1]}.get(w1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[i] = u[i] * inv * w0[i];
          v[i] = v[i] * inv * w1[i];
        }
      }
      if (turned) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (INTER) {              // pairs 8 l + i: u holds four of them, then v
            float* e = i < 4 ? u + 2 * i : v + 2 * (i - 4);
            const float2 k = cs[8 * l + i];
            const float a = e[0], b = e[1];
            e[0] = a * k.x - b * k.y;
            e[1] = b * k.x + a * k.y;
          } else {
            const float2 k = cs[8 * l + i];
            const float a = u[i], b = v[i];
            u[i] = a * k.x - b * k.y;
            v[i] = b * k.x + a * k.y;
          }
        }
      }
      r0 = pack8(u);
      r1 = pack8(v);
    }
    const size_t at = row;
    uint16_t* to = is_q ? p.q + (at * p.hq + head) * D
                        : is_v ? p.v + (at * p.hkv + (head - p.hq - p.hkv)) * D : p.k + (at * p.hkv + (head - p.hq)) * D;
    *reinterpret_cast<uint4*>(to + 8 * c0) = r0;
    *reinterpret_cast<uint4*>(to + 8 * c1) = r1;
  }
}

}  // namespace

void launch_qk_rope(const QkRopeArgs& p, int head_dim, bool fp32, bool interleaved, hipStream_t stream) {
  // Passes of 32 heads (64 of 64 dims) over a row; each a workgroup of its own where rows are fewer
  // than CUs.  32 + 8 + 8 heads of 128: 1 row 2.8 us (3.5 undivided), 736 rows of fp32 7.5 (8.4 divided), 20 560 rows
  // 85 (505 MB, 5.9 TB/s; 96 to 99 divided, with 4 rows a workgroup, or in one pass of 384 threads).
  const int per_pass = kThreads / (head_dim / 16);
  const int passes = p.rows < 256 ? (p.hq + 2 * p.hkv + per_pass - 1) / per_pass : 1;
  auto go = [&](auto kernel) { kernel<<<dim3(p.rows, passes), kThreads, 0, stream>>>(p); };
  if (head_dim == 128) {
    if (fp32) interleaved ? go(qk_rope_kernel<128, true, true>) : go(qk_rope_kernel<128, true, false>);
    else interleaved ? go(qk_rope_kernel<128, false, true>) : go(qk_rope_kernel<128, false, false>);
  } else {
    if (fp32) interleaved ? go(qk_rope_kernel<64, true, true>) : go(qk_rope_kernel<64, true, false>);
    else interleaved ? go(qk_rope_kernel<64, false, true>) : go(qk_rope_kernel<64, false, false>);
  }
}

}  // namespace epic

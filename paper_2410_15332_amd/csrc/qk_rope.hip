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
// takes a row, or several short ones (MANY), in passes of 256 threads, the next pass's loads ahead of this one's
// work; the angles are computed once, into LDS, while the first loads are in flight.
#include <type_traits>

#include "device_common.h"
#include "qk_rope.h"

namespace epic {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxPairs = 64, kMaxRows = 8;

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

template <int D, bool F32, bool INTER, bool MANY>
__global__ __launch_bounds__(kThreads) void qk_rope_kernel(QkRopeArgs p, int rows_per_group) {
  constexpr int L = D / 16;                   // lanes per head
  __shared__ float2 cs[MANY ? kMaxRows : 1][kMaxPairs];
  const int heads = p.hq + 2 * p.hkv, half = p.rot / 2, step = kThreads / L * gridDim.y;
  const int row0 = blockIdx.x * (MANY ? rows_per_group : 1), rows = MANY ? min(rows_per_group, p.rows - row0) : 1;
  const int total = rows * heads;
  const int l = threadIdx.x % L;
  // this lane's two pieces of 8 dims: the two sides of its pairs (half layout), or neighbours
  const int R = p.rot / 8;                    // rotated pieces, an even number
  const bool turned = l < R / 2;
  const int c0 = INTER || !turned ? 2 * l : l, c1 = INTER || !turned ? 2 * l + 1 : l + R / 2;

  int at = blockIdx.y * (kThreads / L) + threadIdx.x / L;       // (row of the group, head), and the next one's values
  Piece<F32> x[2];
  auto fetch = [&](int i) __attribute__((always_inline)) {
    i = min(i, total - 1);
    const int row = MANY ? i / heads : 0;
    const size_t from = size_t(row0 + row) * p.ld + size_t(i - row * heads) * D;
    x[0].load(p.qkv, from + 8 * c0);
    x[1].load(p.qkv, from + 8 * c1);
  };
  fetch(at);
  uint4 wq[2] = {}, wk[2] = {};
  if (p.q_norm) {
    wq[0] = *reinterpret_cast<const uint4*>(p.q_norm + 8 * c0);
    wq[1] = *reinterpret_cast<const uint4*>(p.q_norm + 8 * c1);
  }
  if (p.k_norm) {
    wk[0] = *reinterpret_cast<const uint4*>(p.k_norm + 8 * c0);
    wk[1] = *reinterpret_cast<const uint4*>(p.k_norm + 8 * c1);
  }
  for (int i = threadIdx.x; i < rows * half; i += kThreads) {
    const int row = MANY ? i / half : 0;
    const float2 t = turn_of(p.pos[row0 + row], p.freqs[i - row * half]);
    cs[row][i - row * half] = make_float2(p.amplitude * t.x, p.amplitude * t.y);
  }
  __syncthreads();
  for (;; at += step) {
    const Piece<F32> y0 = x[0], y1 = x[1];
    if (at + step < total) fetch(at + step);
    const int row = MANY ? at / heads : 0, head = at - row * heads;
    const bool is_q = head < p.hq, is_v = head >= p.hq + p.hkv;
    float u[8], v[8];
    y0.get(u);
    y1.get(v);
    float ss = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) ss += u[i] * u[i] + v[i] * v[i];
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) ss += __shfl_xor(ss, off);
    if (at >= total) break;                   // after the exchange: all lanes of a head together
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
            const float2 k = cs[row][8 * l + i];
            const float a = e[0], b = e[1];
            e[0] = a * k.x - b * k.y;
            e[1] = b * k.x + a * k.y;
          } else {
            const float2 k = cs[row][8 * l + i];
            const float a = u[i], b = v[i];
            u[i] = a * k.x - b * k.y;
            v[i] = b * k.x + a * k.y;
          }
        }
      }
      r0 = pack8(u);
      r1 = pack8(v);
    }
    const size_t r = row0 + row;
    uint16_t* to = is_q ? p.q + (r * p.hq + head) * D
                        : is_v ? p.v + (r * p.hkv + (head - p.hq - p.hkv)) * D : p.k + (r * p.hkv + (head - p.hq)) * D;
    *reinterpret_cast<uint4*>(to + 8 * c0) = r0;
    *reinterpret_cast<uint4*>(to + 8 * c1) = r1;
  }
}

}  // namespace

void launch_qk_rope(const QkRopeArgs& p, int head_dim, bool fp32, bool interleaved, hipStream_t stream) {
  // A pass takes 32 heads (64 of 64 dims).  Rows fewer than CUs: a workgroup for each pass over a row (1 row of 32 + 8 + 8
  // heads of 128: 2.8 us, 3.5 undivided).  Else a row a workgroup: 736 rows of fp32 7.3 us, 20 560 rows 87 (505 MB, 5.8
  // TB/s; 92 to 99 with more rows, divided, or in one pass of more threads).  Rows that are less than a pass go
  // several to a workgroup, to two passes, where these are as many as CUs: 16 + 1 + 1 heads of 64, 900 rows 3.8 us (4.2 if
  // they did), 2000 rows 5.0 (5.4 by rows), 20 560 rows 20 (33 by rows, 22 to one pass).
  const int heads = p.hq + 2 * p.hkv, per_pass = kThreads / (head_dim / 16);
  const bool few = p.rows < 256;
  const int most = heads >= per_pass ? 1 : min(kMaxRows, 2 * per_pass / heads), rows = p.rows >= 256 * most ? most : 1;
  const dim3 grid((p.rows + rows - 1) / rows, few ? (heads + per_pass - 1) / per_pass : 1);
  auto go = [&](auto one, auto many) {
    if (rows == 1) one<<<grid, kThreads, 0, stream>>>(p, 1);
    else many<<<grid, kThreads, 0, stream>>>(p, rows);
  };
  auto pairs = [&](auto d, auto f32) {
    constexpr int D = decltype(d)::value;
    constexpr bool F32 = decltype(f32)::value;
    if (interleaved) go(qk_rope_kernel<D, F32, true, false>, qk_rope_kernel<D, F32, true, true>);
    else go(qk_rope_kernel<D, F32, false, false>, qk_rope_kernel<D, F32, false, true>);
  };
  auto type = [&](auto d) { fp32 ? pairs(d, std::true_type{}) : pairs(d, std::false_type{}); };
  if (head_dim == 128) type(std::integral_constant<int, 128>{});
  else type(std::integral_constant<int, 64>{});
}

}  // namespace epic

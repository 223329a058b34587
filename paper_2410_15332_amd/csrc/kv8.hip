// The 8-bit cache: blocks from a bf16 cache and back, and the link write of an 8-bit cache.
//
// A row y (the D values of K or of V of a token and KV head) is stored as q = e4m3(y / 2^t),
// rounded once, to nearest even, with t the smallest integer such that max |y| <= 448 2^t.  A
// power of two costs no relative precision against a finer scale (e4m3 has an exponent of its
// own), and attention applies it after the products: K's to the scores, V's to the
// probabilities, where it is exact.  A token of which a value of K or V is not finite is
// stored as NaN, both rows: byte 255, K all NaN, V all 0.  Whatever attends to it gets NaN
// from the score; whatever does not meets only the zeros, since a weight of 0 times a NaN in
// V would be NaN.
//
// One wavefront per (block, KV head), the slab in registers (kv8_device.h).  The kernels are bound by
// reading and writing these bytes; all do it once but the widening that also writes private blocks, which
// forms a linked private block from its source and rows a second time.
#include <cmath>

#include "kv8_device.h"

namespace epic {

namespace {

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;

// The (list entry, KV head) of this wavefront: pairs in order, so few heads fill workgroups too.
struct Place {
  int i, g;
  bool in;
  __device__ __forceinline__ Place(int n, int hkv, int group) {
    const int pair = group * kWaves + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
    i = pair / hkv;
    g = pair - i * hkv;
    in = i < n;
  }
};

// Four bf16 (two pairs), each over its own 2^(byte - 127), as e4m3.  NaN rows (255) hold zeros in V.
__device__ __forceinline__ uint32_t round4_each(uint32_t lo, uint32_t hi, const int (&b)[4]) {
  auto in = [&](uint32_t bits, int byte) {
    return byte == kKv8Nan ? 0.0f : __builtin_amdgcn_ldexpf(__uint_as_float(bits), 127 - byte);
  };
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(in(lo << 16, b[0]), in(lo & 0xFFFF0000u, b[1]), 0, false);
  return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(in(hi << 16, b[2]), in(hi & 0xFFFF0000u, b[3]), r, true));
}

// 8192 blocks of 8 heads of 128 (806 MB): 155 us, 5.2 TB/s (two bytes read per byte written; 161 through the caches).
template <int D>
__global__ __launch_bounds__(kThreads) void kv8_pack_kernel(Kv8Move mv, const uint16_t* __restrict__ k,
                                                            const uint16_t* __restrict__ v, epic_kv8_cache c) {
  constexpr int J = D / 64;
  const Place at(mv.n, mv.hkv, blockIdx.x);
  if (!at.in) return;
  const int src = mv.src ? mv.src[at.i] : at.i, dst = mv.dst ? mv.dst[at.i] : at.i;
  if (unsigned(src) >= unsigned(mv.src_blocks) || unsigned(dst) >= unsigned(mv.dst_blocks)) return;
  const int lane = threadIdx.x & 63, r = lane & 15, a = lane >> 4;
  const size_t from = (size_t(src) * mv.hkv + at.g) * 16 * D, to = (size_t(dst) * mv.hkv + at.g) * 16 * D;
  uint4 x[2 * J];
  uint2 y[4 * J];                              // tokens 4 a .. of dims 16 i + r
#pragma unroll
  for (int i = 0; i < 2 * J; ++i)
    x[i] = load16(k + from + r * D + 64 * (i >> 1) + 16 * a + 8 * (i & 1));
#pragma unroll
  for (int i = 0; i < 4 * J; ++i) y[i] = load8(v + from + (16 * i + r) * 16 + 4 * a);
  int kb = kv8_byte(row_top<J>(x));
  uint32_t m0 = 0, m1 = 0;
#pragma unroll
  for (int i = 0; i < 4 * J; ++i) {
    m0 = pair_max(m0, pair_abs(y[i].x));
    m1 = pair_max(m1, pair_abs(y[i].y));
  }
  m0 = row16_pair_max(m0);
  m1 = row16_pair_max(m1);
  int vb[4] = {kv8_byte(m0 & 0xFFFFu), kv8_byte(m0 >> 16), kv8_byte(m1 & 0xFFFFu), kv8_byte(m1 >> 16)};
  const bool bad = kb == kKv8Nan || vb[0] == kKv8Nan || vb[1] == kKv8Nan || vb[2] == kKv8Nan || vb[3] == kKv8Nan;
  if (__ballot(bad)) {                         // a token that is NaN in K or V is so in both
    uint32_t tokens = uint32_t(__ballot(kb == kKv8Nan)) & 0xFFFFu;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint64_t b = __ballot(vb[i] == kKv8Nan);
#pragma unroll
      for (int q = 0; q < 4; ++q) tokens |= uint32_t(b >> (16 * q) & 1) << (4 * q + i);
    }
    if (tokens >> r & 1) kb = kKv8Nan;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (tokens >> (4 * a + i) & 1) vb[i] = kKv8Nan;
  }
#pragma unroll
  for (int j = 0; j < J; ++j) {
    uint4 q = round16(x[2 * j], x[2 * j + 1], kb);
    if (kb == kKv8Nan) q = make_uint4(kNanBytes, kNanBytes, kNanBytes, kNanBytes);
    store16(c.k + to + 1024 * j + 16 * lane, q);
    store16(c.v + to + 1024 * j + 16 * lane,
            make_uint4(round4_each(y[4 * j].x, y[4 * j].y, vb), round4_each(y[4 * j + 1].x, y[4 * j + 1].y, vb),
                       round4_each(y[4 * j + 2].x, y[4 * j + 2].y, vb), round4_each(y[4 * j + 3].x, y[4 * j + 3].y, vb)));
  }
  uint8_t* s = c.scale + (size_t(dst) * mv.hkv + at.g) * kKv8Scales;
  if (lane < 16) s[lane] = uint8_t(kb);
  if (r == 0) *reinterpret_cast<uint32_t*>(s + 16 + 4 * a) = vb[0] | vb[1] << 8 | vb[2] << 16 | uint32_t(vb[3]) << 24;
}

// Four e4m3 of a dword times their 2^(byte - 127), as bf16: exact, but for results outside bf16's
// range.  (In fp32: 2^-127 is no float to multiply by in bf16.)  Byte 255: `nan`.
__device__ __forceinline__ uint2 wide4(uint32_t w, int b0, int b1, int b2, int b3, float nan) {
  auto one = [&](float f, int b) {
    const float z = __builtin_amdgcn_ldexpf(f, b - 127);
    return b == kKv8Nan ? nan : z;
  };
  const float f0 = one(__builtin_amdgcn_cvt_f32_fp8(int(w), 0), b0), f1 = one(__builtin_amdgcn_cvt_f32_fp8(int(w), 1), b1);
  const float f2 = one(__builtin_amdgcn_cvt_f32_fp8(int(w), 2), b2), f3 = one(__builtin_amdgcn_cvt_f32_fp8(int(w), 3), b3);
  return make_uint2(pack_bf16x2(f0, f1), pack_bf16x2(f2, f3));
}

// A block's K and V, as a wavefront holds them, into block `block_head` of a bf16 cache; V of NaN tokens: nan_v.
template <int D>
__device__ __forceinline__ void store_wide(const uint4 (&x)[D / 64], const uint4 (&y)[D / 64], int kb, uint32_t vs, float nan_v,
                                           uint16_t* k, uint16_t* v, size_t block_head, int lane) {
  const int r = lane & 15, a = lane >> 4;
  const size_t to = block_head * 16 * D;
  const float scale = __uint_as_float(uint32_t(kb) << 23);
  constexpr uint32_t kNanPair = 0x7FC07FC0u;
#pragma unroll
  for (int j = 0; j < D / 64; ++j) {
    const uint32_t w[4] = {x[j].x, x[j].y, x[j].z, x[j].w}, u[4] = {y[j].x, y[j].y, y[j].z, y[j].w};
    uint2 q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      q[i] = make_uint2(e4m3_pair<false>(w[i], scale), e4m3_pair<true>(w[i], scale));
      if (kb == kKv8Nan) q[i] = make_uint2(kNanPair, kNanPair);
    }
    uint4* kp = reinterpret_cast<uint4*>(k + to + r * D + 64 * j + 16 * a);
    kp[0] = make_uint4(q[0].x, q[0].y, q[1].x, q[1].y);
    kp[1] = make_uint4(q[2].x, q[2].y, q[3].x, q[3].y);
#pragma unroll
    for (int t = 0; t < 4; ++t)
      *reinterpret_cast<uint2*>(v + to + (64 * j + 16 * t + r) * 16 + 4 * a) =
          wide4(u[t], vs & 255, vs >> 8 & 255, vs >> 16 & 255, vs >> 24, nan_v);
  }
}

// 8192 blocks of 8 heads of 128 (806 MB): 166 us, 4.9 TB/s, the rate of a large copy (176 with stores past the caches).
template <int D>
__global__ __launch_bounds__(kThreads) void kv8_unpack_kernel(Kv8Move mv, epic_kv8_cache c, uint16_t* __restrict__ k,
                                                              uint16_t* __restrict__ v) {
  const Place at(mv.n, mv.hkv, blockIdx.x);
  if (!at.in) return;
  const int src = mv.src ? mv.src[at.i] : at.i, dst = mv.dst ? mv.dst[at.i] : at.i;
  if (unsigned(src) >= unsigned(mv.src_blocks) || unsigned(dst) >= unsigned(mv.dst_blocks)) return;
  const int lane = threadIdx.x & 63;
  uint4 x[D / 64], y[D / 64];
  int kb;
  uint32_t vs;
  kv8_load_block<D>(c, size_t(src) * mv.hkv + at.g, lane, x, y, kb, vs);
  store_wide<D>(x, y, kb, vs, __uint_as_float(0x7FC00000u), k, v, size_t(dst) * mv.hkv + at.g, lane);
}

// The attention kernel of wide tiles reads a bf16 cache: block i of the list (null: block i of the pool) into block i of
// one, with K = NaN, V = 0 for NaN tokens (that kernel multiplies masked V by 0).  8208 blocks of 8 heads of 128 (809 MB):
// 137 us, 5.9 TB/s.
// JOINED: few private blocks (w) are written by the workgroups in front, and nothing waits for these: a private block is
// formed again here, from its source and its rows of S.  That saves a launch: up to 1024 (block, KV head) pairs a link
// step is 1 to 2 us shorter whether it writes 6 private blocks or 64; past them that is lost, the sooner the more private
// blocks there are, as every wavefront looks through them.  One request of 32 / 8 heads of 128, us joined (two launches):
//   pairs              128          512          768          1024         2048         3072           4128
//   few private blocks 20.5 (22.5)  26.0 (28.1)  28.9 (30.9)  31.4 (32.9)  40.7 (41.6)  51.8 (52.8)
//   32 private blocks               37.0 (38.5)  44.5 (44.9)  50.6 (51.6)  61.4 (61.5)  80.3 (79.3)    89.9 (88.2)
//   64 private blocks                                                      81.0 (80.5)  105.7 (104.9)  135.0 (131.1)
template <int D, bool JOINED>
__global__ __launch_bounds__(kThreads) void kv8_expand_kernel(const int32_t* __restrict__ list, int n, epic_kv8_cache c,
                                                              Kv8Rows w, int hkv, uint16_t* __restrict__ k,
                                                              uint16_t* __restrict__ v, int32_t* __restrict__ table) {
  __shared__ uint32_t turn[JOINED ? kWaves : 1][JOINED ? kTurnInts<D / 64> : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (JOINED && int(blockIdx.x) < w.groups) {
    const Place at(w.n, hkv, blockIdx.x);
    if (at.in) kv8_write_private<D>(w, c, at.i, hkv, at.g, lane, turn[wave]);
    return;
  }
  const Place at(n, hkv, blockIdx.x - (JOINED ? w.groups : 0));
  if (!at.in) return;
  const int phys = list ? list[at.i] : at.i;
  uint4 x[D / 64], y[D / 64];
  int kb, block = -1, block_src = 0;
  uint32_t vs;
  if constexpr (JOINED) {
    block = w.block[min(lane, w.n - 1)];
    block_src = w.src[min(lane, w.n - 1)];
  }
  kv8_load_block<D>(c, size_t(phys) * hkv + at.g, lane, x, y, kb, vs);
  if constexpr (JOINED) {
    const uint64_t mine = __ballot(lane < w.n && block == phys);
    if (mine != 0) {
      const int p = __builtin_ctzll(mine), src = __builtin_amdgcn_readlane(block_src, p);
      const int row = w.rows[p * 16 + (lane & 15)];
      if (src >= 0 && src != phys) kv8_load_block<D>(c, size_t(src) * hkv + at.g, lane, x, y, kb, vs);
      const Kv8Fresh<D / 64> f = kv8_fresh<D>(row, w.k_s, w.v_s, hkv, at.g, lane, turn[wave]);
      if (src < 0) kv8_no_block<D>(x, y, kb, vs);
      kv8_merge<D>(f, x, y, kb, vs, lane);
    }
  }
  store_wide<D>(x, y, kb, vs, 0.0f, k, v, size_t(at.i) * hkv + at.g, lane);
  if (table != nullptr && at.g == 0 && lane == 0) table[at.i] = at.i;
}

// The link write: every private block takes what its source block holds, then the rows of S,
// rounded to 8 bits, in their slots.  A slot that neither fills holds a row of zeros.
template <int D>
__global__ __launch_bounds__(kThreads) void kv8_write_kernel(Kv8Rows w, epic_kv8_cache c, int hkv) {
  __shared__ uint32_t turn[kWaves][kTurnInts<D / 64>];
  const Place at(w.n, hkv, blockIdx.x);
  if (at.in) kv8_write_private<D>(w, c, at.i, hkv, at.g, threadIdx.x & 63, turn[threadIdx.x >> 6]);
}

// The same for plans whose cached keys move: K of a block with priv_rot = off != 0 is turned by off
// (R(off) R(t) = R(off + t)): pairs (i, i + D / 2), angle off * theta^(-2 i / D) in float64, from its
// 8-bit values in fp32 to 8 bits again, with a scale of its own.
template <int D>
__global__ __launch_bounds__(kThreads) void kv8_write_rotate_kernel(Kv8Rows w, const int32_t* __restrict__ priv_rot,
                                                                    epic_kv8_cache c, int hkv, double log2_theta) {
  constexpr int J = D / 64;
  __shared__ uint32_t turn[kWaves][kTurnInts<J>];
  __shared__ float2 cs[D / 2];
  // a block's heads four by four: its wavefronts share the angles, and all meet at the barrier
  const int groups = (hkv + kWaves - 1) / kWaves, i = int(blockIdx.x) / groups;
  const int head = (int(blockIdx.x) % groups) * kWaves + __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int g = min(head, hkv - 1);
  const int lane = threadIdx.x & 63, a = lane >> 4;
  const int dst = w.block[i], src = w.src[i];
  const int rot = src >= 0 ? priv_rot[i] : 0;
  uint4 kq[J], vq[J];
  int kb;
  uint32_t vs;
  const int row = w.rows[i * 16 + (lane & 15)];
  kv8_load_block<D>(c, size_t(max(src, 0)) * hkv + g, lane, kq, vq, kb, vs);
  if (rot != 0) {                            // one block per workgroup: all of its wavefronts or none
    if (threadIdx.x < D / 2) {
      double sn, cn;
      sincos(double(rot) * exp2(-double(2 * int(threadIdx.x)) / double(D) * log2_theta), &sn, &cn);
      cs[threadIdx.x] = make_float2(float(cn), float(sn));
    }
    __syncthreads();
    float f[16 * J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint32_t w[4] = {kq[j].x, kq[j].y, kq[j].z, kq[j].w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[16 * j + 4 * i] = __builtin_amdgcn_cvt_f32_fp8(int(w[i]), 0);
        f[16 * j + 4 * i + 1] = __builtin_amdgcn_cvt_f32_fp8(int(w[i]), 1);
        f[16 * j + 4 * i + 2] = __builtin_amdgcn_cvt_f32_fp8(int(w[i]), 2);
        f[16 * j + 4 * i + 3] = __builtin_amdgcn_cvt_f32_fp8(int(w[i]), 3);
      }
    }
    // the values over their scale: turning commutes with it, and nothing overflows
    uint32_t top = 0;
    float z[16 * J];
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      if constexpr (J == 2) {                // dims 16 a + e and 64 more
        const float2 t = cs[16 * a + e];
        z[e] = f[e] * t.x - f[16 + e] * t.y;
        z[16 + e] = f[16 + e] * t.x + f[e] * t.y;
        top = max(top, max(finite_abs(z[e]), finite_abs(z[16 + e])));
      } else {                               // the partner is 32 dims, 32 lanes away
        const float2 t = cs[16 * (a & 1) + e];
        const float o = __shfl_xor(f[e], 32);
        z[e] = a < 2 ? f[e] * t.x - o * t.y : f[e] * t.x + o * t.y;
        top = max(top, finite_abs(z[e]));
      }
    }
    top = max(top, uint32_t(__shfl_xor(int(top), 16)));
    top = max(top, uint32_t(__shfl_xor(int(top), 32)));
    if (kb != kKv8Nan) {
      // z is over 2^(kb - 127), and so is its scale; rows of bf16 leave bytes far below 254
      const int byte = top == 0 ? 127 : min(max(scale_byte(top) + kb - 127, 0), kKv8Nan - 1), t = byte - kb + 127;
#pragma unroll
      for (int j = 0; j < J; ++j)
        kq[j] = make_uint4(pack_e4m3x4(z[16 * j], z[16 * j + 1], z[16 * j + 2], z[16 * j + 3], t),
                           pack_e4m3x4(z[16 * j + 4], z[16 * j + 5], z[16 * j + 6], z[16 * j + 7], t),
                           pack_e4m3x4(z[16 * j + 8], z[16 * j + 9], z[16 * j + 10], z[16 * j + 11], t),
                           pack_e4m3x4(z[16 * j + 12], z[16 * j + 13], z[16 * j + 14], z[16 * j + 15], t));
      kb = byte;
    }
  }
  const Kv8Fresh<J> f = kv8_fresh<D>(row, w.k_s, w.v_s, hkv, g, lane, turn[threadIdx.x >> 6]);
  if (src < 0) kv8_no_block<D>(kq, vq, kb, vs);
  kv8_merge<D>(f, kq, vq, kb, vs, lane);
  if (head < hkv) kv8_store_block<D>(kq, vq, kb, vs, c, size_t(dst) * hkv + g, lane);
}

unsigned grid_of(int n, int hkv) { return unsigned((int64_t(n) * hkv + kWaves - 1) / kWaves); }

}  // namespace

void launch_kv8_pack(const Kv8Move& mv, int head_dim, const uint16_t* k, const uint16_t* v, const epic_kv8_cache& c,
                     hipStream_t stream) {
  auto go = [&](auto kernel) { kernel<<<grid_of(mv.n, mv.hkv), kThreads, 0, stream>>>(mv, k, v, c); };
  if (head_dim == 128) go(kv8_pack_kernel<128>);
  else go(kv8_pack_kernel<64>);
}

void launch_kv8_unpack(const Kv8Move& mv, int head_dim, const epic_kv8_cache& c, uint16_t* k, uint16_t* v,
                       hipStream_t stream) {
  auto go = [&](auto kernel) { kernel<<<grid_of(mv.n, mv.hkv), kThreads, 0, stream>>>(mv, c, k, v); };
  if (head_dim == 128) go(kv8_unpack_kernel<128>);
  else go(kv8_unpack_kernel<64>);
}

void launch_kv8_expand(const int32_t* list, int n, int hkv, int head_dim, const epic_kv8_cache& c, const Kv8Rows& rows,
                       uint16_t* k, uint16_t* v, int32_t* table, hipStream_t stream) {
  Kv8Rows w = rows;
  w.groups = int(grid_of(w.n, hkv));
  auto go = [&](auto kernel) { kernel<<<w.groups + grid_of(n, hkv), kThreads, 0, stream>>>(list, n, c, w, hkv, k, v, table); };
  if (head_dim == 128) w.n > 0 ? go(kv8_expand_kernel<128, true>) : go(kv8_expand_kernel<128, false>);
  else w.n > 0 ? go(kv8_expand_kernel<64, true>) : go(kv8_expand_kernel<64, false>);
}

void launch_kv8_write(const Kv8Rows& w, const int32_t* priv_rot, int hkv, int head_dim, float rope_theta,
                      const epic_kv8_cache& c, hipStream_t stream) {
  if (w.n == 0) return;
  if (priv_rot != nullptr) {
    const dim3 grid(kv8_groups(w.n, hkv));
    const double l2t = std::log2(double(rope_theta));
    if (head_dim == 128) kv8_write_rotate_kernel<128><<<grid, kThreads, 0, stream>>>(w, priv_rot, c, hkv, l2t);
    else kv8_write_rotate_kernel<64><<<grid, kThreads, 0, stream>>>(w, priv_rot, c, hkv, l2t);
  } else {
    const dim3 grid(grid_of(w.n, hkv));
    if (head_dim == 128) kv8_write_kernel<128><<<grid, kThreads, 0, stream>>>(w, c, hkv);
    else kv8_write_kernel<64><<<grid, kThreads, 0, stream>>>(w, c, hkv);
  }
}

}  // namespace epic

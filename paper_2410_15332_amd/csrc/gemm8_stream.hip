// 8-bit GEMMs of short row sets: the weights streamed once, partial sums left in planes.
//
// What bounds it is reading W once, as in the bf16 kernel (gemm_stream.hip), whose deal
// this is: tiles of TM rows x TN columns, K in stages of 128 (a row's 128 bytes, one scale
// group), the tiles' stages dealt in G equal contiguous shares, a share's part of a tile
// to a plane of its own (stream_sum.h), LDS a ring of NS stages.
//
// Scales: a worker's are few (a byte per row and stage, and one per unit for the weight
// block, which a tile's columns never leave), so they go to LDS once, while the first
// stages are in flight.
//
// Stage layout: (TM + TN) rows of 128 bytes, A rows then W rows, in groups of 8 rows
// (1 KB, one load instruction); the eight 16-byte chunks of row r are XOR-swizzled by
// (r / 2) % 8, so the 16 lanes of each ds_read_b128 group touch distinct banks.
// Rows past M are read as row M - 1 and never stored.
#include <algorithm>

#include "gemm8.h"
#include "gemm8_device.h"
#include "quant.h"

namespace epic {

namespace {

constexpr int kBK = 128;
constexpr int kWorkers = 256;                           // one workgroup per CU
constexpr int kMinUnits = 4;                            // K stages per worker, at least

constexpr int kRowScales = 14336, kUnitScales = 2048;   // bytes of LDS for them: what the ring leaves

template <int TM, int TN, int NW, int CT, int NS>
__global__ __launch_bounds__(512, 1) void gemm8_stream_kernel(Gemm8Args g, StreamSum s) {
  constexpr int NG = (TM + TN) / 8;                     // 1 KB row groups per stage
  constexpr int NL = NG / NW;                           // ... per wavefront
  static_assert(NG % NW == 0, "row groups per wavefront");
  static_assert((TM / 32) * (TN / 32 / CT) == NW, "a wavefront per 32 rows x 32 CT columns");
  static_assert(TN <= 128, "one weight scale per unit");
  constexpr int SB = (TM + TN) * 128;                   // operand bytes per stage
  // One array: with several, the compiler sees that reads of the scales cannot be told from
  // the loads in flight to LDS, and has every stage wait for all of them.
  __shared__ __attribute__((aligned(1024))) char lds[NS * SB + kRowScales + kUnitScales];
  char* const row_scale = lds + NS * SB;                // [K stage][ld]
  char* const unit_scale = row_scale + kRowScales;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int w = blockIdx.x, G = s.G;
  const int wr = G % 8 == 0 ? (w % 8) * (G / 8) + w / 8 : w;   // XCD-contiguous worker index
  const int ks = s.ks, m_tiles = s.m_tiles;
  const int u0 = s.begin(wr), u1 = s.begin(wr + 1);
  if (u0 >= u1) return;
  constexpr int WC = TN / 32 / CT;                      // wavefronts along N
  const int rt = wv / WC, ct = wv % WC * CT;            // row block, first column block

  // ---- loads: row group gi of a stage, A rows first
  const int lrow = lane >> 3;
  __amdgpu_buffer_rsrc_t rs[NL];
  int vo[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const bool is_a = wv * NL + i < TM / 8;
    rs[i] = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(is_a ? g.A : g.W), 0, (is_a ? g.M : g.N) * g.K,
                                              kBufWord3);
  }
  const int ld = (g.M + 3) & ~3;
  auto setup = [&](int tile) __attribute__((always_inline)) {
    const int nt = tile / m_tiles, mt = tile - nt * m_tiles;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int gi = wv * NL + i;
      const bool is_a = gi < TM / 8;
      const int row = (is_a ? gi : gi - TM / 8) * 8 + lrow;
      const int gr = is_a ? min(mt * TM + row, g.M - 1) : nt * TN + row;
      vo[i] = gr * g.K + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
  };
  int du = u0, dtile = u0 / ks, dkt = u0 - dtile * ks;   // next unit to load
  setup(dtile);
  auto dma_next = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) dma16(rs[i], lds + buf * SB + (wv * NL + i) * 1024, vo[i], dkt * kBK);
    if (du + 1 < u1) {                                  // past the last unit: that one again
      ++du;
      if (++dkt == ks) {
        dkt = 0;
        setup(++dtile);
      }
    }
  };

  const int lbase = (lane & 31) * 128, lsw = (lane >> 1) & 7, half = lane >> 5;
  const int abase = rt * 4096 + lbase, bbase = (TM / 32 + ct) * 4096 + lbase;

#pragma unroll
  for (int b = 0; b < NS - 1; ++b) dma_next(b);
  {
    const int words = ld / 4, n = min(u1 - u0, ks) * words, k0 = (u0 % ks) * words, all = ks * words;
    for (int i = tid; i < n; i += NW * 64) {            // the K stages of this worker, at their places
      const int at = k0 + i < all ? k0 + i : k0 + i - all;
      reinterpret_cast<uint32_t*>(row_scale)[at] = reinterpret_cast<const uint32_t*>(g.sa)[at];
    }
    for (int i = tid; i < u1 - u0; i += NW * 64) {
      const int t = (u0 + i) / ks;
      unit_scale[i] = char(g.sw[size_t((t / m_tiles * TN) >> 7) * ks + (u0 + i - t * ks)]);
    }
  }
  int buf = 0, u = u0, tile = u0 / ks, kt = u0 - tile * ks, at = 0;   // kt, at: of the unit fetched next
  const int srow = min(rt * 32 + (lane & 31), g.M - 1);
  while (u < u1) {
    const int ue = min(u1, (tile + 1) * ks);
    f32x16 sums[2][CT];                                 // a chain of additions for each half of a stage
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int j = 0; j < CT; ++j) sums[i][j] = f32x16{};
    // unit u is read while unit u - 1 is on the matrix cores
    struct Frags {
      i32x8 a[2], b[2][CT];
      int sa, sb;
    } f0, f1;
    auto fetch = [&](Frags& f) __attribute__((always_inline)) {
      wait_vmem<(NS - 2) * NL>();                       // this wavefront's loads of unit u
      barrier_lds();                                    // everyone's; and unit u - 1 is read
      dma_next(buf == 0 ? NS - 1 : buf - 1);            // unit u + NS - 1, where u - 1 was
      const char* p = lds + buf * SB;
      f.sa = uint8_t(row_scale[kt * ld + srow]);
      f.sb = uint8_t(unit_scale[at++]);
      kt = kt + 1 == ks ? 0 : kt + 1;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c0 = ((4 * i + 2 * half) ^ lsw) * 16, c1 = c0 ^ 16;
        f.a[i] = read32(p + abase, c0, c1);
#pragma unroll
        for (int j = 0; j < CT; ++j) f.b[i][j] = read32(p + bbase + j * 4096, c0, c1);
      }
      buf = buf + 1 == NS ? 0 : buf + 1;
      __builtin_amdgcn_sched_barrier(0);
    };
    auto mma = [&](const Frags& f) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) sums[i][j] = mfma8<0, 0>(f.a[i], f.b[i][j], sums[i][j], f.sa, f.sb);
      __builtin_amdgcn_sched_barrier(0);
    };
    fetch(f0);
    for (++u; u + 1 < ue; u += 2) {
      fetch(f1);
      mma(f0);
      fetch(f0);
      mma(f1);
    }
    if (u < ue) {
      ++u;
      fetch(f1);
      mma(f0);
      mma(f1);
    } else {
      mma(f0);
    }
    // this worker's part of the tile: plane (worker - first worker of the tile)
    const int nt = tile / m_tiles, mt = tile - nt * m_tiles;
    const int plane = wr - s.owner(tile * ks);
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(
        g.partial + size_t(plane) * g.M * g.N, 0, g.M * g.N * 4, kBufWord3);   // rows past M: dropped
    const int m0 = mt * TM + rt * 32 + half * 4, n = nt * TN + ct * 32 + (lane & 31);
#pragma unroll
    for (int r = 0; r < 16; ++r)
#pragma unroll
      for (int j = 0; j < CT; ++j) {
        const float x = sums[0][j][r] + sums[1][j][r];
        __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), ro,
                                              ((m0 + (r >> 2) * 8 + (r & 3)) * g.N + n + j * 32) * 4, 0, 0);
      }
    ++tile;
  }
  wait_vmem<0>();                                       // no load may land in LDS after the workgroup ends
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

template <int TM, int TN, int NW, int CT, int NS>
StreamSum launch_tm(const Gemm8Args& g, hipStream_t stream) {
  StreamSum s{};
  s.partial = g.partial;
  s.M = g.M, s.N = g.N;
  s.tm = TM, s.tn = TN;
  s.m_tiles = cdiv(g.M, TM);
  s.ks = g.K / kBK;
  s.units = s.m_tiles * (g.N / TN) * s.ks;
  s.G = s.units < kWorkers * kMinUnits ? cdiv(s.units, kMinUnits) : kWorkers;
  gemm8_stream_kernel<TM, TN, NW, CT, NS><<<s.G, NW * 64, 0, stream>>>(g, s);
  return s;
}

}  // namespace

bool gemm8_stream_fits(int M, int N, int K) {
  const int tm = M <= 32 ? 32 : M <= 64 ? 64 : 128;
  const int64_t units = int64_t(cdiv(M, tm)) * (N / 64) * (K / kBK);
  if (units >= (1 << 23)) return false;                 // 32-bit arithmetic of StreamSum::owner
  const int64_t per = std::max<int64_t>(units / kWorkers, 1);
  const int64_t planes = (K / kBK + per - 1) / per + 1;
  if (M > 128 || K / kBK * ((M + 3) / 4 * 4) > kRowScales || units / kWorkers + 1 > kUnitScales) return false;
  return planes * M * N * 4 <= int64_t(kPartial8Bytes);
}

StreamSum launch_gemm8_stream(const Gemm8Args& g, hipStream_t stream) {
  if (g.M <= 32) return launch_tm<32, 64, 2, 1, 11>(g, stream);
  if (g.M <= 64) return launch_tm<64, 64, 4, 1, 9>(g, stream);
  return launch_tm<128, 64, 8, 1, 6>(g, stream);
}

}  // namespace epic

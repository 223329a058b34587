// 8-bit GEMMs of short row sets: the weights streamed once, partial sums left in planes; and
// small whole tiles, a workgroup each, for row sets between those and the 256-column tiles.
//
// What bounds the first is reading W once, as in the bf16 kernel (gemm_stream.hip), whose deal
// this is: tiles of TM rows x TN columns, K in stages of 128 (a row's 128 bytes, one scale
// group), the tiles' stages dealt in G equal contiguous shares, a share's part of a tile
// to a plane of its own (stream_sum.h), LDS a ring of NS stages.  32 rows, N 4096, K 14 336:
// 14.2 us (59 MB, 4.2 TB/s) and 1.9 to add the planes.
//
// Whole tiles have no second launch.  What bounds them is mostly what a CU can load: one
// tile alone takes 0.18, 0.29 and 0.44 us a stage for the 16, 24 and 32 KB of 64 x 64, 64 x 128
// and 128 x 128 (91 to 74 GB/s, where loads alone of this shape reach 100), and a third less read from
// LDS per product changes nothing.  So larger
// tiles cost less per product, and smaller ones use more CUs.  501 rows, N = K = 4096: 64 x 64
// tiles 22.9 us, 64 x 128 16.4, 128 x 128 21.2, 256-column tiles 22 at best.  SwiGLU of 100 rows,
// N 28 672, K 4096: 128 x 128 29 us (121 MB, 4.1 TB/s), 64 x 128 37, planes 41; to e4m3, where
// a tile has to have whole groups, 64 x 256 34, planes 42.  Two wavefronts share a place
// (KS = 2) where a tile has few: 64 x 64 tiles of 256 rows 13.3 us then, 14.9 without.
//
// Scales: a worker's are few (a byte per row and stage, and one per unit for the weight
// block, which a tile's columns never leave), so they go to LDS once: while the first
// stages are in flight, or, of whole tiles, in front of them (256 rows, N = K = 4096 12.6 -> 12.1 us).
//
// Stage layout: (TM + TN) rows of 128 bytes, A rows then W rows, in groups of 8 rows
// (1 KB, one load instruction); the eight 16-byte chunks of row r are XOR-swizzled by
// (r / 2) % 8, so the 16 lanes of each ds_read_b128 group touch distinct banks.
// Rows past M are read as row M - 1 and never stored.
#include <algorithm>
#include <type_traits>

#include "gemm8.h"
#include "gemm8_device.h"
#include "quant.h"
#include "quant_device.h"

namespace epic {

namespace {

constexpr int kBK = 128;
constexpr int kWorkers = 256;                           // one workgroup per CU
constexpr int kMinUnits = 4;                            // K stages per worker, at least

constexpr int kRowScales = 14336, kUnitScales = 2048;   // bytes of LDS for them: what the ring leaves

// A wavefront has 32 RT rows x 32 CT columns of a tile.  OUT: kPlanesOut, or kBf16Out, kGluOut or
// kGluQuantOut for whole tiles: worker w has tile w, and stores its result itself (GLU: the
// tile's columns are gate and up in turn, 32 each).
constexpr int kPlanesOut = 4;
// KS = 2: two wavefronts share a place, each with half of every stage.
template <int OUT, int TM, int TN, int RT, int CT, int KS, int NS>
__global__ __launch_bounds__(512, 1) void gemm8_stream_kernel(Gemm8Args g, StreamSum s) {
  constexpr bool WHOLE = OUT != kPlanesOut, GLU = OUT == kGluOut || OUT == kGluQuantOut;
  constexpr int NW = (TM / 32 / RT) * (TN / 32 / CT) * KS;
  constexpr int NG = (TM + TN) / 8;                     // 1 KB row groups per stage
  constexpr int NL = NG / NW;                           // ... per wavefront
  static_assert(NG % NW == 0, "row groups per wavefront");
  static_assert(!GLU || CT == 2, "a wavefront holds the gate and up of its columns");
  static_assert(TN <= (GLU ? 256 : 128), "one weight scale per unit (GLU: two)");
  static_assert(!WHOLE || NW * 64 >= kRowScales / TM, "a thread loads one of a whole tile's");
  static_assert(OUT != kGluQuantOut || (TN == 256 && TM * 32 % (NW * 64) == 0), "a tile has whole groups of the result");
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
  const int place = wv / KS, kh = wv % KS;
  const int rt = place / WC * RT, ct = place % WC * CT;   // first row block, first column block
  const int ffn = g.N / 2;

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
      int gr = is_a ? min(mt * TM + row, g.M - 1) : nt * TN + row;
      if (GLU && !is_a) gr = ((row >> 5) & 1) * ffn + nt * (TN / 2) + (row >> 6) * 32 + (row & 31);
      vo[i] = gr * g.K + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
  };
  // Whole tiles: each XCD's start at a K stage of their own.  Rows a multiple of 4 KB apart have
  // one stage on the same few memory channels, which all would ask for at once: 256 rows,
  // N = K = 4096 15.8 -> 15.1 us, SwiGLU of 100 rows, N 28 672 31.3 -> 29.2, K = 5120 1% less.
  const int rot = WHOLE ? w % 8 * ks / 8 : 0;
  int du = u0, dtile = u0 / ks, dkt = WHOLE ? rot : u0 - dtile * ks;   // next unit to load
  setup(dtile);
  auto dma_next = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NL; ++i) dma16(rs[i], lds + buf * SB + (wv * NL + i) * 1024, vo[i], dkt * kBK);
    if (du + 1 < u1) {                                  // past the last unit: that one again
      ++du;
      if (++dkt == ks) {
        dkt = 0;
        if (!WHOLE) setup(++dtile);
      }
    }
  };

  const int lbase = (lane & 31) * 128, lsw = (lane >> 1) & 7, half = lane >> 5;
  const int abase = rt * 4096 + lbase, bbase = (TM / 32 + ct) * 4096 + lbase;

  // Whole tiles load their scales in front of the operands, so that the first stage waits for
  // nothing behind it: all of the tile's rows', at the stage's place, and the blocks'.
  uint8_t block = 0, up = 0;
  if constexpr (WHOLE) {
    const __amdgpu_buffer_rsrc_t rsc =
        __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.sa), 0, ks * ld, kBufWord3);
    const int words = min(ld, TM) / 4, n = ks * words, m0 = dtile % m_tiles * TM, col = dtile / m_tiles * TN / (GLU ? 2 : 1);
    for (int i = wv * 64; i < n; i += NW * 64) {
      const int at = min(i + lane, n - 1), k = at / words;
      dma4(rsc, row_scale + i * 4, k * ld + min(m0 + (at - k * words) * 4, ld - 4), 0);
    }
    const int k = min(tid, ks - 1);
    block = g.sw[size_t(col >> 7) * ks + k];
    if (GLU) up = g.sw[size_t((ffn + col) >> 7) * ks + k];
  }
#pragma unroll
  for (int b = 0; b < NS - 1; ++b) dma_next(b);
  if constexpr (WHOLE) {
    if (tid < ks) {
      unit_scale[tid] = char(block);
      if (GLU) unit_scale[tid + ks] = char(up);
    }
  } else {
    // a stage's scales of all rows (M <= 128), at the stage's place
    const int words = ld / 4, all = ks * words;
    const int n = min(u1 - u0, ks) * words, k0 = (u0 % ks) * words;
    for (int i = tid; i < n; i += NW * 64) {
      const int at = k0 + i < all ? k0 + i : k0 + i - all;
      reinterpret_cast<uint32_t*>(row_scale)[at] = reinterpret_cast<const uint32_t*>(g.sa)[at];
    }
    for (int i = tid; i < u1 - u0; i += NW * 64) {
      const int t = (u0 + i) / ks, k = u0 + i - t * ks;
      unit_scale[i] = char(g.sw[size_t(t / m_tiles * TN >> 7) * ks + k]);
    }
  }
  int buf = 0, u = u0, tile = u0 / ks;
  int kt = WHOLE ? rot : u0 - tile * ks, at = WHOLE ? rot : 0;   // of the unit fetched next
  const int swords = min(ld, TM);
  int srow[RT];
#pragma unroll
  for (int r = 0; r < RT; ++r) srow[r] = min((rt + r) * 32 + (lane & 31), swords - 1);
  while (u < u1) {
    const int ue = min(u1, (tile + 1) * ks);
    // a chain of additions for each half of a stage where a wavefront has one tile
    constexpr int NA = RT * CT * KS == 1 ? 2 : 1;
    constexpr int NH = 2 / KS;                          // halves of a stage per wavefront
    f32x16 sums[NA][RT][CT];
#pragma unroll
    for (int i = 0; i < NA; ++i)
#pragma unroll
      for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int j = 0; j < CT; ++j) sums[i][r][j] = f32x16{};
    // unit u is read while unit u - 1 is on the matrix cores
    struct Frags {
      i32x8 a[NH][RT], b[NH][CT];
      int sa[RT], sb[GLU ? 2 : 1];
    } f0, f1;
    auto fetch = [&](Frags& f) __attribute__((always_inline)) {
      wait_vmem<(NS - 2) * NL>();                       // this wavefront's loads of unit u
      barrier_lds();                                    // everyone's; and unit u - 1 is read
      dma_next(buf == 0 ? NS - 1 : buf - 1);            // unit u + NS - 1, where u - 1 was
      const char* p = lds + buf * SB;
#pragma unroll
      for (int r = 0; r < RT; ++r) f.sa[r] = uint8_t(row_scale[kt * swords + srow[r]]);
      f.sb[0] = uint8_t(unit_scale[at]);
      if (GLU) f.sb[GLU] = uint8_t(unit_scale[at + ks]);
      kt = kt + 1 == ks ? 0 : kt + 1;
      at = WHOLE ? kt : at + 1;
#pragma unroll
      for (int i = 0; i < NH; ++i) {
        const int c0 = ((4 * (KS == 2 ? kh : i) + 2 * half) ^ lsw) * 16, c1 = c0 ^ 16;
#pragma unroll
        for (int r = 0; r < RT; ++r) f.a[i][r] = read32(p + abase + r * 4096, c0, c1);
#pragma unroll
        for (int j = 0; j < CT; ++j) f.b[i][j] = read32(p + bbase + j * 4096, c0, c1);
      }
      buf = buf + 1 == NS ? 0 : buf + 1;
      __builtin_amdgcn_sched_barrier(0);
    };
    auto mma = [&](const Frags& f) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < NH; ++i)
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int j = 0; j < CT; ++j)
            sums[i % NA][r][j] = mfma8<0, 0>(f.a[i][r], f.b[i][j], sums[i % NA][r][j], f.sa[r], f.sb[GLU ? j : 0]);
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
    const int nt = tile / m_tiles, mt = tile - nt * m_tiles;
    if constexpr (WHOLE) {
      // through LDS, so that a row's columns are written in runs (and, quantised, meet)
      typedef std::conditional_t<OUT == kGluQuantOut, float, uint16_t> Value;
      constexpr int COLS = GLU ? TN / 2 : TN, LDO = COLS + 16 / int(sizeof(Value));
      static_assert(TM * LDO * sizeof(Value) <= NS * SB, "the tile fits the ring");
      wait_vmem<0>();                                   // loads past the end land first
      barrier_lds();
      Value* room = reinterpret_cast<Value*>(lds);
      typedef Border<NW, NW * 2> List;                  // kGluQuantOut: one for each pass over the tile's groups
      constexpr int LISTS = (TM * LDO * int(sizeof(Value)) + 1023) / 1024 * 1024, PASSES = TM * 32 / (NW * 64);
      static_assert(OUT != kGluQuantOut || LISTS + PASSES * int(sizeof(List)) <= NS * SB, "the lists fit beside the tile");
      List* lists = reinterpret_cast<List*>(lds + LISTS);
      if (OUT == kGluQuantOut && tid < PASSES) lists[tid].count = 0;
      if constexpr (KS == 2) {                          // the two halves meet
        constexpr int ROOM = (TM * LDO * int(sizeof(Value)) + 1023) / 1024 * 1024;
        static_assert(ROOM + TM * TN * 4 <= NS * SB, "the sums fit beside the tile");
        float* sum = reinterpret_cast<float*>(lds + ROOM) + place * RT * CT * 1024 + lane;
#pragma unroll
        for (int x = 0; x < RT * CT * 16; ++x)
          if (kh == 1) sum[x * 64] = sums[0][x / 16 / CT][x / 16 % CT][x % 16];
        barrier_lds();
#pragma unroll
        for (int x = 0; x < RT * CT * 16; ++x)
          if (kh == 0) sums[0][x / 16 / CT][x / 16 % CT][x % 16] += sum[x * 64];
      }
      if (kh == 0) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
          for (int j = 0; j < CT; j += GLU ? 2 : 1)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              float x = sums[0][r][j][e];
              if constexpr (NA == 2) x += sums[1][r][j][e];
              if constexpr (GLU) x = silu(x) * sums[0][r][j + 1][e];
              const int row = (rt + r) * 32 + half * 4 + (e >> 2) * 8 + (e & 3);
              const int col = (GLU ? ct / 2 + j / 2 : ct + j) * 32 + (lane & 31);
              if constexpr (OUT == kGluQuantOut) room[row * LDO + col] = x;
              else room[row * LDO + col] = uint16_t(pack_bf16x2(x, 0.0f));
            }
      }
      barrier_lds();
      const int cols = GLU ? ffn : g.N;
      if constexpr (OUT == kGluQuantOut) {              // 32 lanes a row, one group
        for (int i = tid; i < TM * 32; i += NW * 64) {
          const int row = i >> 5, c = (i & 31) * 4, m = mt * TM + row;
          const float4 v = *reinterpret_cast<const float4*>(room + row * LDO + c);
          const uint32_t top = half_max(max(max(finite_abs(v.x), finite_abs(v.y)), max(finite_abs(v.z), finite_abs(v.w))));
          const int byte = group_byte(lists[i / (NW * 64)], g, top, v, m, nt * COLS + c, m < g.M);
          if (m < g.M) {
            *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(g.out) + size_t(m) * cols + nt * COLS + c) =
                pack_e4m3x4(v.x, v.y, v.z, v.w, byte);
            if (c == 0) g.out_scale[size_t(nt) * ld + m] = uint8_t(byte);
          }
        }
      } else {
        constexpr int LR = COLS / 8;                    // lanes a row
        for (int i = tid; i < TM * LR; i += NW * 64) {
          const int row = i / LR, c = i % LR * 8, m = mt * TM + row;
          if (m < g.M)
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(g.out) + size_t(m) * cols + nt * COLS + c) =
                *reinterpret_cast<const uint4*>(room + row * LDO + c);
        }
      }
      return;
    }
    // this worker's part of the tile: plane (worker - first worker of the tile)
    const int plane = wr - s.owner(tile * ks);
    const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(
        g.partial + size_t(plane) * g.M * g.N, 0, g.M * g.N * 4, kBufWord3);   // rows past M: dropped
    const int n = nt * TN + ct * 32 + (lane & 31);
#pragma unroll
    for (int q = 0; q < RT; ++q) {
      const int m0 = mt * TM + (rt + q) * 32 + half * 4;
#pragma unroll
      for (int r = 0; r < 16; ++r)
#pragma unroll
        for (int j = 0; j < CT; ++j) {
          float x = sums[0][q][j][r];
          if constexpr (NA == 2) x += sums[1][q][j][r];
          __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x), ro,
                                                ((m0 + (r >> 2) * 8 + (r & 3)) * g.N + n + j * 32) * 4, 0, 0);
        }
    }
    ++tile;
  }
  wait_vmem<0>();                                       // no load may land in LDS after the workgroup ends
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

constexpr int kStreamTN = 64;                           // columns of a streamed tile
int stream_tm(int M) { return M <= 32 ? 32 : M <= 64 ? 64 : 128; }   // ... and its rows

template <int TM, int NS>
void launch_stream_tm(const Gemm8Args& g, const StreamSum& s, hipStream_t stream) {
  gemm8_stream_kernel<kPlanesOut, TM, kStreamTN, 1, 1, 1, NS><<<s.G, (TM / 32) * (kStreamTN / 32) * 64, 0, stream>>>(g, s);
}

template <int OUT, int TM, int TN, int RT, int CT, int KS, int NS>
void launch_whole(const Gemm8Args& g, hipStream_t stream) {
  StreamSum s{};
  s.M = g.M, s.N = g.N;
  s.tm = TM, s.tn = TN;
  s.m_tiles = cdiv(g.M, TM);
  s.ks = g.K / kBK;
  s.G = s.m_tiles * cdiv(g.N, TN);
  s.units = s.G * s.ks;
  gemm8_stream_kernel<OUT, TM, TN, RT, CT, KS, NS><<<s.G, (TM / 32 / RT) * (TN / 32 / CT) * KS * 64, 0, stream>>>(g, s);
}

}  // namespace

bool gemm8_stream_fits(int M, int N, int K) {
  const int64_t units = int64_t(cdiv(M, stream_tm(M))) * (N / kStreamTN) * (K / kBK);
  if (units >= (1 << 23)) return false;                 // 32-bit arithmetic of StreamSum::owner
  const int64_t per = std::max<int64_t>(units / kWorkers, 1);
  const int64_t planes = (K / kBK + per - 1) / per + 1;
  if (M > 128 || K / kBK * ((M + 3) / 4 * 4) > kRowScales || units / kWorkers + 1 > kUnitScales) return false;
  return planes * M * N * 4 <= int64_t(kPartial8Bytes);
}

// Whole tiles of tm x tn, a workgroup each: what LDS has left holds the scales of so many stages.
bool gemm8_narrow_fits(int N, int K, int epi, int tm, int tn) {
  const int ks = K / kBK;
  if (epi == kGluQuantOut ? tm != 64 || tn != 256 : tn > 128) return false;
  return epi != kRopeOut && N % tn == 0 && ks * tm <= kRowScales && 2 * ks <= kUnitScales;
}

void launch_gemm8_narrow(const Gemm8Args& g, int epi, int tm, int tn, hipStream_t stream) {
  if (epi == kGluQuantOut) {
    launch_whole<kGluQuantOut, 64, 256, 1, 2, 1, 3>(g, stream);
  } else if (epi == kGluOut) {
    if (tm == 64 && tn == 64) launch_whole<kGluOut, 64, 64, 1, 2, 2, 9>(g, stream);
    else if (tm == 64) launch_whole<kGluOut, 64, 128, 1, 2, 2, 6>(g, stream);
    else launch_whole<kGluOut, 128, 128, 1, 2, 1, 4>(g, stream);
  } else {
    if (tm == 64 && tn == 64) launch_whole<kBf16Out, 64, 64, 1, 1, 2, 9>(g, stream);
    else if (tm == 64) launch_whole<kBf16Out, 64, 128, 1, 1, 1, 6>(g, stream);
    else launch_whole<kBf16Out, 128, 128, 1, 2, 1, 4>(g, stream);
  }
}

StreamSum gemm8_stream_sum(int M, int N, int K) {
  StreamSum s{};
  s.M = M, s.N = N;
  s.tm = stream_tm(M), s.tn = kStreamTN;
  s.m_tiles = cdiv(M, s.tm);
  s.ks = K / kBK;
  s.units = s.m_tiles * (N / s.tn) * s.ks;
  s.G = s.units < kWorkers * kMinUnits ? cdiv(s.units, kMinUnits) : kWorkers;
  return s;
}

StreamSum launch_gemm8_stream(const Gemm8Args& g, hipStream_t stream) {
  StreamSum s = gemm8_stream_sum(g.M, g.N, g.K);
  s.partial = g.partial;
  if (s.tm == 32) launch_stream_tm<32, 11>(g, s, stream);
  else if (s.tm == 64) launch_stream_tm<64, 9>(g, s, stream);
  else launch_stream_tm<128, 6>(g, s, stream);
  return s;
}

}  // namespace epic

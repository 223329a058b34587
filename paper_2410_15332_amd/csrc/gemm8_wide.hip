// 8-bit GEMMs of more rows: C[M x N] = A[M x K] . W[N x K]^T on tiles of 256, 192 or 128 rows x
// 256 columns, one workgroup of four wavefronts per CU, epilogues fused.
//
// A stage is 128 of K, which are 128 bytes of a row, as 64 of K are in the bf16 kernel
// (gemm_wide.hip), and the matrix cores take it in the same time with twice the products.
// So the schedule is that kernel's: a wavefront owns TM/2 x 128 outputs in AGPRs, the
// fragments of the next half stage are read and the loads of later stages issued between
// the MFMAs of this one, and LDS is a ring of five half stages (one operand, 128 of K,
// 32 KB each), of which a stage frees two: they take the A half of the stage after next
// and the W half of the one after that: W comes from memory, most of A from the caches (the
// other way round: 736 rows, N 27 648, K 5120 121 us, 114.6 now; 200 rows of 28 672 x 4096 43.2,
// 40.6; 20 560 rows the same).
//
// What bounds it: many tiles run at the chip's power limit.  SwiGLU of 20 560 rows, N 28 672,
// K 4096 to e4m3, 256-row tiles: 1.82-1.93 ms, 2.50-2.66 PFLOP/s, at 1.75 GHz with the
// matrix cores busy for 68% of the cycles (a large library product without the epilogue: 2.97).
// Few tiles wait for memory: 736 rows, 192-row tiles, two each on 224 CUs: 84-89 us, 2.1 GHz,
// busy for 44%, 19% of the wavefronts' time waiting.
// Tile heights, the same two, before W had the longer way: 736 rows 107 us (128), 89 (192), 93 (256);
// 20 560 rows 2109, 1984, 1887.
//
// Scales: one per row and stage, applied by the matrix instruction.  A wavefront's rows
// are dealt to its I row tiles in turn (tile i has rows I r + i), so the I scales of a
// lane are neighbouring bytes of one load, and the instruction picks byte i.  The scale of
// the columns' weight block is one byte per wavefront and stage (SwiGLU: of the gate's
// and of the up block).  They are loaded into registers two stages ahead.
//
// With few tiles the same kernel runs equal parts of K of every tile, one workgroup each,
// into fp32 planes that the consumer adds (stream_sum.h): 736 rows, N 4096, K 14 336, 192-row
// tiles in four parts 54 us with the pass that adds them, whole 96.
//
// Half-stage layout: rows of 128 bytes in groups of 8 (1 KB, one load instruction); the
// eight 16-byte chunks of row r are XOR-swizzled by (r / 2) % 8, so the 16 lanes of each
// ds_read_b128 group touch distinct banks.  For SwiGLU the W rows of a tile are gate and
// up in turn, 32 rows each.  Rows past M and columns past N are read clamped and never
// stored.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "gemm8.h"
#include "gemm8_device.h"
#include "quant.h"
#include "quant_device.h"

namespace epic {

namespace {

constexpr int kBK = 128, kTN = 256;
constexpr int kMaxWorkers = 256;
constexpr int kPlanesOut = 4;  // epilogue: fp32 partial sums into planes

struct WidePlan8 {
  int m_tiles, n_tiles, tiles;
  int ks;                      // K stages per tile
  int gm;                      // row tiles per ordering group
  int G;                       // workgroups, a multiple of 8
  int parts;                   // kPlanesOut: equal parts of K per tile, a workgroup each
};

template <class F, int... M>
__device__ __forceinline__ void for_each_index(const F& f, std::integer_sequence<int, M...>) {
  (f(std::integral_constant<int, M>{}), ...);
}

template <int EPI, int TM>
__global__ __launch_bounds__(256, 1) void gemm8_wide_kernel(Gemm8Args g, WidePlan8 p) {
  constexpr int I = TM / 64, J = 4;                     // 32 x 32 MFMA tiles per wavefront
  constexpr int NLA = TM / 32, NLB = kTN / 32;          // 1 KB row groups per wavefront and stage
  constexpr int SLOTS = 5, SLOT = kTN * 128;            // half stages (one operand, 128 of K)
  constexpr bool SPLIT = EPI == kPlanesOut;
  constexpr bool GLU = EPI == kGluOut || EPI == kGluQuantOut;
  __shared__ __attribute__((aligned(1024))) char lds[SLOTS][SLOT];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wv = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wv >> 1, wn = wv & 1;
  const int w = blockIdx.x;
  const int wr = (w % 8) * (p.G / 8) + w / 8;           // XCD-contiguous worker index (G % 8 == 0)
  // This worker's K stages: whole tiles wr, wr + G, ..; with planes part wr / tiles of
  // tile wr % tiles, so that the workgroups of an XCD are at the same K.
  if (wr >= (SPLIT ? p.parts * p.tiles : p.tiles)) return;
  const int part = SPLIT ? wr / p.tiles : 0;
  const int tile0 = SPLIT ? wr - part * p.tiles : wr;
  const int kt0 = SPLIT ? part * p.ks / p.parts : 0;
  const int n_units = SPLIT ? (part + 1) * p.ks / p.parts - kt0 : (p.tiles - wr + p.G - 1) / p.G * p.ks;

  auto tile_mn = [&](int t, int& mt, int& nt) __attribute__((always_inline)) {
    if constexpr (SPLIT) {
      nt = t / p.m_tiles;
      mt = t - nt * p.m_tiles;
      return;
    }
    const int per_group = p.gm * p.n_tiles;
    const int grp = t / per_group;
    const int first = grp * p.gm;
    const int gsz = min(p.m_tiles - first, p.gm);
    const int r = t - grp * per_group;
    mt = first + r % gsz;
    nt = r / gsz;
  };

  // ---- loads: this wavefront stages A row groups NLA wv .., W row groups NLB wv ..
  const int lrow = lane >> 3;
  const int ffn = g.N / 2, ld = (g.M + 3) & ~3;
  const __amdgpu_buffer_rsrc_t rsa =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.A), 0, g.M * g.K, kBufWord3);
  const __amdgpu_buffer_rsrc_t rsb =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.W), 0, g.N * g.K, kBufWord3);
  const __amdgpu_buffer_rsrc_t rsc =                    // scales; past the end (rows past M only) they read as 0
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.sa), 0, p.ks * ld, kBufWord3);
  const __amdgpu_buffer_rsrc_t rsd =
      __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.sw), 0, (g.N >> 7) * p.ks, kBufWord3);
  int va[NLA], vb[NLB], vsa, vsw, vsu;
  struct Cursor {
    int tile, kt, slot, left;
  };
  // next half stages (ca, cb) and scales (cs) to load
  Cursor ca{tile0, kt0, 1, n_units}, cb{tile0, kt0, 0, n_units}, cs{tile0, kt0, 0, n_units};
  auto setup_a = [&]() __attribute__((always_inline)) {
    int mt, nt;
    tile_mn(ca.tile, mt, nt);
#pragma unroll
    for (int i = 0; i < NLA; ++i) {
      const int row = (NLA * wv + i) * 8 + lrow;        // in LDS: row tile after row tile of a wavefront's
      const int in = row % (TM / 2), gr = row - in + in % 32 * I + in / 32;
      va[i] = min(mt * TM + gr, g.M - 1) * g.K + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
  };
  // the column of a wavefront's 128 that column tile r / 32 has at r % 32: kRopeOut with heads of
  // 128 takes the two halves of rotary pairs in turn, as heads of 64 have them anyway
  const bool halves = EPI == kRopeOut && g.head_dim == 128;
  auto column = [&](int r) __attribute__((always_inline)) {
    return halves ? ((r >> 5) & 1) * 64 + ((r >> 6) & 1) * 32 + (r & 31) : r;
  };
  auto setup_b = [&]() __attribute__((always_inline)) {
    int mt, nt;
    tile_mn(cb.tile, mt, nt);
#pragma unroll
    for (int i = 0; i < NLB; ++i) {
      const int row = (NLB * wv + i) * 8 + lrow;
      int gr;
      if constexpr (GLU) gr = ((row >> 5) & 1) * ffn + nt * (kTN / 2) + (row >> 6) * 32 + (row & 31);
      else gr = min(nt * kTN + (row & ~127) + column(row & 127), g.N - 1);
      vb[i] = gr * g.K + ((lane & 7) ^ ((row >> 1) & 7)) * 16;
    }
  };
  auto setup_s = [&]() __attribute__((always_inline)) {
    int mt, nt;
    tile_mn(cs.tile, mt, nt);
    vsa = mt * TM + wm * (TM / 2) + (lane & 31) * I;
    const int nb = GLU ? nt : min(nt * 2 + wn, (g.N >> 7) - 1);
    vsw = nb * p.ks;
    vsu = (nb + (ffn >> 7)) * p.ks;
  };
  setup_a();
  setup_b();
  setup_s();
  auto bump = [&](int slot) __attribute__((always_inline)) { return slot >= SLOTS - 2 ? slot + 2 - SLOTS : slot + 2; };
  // to the next half stage; past the last, that one again.  True: another tile
  auto advance = [&](Cursor& c) __attribute__((always_inline)) {
    c.slot = bump(c.slot);
    if (--c.left <= 0) return false;
    if (++c.kt < p.ks) return false;
    c.tile += p.G;
    c.kt = 0;
    return true;
  };
  auto dma_a = [&](int i) __attribute__((always_inline)) {
    dma16(rsa, lds[ca.slot] + (NLA * wv + i) * 1024, va[i], ca.kt * kBK);
    if (i == NLA - 1 && advance(ca)) setup_a();
  };
  auto dma_b = [&](int i) __attribute__((always_inline)) {
    dma16(rsb, lds[cb.slot] + (NLB * wv + i) * 1024, vb[i], cb.kt * kBK);
    if (i == NLB - 1 && advance(cb)) setup_b();
  };
  struct Scales {
    int a, w, u;                                        // I rows of a lane; the columns' block (gate, up)
  } sc0, sc1;                                           // of this stage and the next
  // the last ones loaded, in the types loaded: widened here, they would be waited for here
  struct Loaded {
    std::conditional_t<I == 4, uint32_t, uint16_t> a;
    uint8_t a1, a2;                                     // I == 3
    uint8_t w, u;
  } sc2;
  auto load_scales = [&](Loaded& s) __attribute__((always_inline)) {
    if constexpr (I == 4) {
      s.a = __builtin_amdgcn_raw_buffer_load_b32(rsc, vsa, cs.kt * ld, 0);
    } else if constexpr (I == 2) {
      s.a = __builtin_amdgcn_raw_buffer_load_b16(rsc, vsa, cs.kt * ld, 0);
    } else {                                            // any alignment: three bytes
      s.a = __builtin_amdgcn_raw_buffer_load_b8(rsc, vsa, cs.kt * ld, 0);
      s.a1 = __builtin_amdgcn_raw_buffer_load_b8(rsc, vsa + 1, cs.kt * ld, 0);
      s.a2 = __builtin_amdgcn_raw_buffer_load_b8(rsc, vsa + 2, cs.kt * ld, 0);
    }
    s.w = __builtin_amdgcn_raw_buffer_load_b8(rsd, vsw, cs.kt, 0);
    if constexpr (GLU) s.u = __builtin_amdgcn_raw_buffer_load_b8(rsd, vsu, cs.kt, 0);
    if (advance(cs)) setup_s();
  };
  // after sync(), where the loads have landed: left to the compiler, the copies move in
  // front of the next stage's sync() and wait for them
  auto take = [&](Scales& to, const Loaded& from) __attribute__((always_inline)) {
    __asm__ volatile("v_mov_b32 %0, %1" : "=v"(to.a) : "v"(int(from.a)));
    if constexpr (I == 3) {
      __asm__ volatile("v_lshl_or_b32 %0, %1, 8, %0" : "+v"(to.a) : "v"(int(from.a1)));
      __asm__ volatile("v_lshl_or_b32 %0, %1, 16, %0" : "+v"(to.a) : "v"(int(from.a2)));
    }
    __asm__ volatile("v_mov_b32 %0, %1" : "=v"(to.w) : "v"(int(from.w)));
    if constexpr (GLU) __asm__ volatile("v_mov_b32 %0, %1" : "=v"(to.u) : "v"(int(from.u)));
  };

  // ---- fragments
  const int half = lane >> 5, lsw = (lane >> 1) & 7;
  const int la = wm * (TM / 2) * 128 + (lane & 31) * 128;
  const int lb = wn * 128 * 128 + (lane & 31) * 128;
  int sw[2];
#pragma unroll
  for (int s = 0; s < 2; ++s) sw[s] = ((4 * s + 2 * half) ^ lsw) * 16;
  struct Frags {
    i32x8 a[I], b[J];
  } f0, f1;
  auto read1 = [&](Frags& f, const char* sa, const char* sb, int s, int i) __attribute__((always_inline)) {   // a0 b0 .. b3 a1 ..
    if (i == 0) f.a[0] = read32(sa + la, sw[s], sw[s] ^ 16);
    else if (i <= J) f.b[i <= J && i > 0 ? i - 1 : 0] = read32(sb + lb + (i - 1) * 4096, sw[s], sw[s] ^ 16);
    else f.a[i > J ? i - J : 0] = read32(sa + la + (i - J) * 4096, sw[s], sw[s] ^ 16);
  };

  f32x16 acc[I][J];
  constexpr int NM = I * J;
  auto mma = [&](const Frags& f, const Scales& s, auto m) __attribute__((always_inline)) {
    constexpr int i = decltype(m)::value / J, j = decltype(m)::value % J;
    const int b = GLU && j % 2 ? s.u : s.w;
    acc[i][j] = mfma8<0, i>(f.b[j], f.a[i], acc[i][j], b, s.a);
    __asm__ volatile("" : "+a"(acc[i][j]));             // here: the compiler sinks MFMAs past the branches that follow
  };
  // half a stage: its MFMAs on f; the fragments of the next half (half s of the stage at
  // sa, sb) read into fn beside the first of them, and one operand's loads (W: 0, A: 1)
  auto slice = [&](const Frags& f, Frags& fn, const char* sa, const char* sb, int s, auto load) __attribute__((always_inline)) {
    constexpr int L = decltype(load)::value;
    constexpr int NL = L == 0 ? NLB : NLA;
    auto step = [&](auto mi) __attribute__((always_inline)) {
      constexpr int m = decltype(mi)::value;
      mma(f, sc0, mi);
      if constexpr (m < I + J) read1(fn, sa, sb, s, m);
      // few row tiles: the rest of the fragments beside the last MFMA
      if constexpr (m == NM - 1) {
#pragma unroll
        for (int r = NM; r < I + J; ++r) read1(fn, sa, sb, s, r);
      }
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (m == i * NM / NL) {
          if constexpr (L == 0) dma_b(i);
          else dma_a(i);
        }
      __builtin_amdgcn_sched_barrier(0);
    };
    for_each_index(step, std::make_integer_sequence<int, NM>{});
  };
  // the next stage's loads landed, everyone's (the W loads past it stay in flight), and
  // this stage is read
  auto sync = [&]() __attribute__((always_inline)) {
    wait_vmem<NLB>();
    barrier_lds();
  };

  Loaded first;
  load_scales(first);
#pragma unroll
  for (int i = 0; i < NLB; ++i) dma_b(i);
#pragma unroll
  for (int i = 0; i < NLA; ++i) dma_a(i);
  load_scales(sc2);
#pragma unroll
  for (int i = 0; i < NLB; ++i) dma_b(i);
#pragma unroll
  for (int i = 0; i < NLA; ++i) dma_a(i);
  wait_vmem<NLA + NLB + (I == 3 ? 4 : 2) + (GLU ? 1 : 0)>();   // stage 0
  __asm__ volatile("s_barrier" ::: "memory");
  take(sc0, first);
#pragma unroll
  for (int i = 0; i < I + J; ++i) read1(f0, lds[1], lds[0], 0, i);

  int sa = 1, sb = 0;
  for (int tile = tile0, left = n_units; left > 0;) {
    const int n = SPLIT ? n_units : p.ks;
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
      for (int j = 0; j < J; ++j) acc[i][j] = f32x16{};
    for (int kt = 0; kt < n; ++kt) {
      slice(f0, f1, lds[sa], lds[sb], 1, std::integral_constant<int, 0>{});
      sync();
      sa = bump(sa);
      sb = bump(sb);
      take(sc1, sc2);
      load_scales(sc2);
      slice(f1, f0, lds[sa], lds[sb], 0, std::integral_constant<int, 1>{});
      sc0 = sc1;
    }
    // ---- epilogue: lane l has row I (l % 32) + i of the wavefront's in row tile i, and of
    // column tile j the columns 8 q + 4 (l / 32) + 0 .. 3 in registers 4 q .. 4 q + 3.  Results go
    // through LDS, so that a store instruction writes runs of 256 bytes (rows past M fall
    // outside the descriptors): through the half stage that the next W loads will take,
    // which held this stage's A and has been read by everyone.
    int mt, nt;
    tile_mn(tile, mt, nt);
    // Lane numbers that the compiler cannot see through, or it keeps the offsets derived from
    // them over the whole K loop, and spills.
    int el = lane;
    __asm__ volatile("" : "+v"(el));
    const int eh = el >> 5, er = el & 31;
    // Nothing is computed from these tiles before this point: the compiler starts on all of
    // them at once, and runs out of registers.
    auto from_here = [&](int i, int j, int n) __attribute__((always_inline)) {
#pragma unroll
      for (int x = 0; x < n; ++x) __asm__ volatile("" : "+a"(acc[i][j + x]));
    };
    const int mw = mt * TM + wm * (TM / 2);             // the wavefront's first row
    char* room = lds[cb.slot];
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    if constexpr (EPI == kGluQuantOut) {
      // a row's other columns are in lane l ^ 32 and in the wavefront with the other wn: the
      // room takes first the maxima, then the tile
      // the values of a lane wait for their scale where the gate's sums were
      float top[I];
#pragma unroll
      for (int i = 0; i < I; ++i) {
        top[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < J; j += 2) {
          from_here(i, j, 2);
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] = silu(acc[i][j][r]) * acc[i][j + 1][r];
#pragma unroll
          for (int r = 0; r < 16; r += 2)               // NaN is passed over
            top[i] = fmaxf(fmaxf(fabsf(acc[i][j][r]), fabsf(acc[i][j][r + 1])), top[i]);
          from_here(i, j, 1);
          __builtin_amdgcn_sched_barrier(0);
        }
        top[i] = fmaxf(top[i], __shfl_xor(top[i], 32));
      }
      bool inf = false;
#pragma unroll
      for (int i = 0; i < I; ++i) inf |= top[i] == INFINITY;
      if (__any(inf)) {                                 // e4m3 has no infinities: NaN instead
#pragma unroll
        for (int i = 0; i < I; ++i) {
          top[i] = 0.0f;
#pragma unroll
          for (int j = 0; j < J; j += 2) {
            from_here(i, j, 1);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              acc[i][j][r] = fabsf(acc[i][j][r]) == INFINITY ? NAN : acc[i][j][r];
              top[i] = fmaxf(top[i], fabsf(acc[i][j][r]));
            }
            from_here(i, j, 1);
          }
          top[i] = fmaxf(top[i], __shfl_xor(top[i], 32));
        }
      }
      float* tops = reinterpret_cast<float*>(room);     // [wm][wn][i][32]
      int* pick = reinterpret_cast<int*>(room) + 4 * I * 32 + wm * I * 32;   // [wm][i][32]
      typedef Border<4, TM> List;
      static_assert(4096 + sizeof(List) <= SLOT, "the list fits behind them");
      List& list = *reinterpret_cast<List*>(room + 4096);
      if (tid == 0) list.count = 0;
#pragma unroll
      for (int i = 0; i < I; ++i)
        if (eh == 0) tops[(wv * I + i) * 32 + er] = top[i];
      barrier_lds();
      int byte[I];
      bool near = false, mine[I];                       // mine: the largest is one of this wavefront's columns
#pragma unroll
      for (int i = 0; i < I; ++i) {
        const float other = tops[((wv ^ 1) * I + i) * 32 + er];
        mine[i] = wn == 0 ? top[i] >= other : top[i] > other;
        top[i] = fmaxf(top[i], other);
        byte[i] = scale_byte(__float_as_uint(top[i]));
        near |= near_border(__float_as_uint(top[i]));
      }
      if (__any(near)) {                                // next to a border (Border): the same for both wn
#pragma unroll
        for (int i = 0; i < I; ++i) {                   // the first column that has it
          int col = 64;
#pragma unroll
          for (int j = J - 2; j >= 0; j -= 2) {
            from_here(i, j, 1);
#pragma unroll
            for (int r = 15; r >= 0; --r)
              col = fabsf(acc[i][j][r]) == top[i] ? j * 16 + (r >> 2) * 8 + eh * 4 + (r & 3) : col;
          }
          col = min(col, __shfl_xor(col, 32));
          if (mine[i] && eh == 0 && near_border(__float_as_uint(top[i])))
            pick[i * 32 + er] = list.add(min(mw + er * I + i, g.M - 1), nt * (kTN / 2) + wn * 64 + col);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      barrier_lds();
      const int again = list.count;
      if (again > 0) {
        list.compute(g, again, wv, el);
        barrier_lds();
        if (__any(near)) {
#pragma unroll
          for (int i = 0; i < I; ++i)
            if (near_border(__float_as_uint(top[i]))) byte[i] = list.byte(pick[i * 32 + er], __float_as_uint(top[i]));
        }
      }
      barrier_lds();                                    // the maxima and bytes are read
      const int row0 = wm * (TM / 2) + er * I;          // of the tile
#pragma unroll
      for (int i = 0; i < I; ++i) {
#pragma unroll
        for (int j = 0; j < J; j += 2) {
          from_here(i, j, 1);
          const f32x16& v = acc[i][j];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const int row = row0 + i, c = wn * 64 + j * 16 + q * 8 + eh * 4;
            *reinterpret_cast<uint32_t*>(room + row * 128 + ((c >> 4) ^ ((row / I) & 7)) * 16 + (c & 15)) =
                pack_finite_e4m3x4(v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3], byte[i]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      const int first = mw + er * I;
      if (wn == 0 && eh == 0 && first < g.M) {        // I neighbouring rows; those past M are padding
        uint8_t* to = g.out_scale + size_t(nt) * ld + first;
        if constexpr (I == 4) {
          *reinterpret_cast<uint32_t*>(to) = byte[0] | byte[1] << 8 | byte[2] << 16 | byte[3] << 24;
        } else if constexpr (I == 2) {
          *reinterpret_cast<uint16_t*>(to) = uint16_t(byte[0] | byte[1] << 8);
        } else {
#pragma unroll
          for (int i = 0; i < I; ++i)
            if (first + i < g.M) to[i] = uint8_t(byte[i]);
        }
      }
      barrier_lds();
      const __amdgpu_buffer_rsrc_t ro = __builtin_amdgcn_make_buffer_rsrc(g.out, 0, g.M * ffn, kBufWord3);
#pragma unroll
      for (int x = 0; x < TM / 32; ++x) {               // eight lanes a row
        const int row = x * 32 + wv * 8 + (el >> 3), c = el & 7;
        const u32x4 v = *reinterpret_cast<const u32x4*>(room + row * 128 + (c ^ ((row / I) & 7)) * 16);
        __builtin_amdgcn_raw_buffer_store_b128(v, ro, (mt * TM + row) * ffn + nt * (kTN / 2) + c * 16, 0, 0);
      }
    } else {
      // a wavefront's own 8 KB of the room: 32 rows of 256 bytes at a time (bf16: all the
      // columns of a row tile, after SwiGLU half as many; fp32: half of them)
      char* mine = room + wv * 8192;
      constexpr int OUT = SPLIT ? 4 : 2;                // bytes of a result
      constexpr int JS = SPLIT ? 2 : 4;                 // column tiles per pass
      constexpr int W = GLU ? 128 : 256;                // bytes of a row per pass
      constexpr int PAIR = GLU || EPI == kRopeOut ? 2 : 1;   // column tiles that make a result
      const int cols = GLU ? ffn : g.N;
      const int D = g.head_dim, hd2 = D >> 1;           // kRopeOut
      const int n0 = GLU ? nt * (kTN / 2) + wn * 64 : nt * kTN + wn * 128;
      char* out = reinterpret_cast<char*>(SPLIT ? static_cast<void*>(g.partial + size_t(part) * g.M * g.N) : g.out);
      // N % 128 == 0: all of the wavefront's columns, or none
      const __amdgpu_buffer_rsrc_t ro =
          __builtin_amdgcn_make_buffer_rsrc(out, 0, n0 < cols ? g.M * cols * OUT : 0, kBufWord3);
      const int row = er;
#pragma unroll
      for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j0 = 0; j0 < J; j0 += JS) {
          // four results of the lane's row from column c of the pass on
          auto put = [&](int c, float a, float b, float d, float e) __attribute__((always_inline)) {
            char* to = mine + row * W + ((c * OUT >> 4) ^ (row & (W / 16 - 1))) * 16 + (c * OUT & 15);
            if constexpr (SPLIT) *reinterpret_cast<float4*>(to) = make_float4(a, b, d, e);
            else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16x2(a, b), pack_bf16x2(d, e));
          };
          const float2* cs = nullptr;
          if constexpr (EPI == kRopeOut) cs = g.cs + size_t(min(mw + row * I + i, g.M - 1)) * hd2;
#pragma unroll
          for (int j = 0; j < JS; j += PAIR) {
            from_here(i, j0 + j, PAIR);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x16 &v = acc[i][j0 + j], &u = acc[i][j0 + (j + 1) % JS];
              const int c = q * 8 + eh * 4;
              if constexpr (GLU) {
                float x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = silu(v[4 * q + e]) * u[4 * q + e];
                put(j * 16 + c, x[0], x[1], x[2], x[3]);
              } else if constexpr (EPI == kRopeOut) {   // tiles j, j + 1: the halves of a head's pairs
                float x[4], y[4], t[8] = {1.0f, 0.0f, 1.0f, 0.0f, 1.0f, 0.0f, 1.0f, 0.0f};
                if (n0 + (halves ? 0 : j * 32) < (g.hq + g.hkv) * D) {
                  const float4* p = reinterpret_cast<const float4*>(cs + (halves ? j * 16 : 0) + c);
                  const float4 t0 = p[0], t1 = p[1];
                  t[0] = t0.x, t[1] = t0.y, t[2] = t0.z, t[3] = t0.w, t[4] = t1.x, t[5] = t1.y, t[6] = t1.z, t[7] = t1.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  x[e] = v[4 * q + e] * t[2 * e] - u[4 * q + e] * t[2 * e + 1];
                  y[e] = u[4 * q + e] * t[2 * e] + v[4 * q + e] * t[2 * e + 1];
                }
                put(column(j * 32) + c, x[0], x[1], x[2], x[3]);
                put(column(j * 32 + 32) + c, y[0], y[1], y[2], y[3]);
              } else {
                put(j * 32 + c, v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]);
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
          constexpr int LR = W / 16;                    // lanes a row
#pragma unroll
          for (int x = 0; x < 32 * LR / 64; ++x) {
            const int r = x * (64 / LR) + el / LR, c = el % LR;
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * W + (c ^ (r & (LR - 1))) * 16);
            if constexpr (EPI == kRopeOut) {
              const int m = mw + r * I + i, n = n0 + c * 8, head = n / D;
              uint16_t* base = head < g.hq ? g.q : head < g.hq + g.hkv ? g.k : g.v;
              const int heads = head < g.hq ? g.hq : g.hkv;
              const int hd = head < g.hq ? head : head < g.hq + g.hkv ? head - g.hq : head - g.hq - g.hkv;
              if (m < g.M && n < g.N)
                *reinterpret_cast<u32x4*>(base + (size_t(m) * heads + hd) * D + (n - head * D)) = v;
            } else {
              __builtin_amdgcn_raw_buffer_store_b128(v, ro, ((mw + r * I + i) * cols + n0 + j0 * 32) * OUT + c * 16, 0, 0);
            }
          }
          __builtin_amdgcn_sched_barrier(0);
        }
    }
    barrier_lds();                                      // the room is read: the next W loads may land
    left -= n;
    tile += p.G;
  }
  wait_vmem<0>();                                       // no load may land in LDS after the workgroup ends
}

int cdiv(int a, int b) { return (a + b - 1) / b; }

WidePlan8 plan_of(const Gemm8Args& g, int tm) {
  WidePlan8 p{};
  p.m_tiles = cdiv(g.M, tm);
  p.n_tiles = cdiv(g.N, kTN);
  p.tiles = p.m_tiles * p.n_tiles;
  p.ks = g.K / kBK;
  p.gm = std::min(p.m_tiles, 8);
  p.parts = 1;
  p.G = cdiv(cdiv(p.tiles, cdiv(p.tiles, kMaxWorkers)), 8) * 8;
  return p;
}

template <int TM>
void launch_wide_tm(const Gemm8Args& g, int epi, hipStream_t stream) {
  const WidePlan8 p = plan_of(g, TM);
  if (epi == kBf16Out) gemm8_wide_kernel<kBf16Out, TM><<<p.G, 256, 0, stream>>>(g, p);
  else if (epi == kGluOut) gemm8_wide_kernel<kGluOut, TM><<<p.G, 256, 0, stream>>>(g, p);
  else if (epi == kRopeOut) gemm8_wide_kernel<kRopeOut, TM><<<p.G, 256, 0, stream>>>(g, p);
  else gemm8_wide_kernel<kGluQuantOut, TM><<<p.G, 256, 0, stream>>>(g, p);
}

}  // namespace

void launch_gemm8_wide(const Gemm8Args& g, int epi, int tm, hipStream_t stream) {
  if (tm == 256) launch_wide_tm<256>(g, epi, stream);
  else if (tm == 192) launch_wide_tm<192>(g, epi, stream);
  else launch_wide_tm<128>(g, epi, stream);
}

StreamSum launch_gemm8_split(const Gemm8Args& g, int tm, int parts, hipStream_t stream) {
  WidePlan8 p = plan_of(g, tm);
  p.parts = parts;
  p.G = cdiv(p.tiles * parts, 8) * 8;
  StreamSum s{};
  s.partial = g.partial;
  s.M = g.M, s.N = g.N, s.fixed = parts;
  if (tm == 256) gemm8_wide_kernel<kPlanesOut, 256><<<p.G, 256, 0, stream>>>(g, p);
  else if (tm == 192) gemm8_wide_kernel<kPlanesOut, 192><<<p.G, 256, 0, stream>>>(g, p);
  else gemm8_wide_kernel<kPlanesOut, 128><<<p.G, 256, 0, stream>>>(g, p);
  return s;
}

}  // namespace epic

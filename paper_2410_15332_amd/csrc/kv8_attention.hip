// Causal attention (Eq. 1) over the 8-bit linked cache for tiles of 16 query rows: decode.
//
// Workgroup = (work item, KV head), tile rows and items as in the bf16 kernel of such tiles.  A
// wavefront takes pairs of the item's linked blocks, 32 keys, through a ring of registers:
//   S^T (16 keys x 16 rows) = K Q^T per block by v_mfma_f32_16x16x32_bf16, K's bytes widened in
//     registers (exact); lane l = r + 16 a holds the scores of row r for keys 4 a + i, which
//     are scaled by their keys' 2^t;
//   online softmax per row in the scaled log2 domain; the running maximum lags by up to kLag,
//     so that rows are merged over lanes and the output is rescaled only when one grows past it;
//   O^T (D x 16) += V^T P^T by v_mfma_f32_16x16x32_bf16 over both blocks' keys: the P operand of
//     a lane is its own 8 probabilities times their keys' 2^t (exact), rounded to bf16, the operands'
//     type, and V's is the dword of 4 keys of its dim that the cache's order keeps together, for each
//     block.  That rounding is 2^-8 of a probability at most, beside the 2^-4 that V's rounding to e4m3
//     left; the sum of probabilities is taken before it.  Outputs are 0.0017 to 0.0024 of their norm
//     from float64 over the same cache, where rounding them to bf16 alone is 0.0016 to 0.0017; what
//     the probabilities lose would take a second product of as many instructions.
// What bounds it is the read of K and V, once per item.  K's registers take the next pair as soon
// as its scores are formed, V's after the product, and three workgroups of four wavefronts fit a
// CU: 131 323 keys of 8 heads of 128 (271 MB) in 45.5 us, 6.0 TB/s, above what a plain read reaches
// (55.8 with all loads behind the product and two workgroups).  With a single tile no block is read
// twice, and K and V pass the caches (NT): 51 us a step, merge among it, for 58 through them; 131 103 keys of 8
// heads of 64: 31 for 34.  Requests that share blocks read them through the caches: 32 of them 63 us for 71, of
// short documents 25 for 29 (of 64 dims 41.5 for 40.7).
// Up to 256 workgroups, one a CU, have eight wavefronts: what bounds these is the chain of loads (529 keys
// of 8 heads of 64 6.7 us a step, 8.1 by four; 4113 keys 9.5 and 9.9).  They read past the caches whether or not blocks
// are shared, at most 256 / Hkv items then: four requests over the same 32 000 keys of a head of 128 14.8 us, 15.3 through
// the caches, two of them 13.0 and 14.2, of 64 dims 12.3 and 13.2; 24 over the same 2000 keys 11.3 both; 24 over 300 keys
// of 8 heads 8.7 and 8.5.
//
// The link write of few private blocks (decode: one or two a request) is done here too, by
// workgroups in front of the others, and nothing waits for them: the rows of S that a private block
// receives are read from the call's inputs and rounded by whoever attends to them, as a block of
// their own; of the block itself the other tokens are read, from its source, and a block that is its
// own source has only the new rows' bytes stored.  The launch saved makes every step shorter (529 keys
// 6.7 us for 8.5, 131 323 keys 51 for 54, one of 32 requests 63 for 66).
#include <cmath>
#include <type_traits>

#include "kv8_device.h"
#include "plan_internal.h"

namespace epic {

namespace {

constexpr int kDecRows = 16;
constexpr float kLag = 8.0f;

template <int D, int W>
struct Kv8DecodeLds {
  float m[W][kDecRows];
  float l[W][kDecRows];
  float o[W][D][kDecRows];
};

// What a wavefront holds of a block in flight.
template <int J>
struct Kv8Block {
  uint4 k[J], v[J];
  uint32_t ks, vs;                            // scales of keys 4 a ..
};

// W wavefronts, RING pairs of blocks in flight of each.  NT: K and V are read past the caches.
template <int D, int W, int RING, bool NT>
__global__ __launch_bounds__(64 * W, W == 4 ? 3 : 1) void kv8_decode_kernel(AttnArgs a, epic_kv8_cache c, Kv8Rows w) {
  constexpr int J = D / 64;
  constexpr int NDT = D / 16;                 // 16-dim tiles of O^T
  __shared__ Kv8DecodeLds<D, W> lds;

  const int hkv = a.hkv;
  if (int(blockIdx.x) < w.groups) {           // the link write: W KV heads of a private block
    const int ng = (hkv + W - 1) / W, i = blockIdx.x / ng, g = (blockIdx.x % ng) * W + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    if (g >= hkv) return;
    kv8_write_private<D>(w, c, i, hkv, g, lane, reinterpret_cast<uint32_t*>(lds.o[threadIdx.x >> 6]));
    return;
  }
  const int g = (blockIdx.x - w.groups) % hkv;
  const int item = (blockIdx.x - w.groups) / hkv;
  const int32_t* wk = a.work + kWorkInts * item;
  const int tile = wk[0], b0 = wk[1], b1 = wk[2], kind = wk[7];
  if (tile < 0) return;                       // list entries of other items
  const int row0 = a.tiles[4 * tile + 0];
  const int32_t* list = a.work + kWorkInts * wk[6] + 2;   // kItemShared, kItemList: entry i at i / 6 * 8 + i % 6
  auto listed = [&](int i) __attribute__((always_inline)) { return list[i / kExtInts * kWorkInts + i % kExtInts]; };
  const int nrows = kind == kItemShared ? wk[5] : a.tiles[4 * tile + 1];
  // S row, partial (-1: the output) and row within its request's tile of row s
  auto slot = [&](int s, int& srow, int& part, int& lr) __attribute__((always_inline)) {
    if (kind == kItemShared) {
      srow = listed(2 * s);
      const int to = listed(2 * s + 1);
      part = to < 0 ? -1 : to / kDecRows;
      lr = to < 0 ? 0 : to % kDecRows;
    } else {
      srow = row0 + s;
      part = wk[3];
      lr = s;
    }
  };

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);

  // The wavefront's blocks, in pairs: block i of its own (i = 2 p + e) is b0 + 2 (wave + W p) + e.
  // Their ids, positions and lengths come 64 at a time, one per lane, so that no load of a block
  // waits for a chain of loads; past the item's end stands its last block, with no keys.
  const int n_pairs = (b1 - b0 + 1) / 2;
  const int mine = n_pairs > wave ? 2 * ((n_pairs - wave + W - 1) / W) : 0;
  int phys_l, pos_l, valid_l;                 // valid: bit s for token s of the block
  // Private blocks are written by other workgroups of this launch: what they keep is read from their source, their
  // rows of S from the call's inputs.  (Shared blocks are no request's own.)
  const bool own = w.n > 0 && kind != kItemShared;
  int priv_block = 0, priv_src = 0;           // of private block `lane`
  auto fetch = [&](int first) __attribute__((always_inline)) {
    const int i = first + lane;
    const int b = b0 + 2 * (wave + W * (i >> 1)) + (i & 1);
    const bool in = i < mine && b < b1;
    const int bc = in ? b : b1 - 1;
    const int lb = kind == kItemList ? listed(bc) : bc;
    phys_l = a.linked_blocks[lb];
    pos_l = a.block_pos0[lb];
    valid_l = in ? (1 << a.block_len[lb]) - 1 : 0;
    if (own) {
      const int at = min(lane, w.n - 1);
      priv_block = w.block[at];
      priv_src = w.src[at];
    }
  };
  fetch(0);

  const int r = lane & 15;                    // tile row of this lane
  const int qd = lane >> 4;                   // its quarter: keys 4 qd ..
  const int R = a.rows_per_tile;
  const int srl = r % R;
  const int h = g * a.G + r / R;
  const bool row_ok = srl < nrows;
  int srow, part_, lr_;
  slot(row_ok ? srl : nrows - 1, srow, part_, lr_);
  // shared blocks precede every row of the item; lanes without a row see what the last row sees, for nothing
  const int qpos = kind == kItemShared ? 0x7fffff00 : a.s_pos[srow];
  int first_row = qpos;                       // the first position of the tile's rows
#pragma unroll
  for (int off = 1; off < 16; off *= 2) first_row = min(first_row, __shfl_xor(first_row, off));
  first_row = __builtin_amdgcn_readfirstlane(first_row);

  bf16x8 qf[2 * J];                           // Q^T operand: row r, dims 64 j + 16 qd + 8 e ..
  {
    const uint16_t* qp = a.q + (size_t(srow) * a.hq + h) * D + qd * 16;
#pragma unroll
    for (int i = 0; i < 2 * J; ++i) {
      bf16x8 x = *reinterpret_cast<const bf16x8*>(qp + 64 * (i >> 1) + 8 * (i & 1));
      qf[i] = row_ok ? x : bf16x8{0, 0, 0, 0, 0, 0, 0, 0};
    }
  }

  const float sl2 = a.scale_log2;
  const size_t blk_bytes = size_t(hkv) * 16 * D, blk_scales = size_t(hkv) * kKv8Scales;
  const uint8_t* kbase = c.k + size_t(g) * 16 * D + 16 * lane;
  const uint8_t* vbase = c.v + size_t(g) * 16 * D + 16 * lane;
  const uint8_t* sbase = c.scale + size_t(g) * kKv8Scales + 4 * qd;
  auto piece = [&](const uint8_t* p) __attribute__((always_inline)) {
    return NT ? load16(p) : *reinterpret_cast<const uint4*>(p);
  };
  auto load_k = [&](int phys, Kv8Block<J>& x) __attribute__((always_inline)) {
    x.ks = *reinterpret_cast<const uint32_t*>(sbase + size_t(phys) * blk_scales);
#pragma unroll
    for (int j = 0; j < J; ++j) x.k[j] = piece(kbase + size_t(phys) * blk_bytes + 1024 * j);
  };
  auto load_v = [&](int phys, Kv8Block<J>& x) __attribute__((always_inline)) {
    x.vs = *reinterpret_cast<const uint32_t*>(sbase + size_t(phys) * blk_scales + 16);
#pragma unroll
    for (int j = 0; j < J; ++j) x.v[j] = piece(vbase + size_t(phys) * blk_bytes + 1024 * j);
  };

  f32x4 o[NDT];
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt) o[dt] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  float m = -INFINITY, lsum = 0.0f;           // lsum: of this lane's keys

  // one block's scores, in the log2 domain
  auto scores = [&](const Kv8Block<J>& x, float (&s)[4]) __attribute__((always_inline)) {
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const uint4 w = x.k[j];
      const u32x4 lo = {e4m3_pair<false>(w.x, 1.0f), e4m3_pair<true>(w.x, 1.0f), e4m3_pair<false>(w.y, 1.0f),
                        e4m3_pair<true>(w.y, 1.0f)};
      const u32x4 hi = {e4m3_pair<false>(w.z, 1.0f), e4m3_pair<true>(w.z, 1.0f), e4m3_pair<false>(w.w, 1.0f),
                        e4m3_pair<true>(w.w, 1.0f)};
      acc = mfma_16x16x32(__builtin_bit_cast(bf16x8, lo), qf[2 * j], acc);
      acc = mfma_16x16x32(__builtin_bit_cast(bf16x8, hi), qf[2 * j + 1], acc);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = __builtin_amdgcn_ldexpf(acc[i] * sl2, int(x.ks >> (8 * i) & 255u) - 127);
  };
  // One step of two blocks, at positions pos0 and pos1, of whose tokens those of the bits valid0 and valid1 are read.
  // ONE: of x0 alone, whose V is finite; x1 is x0.
  auto step = [&](auto one, Kv8Block<J>& x0, Kv8Block<J>& x1, int pos0, int pos1, int valid0, int valid1, auto after_k,
                  auto after_v) __attribute__((always_inline)) {
    constexpr bool ONE = decltype(one)::value;
    float t0[4], t1[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    scores(x0, t0);
    if constexpr (!ONE) scores(x1, t1);
    float s[8] = {t0[0], t0[1], t0[2], t0[3], t1[0], t1[1], t1[2], t1[3]};
    after_k();
    // masked: tokens that are not valid, or after the row (whole blocks before every row need nothing)
    const bool whole = !ONE && (valid0 & valid1) == 0xFFFF;
    if (!whole || max(pos0, pos1) + 15 > first_row) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[i] = (valid0 >> (4 * qd + i) & 1) && pos0 + 4 * qd + i <= qpos ? s[i] : -INFINITY;
        if constexpr (!ONE) s[4 + i] = (valid1 >> (4 * qd + i) & 1) && pos1 + 4 * qd + i <= qpos ? s[4 + i] : -INFINITY;
      }
    }
    float mb = fmaxf(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])), fmaxf(fmaxf(s[4], s[5]), fmaxf(s[6], s[7])));
    if (__ballot(mb > m + kLag)) {            // a row's maximum grew past the lag (at first: from nothing)
      mb = fmaxf(mb, __shfl_xor(mb, 16));
      mb = fmaxf(mb, __shfl_xor(mb, 32));
      const bool grow = mb > m + kLag;        // row by row: a row's result depends on no other row
      const float alpha = grow ? fast_exp2(m - mb) : 1.0f;
      m = grow ? mb : m;
      lsum *= alpha;
#pragma unroll
      for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[dt][i] *= alpha;
    }
    const float m_use = m == -INFINITY ? 0.0f : m;
    float pv[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float q = fast_exp2(s[i] - m_use);
      lsum += q;
      pv[i] = __builtin_amdgcn_ldexpf(q, int((i < 4 ? x0.vs : x1.vs) >> (8 * (i & 3)) & 255u) - 127);
    }
    const u32x4 pw = {pack_bf16x2(pv[0], pv[1]), pack_bf16x2(pv[2], pv[3]), pack_bf16x2(pv[4], pv[5]),
                      pack_bf16x2(pv[6], pv[7])};
    const bf16x8 pb = __builtin_bit_cast(bf16x8, pw);
    if (!ONE && !whole) {                     // other tokens' bytes may be any, and a weight of 0 would not hide NaN
      const uint32_t keep0 = byte_mask(valid0 >> (4 * qd) & 15), keep1 = byte_mask(valid1 >> (4 * qd) & 15);
#pragma unroll
      for (int q = 0; q < J; ++q) {
        x0.v[q] = merge(make_uint4(0, 0, 0, 0), x0.v[q], keep0);
        x1.v[q] = merge(make_uint4(0, 0, 0, 0), x1.v[q], keep1);
      }
    }
#pragma unroll
    for (int q = 0; q < J; ++q) {
      const uint32_t w0[4] = {x0.v[q].x, x0.v[q].y, x0.v[q].z, x0.v[q].w};
      const uint32_t w1[4] = {x1.v[q].x, x1.v[q].y, x1.v[q].z, x1.v[q].w};
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        const u32x4 vv = {e4m3_pair<false>(w0[t], 1.0f), e4m3_pair<true>(w0[t], 1.0f), e4m3_pair<false>(w1[t], 1.0f),
                          e4m3_pair<true>(w1[t], 1.0f)};
        o[4 * q + t] = mfma_16x16x32(__builtin_bit_cast(bf16x8, vv), pb, o[4 * q + t]);
      }
    }
    after_v();
  };

  for (int first = 0; first < mine; first += 64) {
    if (first > 0) fetch(first);
    const int n = min(64, mine - first) / 2;  // pairs of this batch
    Kv8Block<J> ring[RING][2];
    auto fill = [&]() __attribute__((always_inline)) {
#pragma unroll
      for (int j = 0; j < RING; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int phys = __builtin_amdgcn_readlane(phys_l, 2 * min(j, n - 1) + e);
          load_k(phys, ring[j][e]);
          load_v(phys, ring[j][e]);
        }
    };
    fill();
    int priv_l = -1;                          // this block's place among the private ones
    if (own) {
      for (int q = 0; q < w.n; ++q) priv_l = phys_l == __builtin_amdgcn_readlane(priv_block, q) ? q : priv_l;
      if (valid_l == 0) priv_l = -1;
      // in decode a block is its own source, or has none and holds nothing but rows of S
      const int from = __shfl(priv_src, max(priv_l, 0));
      const bool moved = priv_l >= 0 && from >= 0 && from != phys_l;
      const uint64_t any_moved = __ballot(moved);
      if (moved) phys_l = from;
      uint64_t left = __ballot(priv_l >= 0);
      if (left != 0) {
        // the rows of S of private blocks, each a block of its own
        do {
          const int i = __builtin_ctzll(left), q = __builtin_amdgcn_readlane(priv_l, i);
          left &= left - 1;
          const Kv8Fresh<J> f =
              kv8_fresh<D>(w.rows[q * 16 + r], w.k_s, w.v_s, hkv, g, lane, reinterpret_cast<uint32_t*>(lds.o[wave]));
          Kv8Block<J> x;
#pragma unroll
          for (int j = 0; j < J; ++j) x.k[j] = f.k[j], x.v[j] = f.v[j];
          x.ks = f.ks, x.vs = f.vs;
          const int pos = __builtin_amdgcn_readlane(pos_l, i);
          step(std::true_type{}, x, x, pos, pos, int(f.tokens), 0, [] {}, [] {});
          if (lane == i) valid_l &= ~int(f.tokens);
        } while (left != 0);
        // from the sources; and four wavefronts have no registers for this and the ring at once
        if (W <= 4 || any_moved != 0) fill();
      }
    }
    for (int base = 0; base < n; base += RING) {
#pragma unroll
      for (int j = 0; j < RING; ++j) {
        const int p = base + j;
        if (p < n) {
          // what this slot holds next; past the batch's end block 0 of the pool, which every wavefront reads there and
          // the caches keep, so that the same loads are in flight behind every wait (the last pair again: 7% more bytes)
          const int next = 2 * min(p + RING, n - 1);
          const bool more = p + RING < n;
          const int phys0 = more ? __builtin_amdgcn_readlane(phys_l, next) : 0;
          const int phys1 = more ? __builtin_amdgcn_readlane(phys_l, next + 1) : 0;
          auto after_k = [&]() __attribute__((always_inline)) {
            load_k(phys0, ring[j][0]);
            load_k(phys1, ring[j][1]);
          };
          auto after_v = [&]() __attribute__((always_inline)) {
            load_v(phys0, ring[j][0]);
            load_v(phys1, ring[j][1]);
          };
          step(std::false_type{}, ring[j][0], ring[j][1], __builtin_amdgcn_readlane(pos_l, 2 * p),
               __builtin_amdgcn_readlane(pos_l, 2 * p + 1), __builtin_amdgcn_readlane(valid_l, 2 * p),
               __builtin_amdgcn_readlane(valid_l, 2 * p + 1), after_k, after_v);
        }
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): the ring's last loads land before the exit

  lsum += __shfl_xor(lsum, 16);
  lsum += __shfl_xor(lsum, 32);
  // merge the wavefronts: O^T of lane l holds dims 16 dt + 4 qd + i of row r
  if (qd == 0) {
    lds.m[wave][r] = m;
    lds.l[wave][r] = lsum;
  }
#pragma unroll
  for (int dt = 0; dt < NDT; ++dt)
#pragma unroll
    for (int i = 0; i < 4; ++i) lds.o[wave][dt * 16 + qd * 4 + i][r] = o[dt][i];
  __syncthreads();
  // thread -> (row rr, dims dd, dd + 4 W, ...): 16 rows x 4 W dim groups
  const int rr = tid & 15, d0 = tid >> 4;
  float mw[W], M = -INFINITY;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    mw[w] = lds.m[w][rr];
    M = fmaxf(M, mw[w]);
  }
  const float Mu = M == -INFINITY ? 0.0f : M;
  float wt[W], L = 0.0f;
#pragma unroll
  for (int w = 0; w < W; ++w) {
    wt[w] = fast_exp2(mw[w] - Mu);
    L += lds.l[w][rr] * wt[w];
  }
  const int s2 = rr % R;
  if (s2 >= nrows) return;
  int srow2, part, lr2;
  slot(s2, srow2, part, lr2);
  const int hh = rr / R, h2 = g * a.G + hh, rp = hh * R + lr2;   // rp: its row in its request's tile
  const float inv = L == 0.0f ? 0.0f : 1.0f / L;
  for (int d = d0; d < D; d += 4 * W) {
    float acc = 0.0f;
#pragma unroll
    for (int w = 0; w < W; ++w) acc += lds.o[w][d][rr] * wt[w];
    acc *= inv;
    if (part < 0)
      a.out[(size_t(srow2) * a.hq + h2) * D + d] = uint16_t(pack_bf16x2(acc, 0.0f) & 0xFFFFu);
    else
      a.part_o[((size_t(part) * hkv + g) * kDecRows + rp) * D + d] = acc;
  }
  if (d0 == 0) {
    if (part < 0) {
      if (a.lse) a.lse[size_t(srow2) * a.hq + h2] = (M + fast_log2(L)) * kLn2;
    } else {
      a.part_lse[(size_t(part) * hkv + g) * kDecRows + rp] = L == 0.0f ? -INFINITY : M + fast_log2(L);
    }
  }
}

}  // namespace

void launch_kv8_decode(const AttnArgs& a, const epic_kv8_cache& c, const Kv8Rows& rows, int head_dim, int n_work, bool once,
                       hipStream_t stream) {
  const unsigned items = unsigned(n_work) * unsigned(a.hkv);
  auto groups = [&](int waves) { return rows.n * ((a.hkv + waves - 1) / waves); };
  auto go = [&](auto kernel, int waves) {
    Kv8Rows w = rows;
    w.groups = groups(waves);
    if (items + w.groups > 0) kernel<<<items + w.groups, 64 * waves, 0, stream>>>(a, c, w);
  };
  if (items + groups(8) <= 256) {              // (NT whatever `once` says: figures above)
    if (head_dim == 128) go(kv8_decode_kernel<128, 8, 1, true>, 8);
    else go(kv8_decode_kernel<64, 8, 1, true>, 8);
    return;
  }
  if (head_dim == 128) once ? go(kv8_decode_kernel<128, 4, 1, true>, 4) : go(kv8_decode_kernel<128, 4, 1, false>, 4);
  else once ? go(kv8_decode_kernel<64, 4, 2, true>, 4) : go(kv8_decode_kernel<64, 4, 2, false>, 4);
}

}  // namespace epic

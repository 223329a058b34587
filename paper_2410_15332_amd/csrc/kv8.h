// Cache blocks in 8 bits: e4m3 values and, for each token and KV head, one power-of-two scale
// (an e8m0 byte) for its K and one for its V.  Host side of kv8.hip and kv8_attention.hip;
// arguments are validated by the callers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "kernels.h"

namespace epic {

// Bytes of a (block, KV head): values of K, as many of V, and 16 + 16 scales.
constexpr int kKv8Scales = 32;
constexpr int kKv8Nan = 255;                  // scale byte of a token whose K or V is not finite

// Workgroups of the re-rotating write: four KV heads of a block each.  The other launches fill theirs with (block, KV
// head) pairs and take no more than that; their limit is held by this count too.
inline int64_t kv8_groups(int64_t n, int hkv) { return n * ((hkv + 3) / 4); }
constexpr int64_t kKv8MaxGroups = (int64_t(1) << 24) - 1;        // x 256 threads < 2^32

struct Kv8Move {
  const int32_t* src;                         // block ids, or null for 0 .. n - 1
  const int32_t* dst;
  int n, src_blocks, dst_blocks;              // ids outside their pool are passed over
  int hkv;
};

void launch_kv8_pack(const Kv8Move& mv, int head_dim, const uint16_t* k, const uint16_t* v, const epic_kv8_cache& c,
                     hipStream_t stream);
void launch_kv8_unpack(const Kv8Move& mv, int head_dim, const epic_kv8_cache& c, uint16_t* k, uint16_t* v,
                       hipStream_t stream);
// Private blocks, their sources and the rows of S that they receive.
struct Kv8Rows {
  const int32_t *block, *src, *rows;          // priv_block, priv_src, priv_rows
  const uint16_t *k_s, *v_s;
  int n;                                      // private blocks; 0 in launches that find them written
  int groups;                                 // workgroups of the launch that write them (set by the launcher)
};
// Most that the launch that reads them writes itself: each of its wavefronts looks through them, a lane each.
constexpr int kKv8JoinedRows = 64;
constexpr int kKv8JoinedPairs = 1024;         // (linked block, KV head) of wide tiles; measured at kv8_expand_kernel

// As launch_link_write and (priv_rot not null) launch_link_write_rotated.
void launch_kv8_write(const Kv8Rows& w, const int32_t* priv_rot, int hkv, int head_dim, float rope_theta,
                      const epic_kv8_cache& c, hipStream_t stream);
// Listed blocks (null: blocks 0 .. n - 1) as a bf16 cache of n blocks, for the attention kernel of wide tiles, and the
// table 0 .. n - 1 where not null; writes the private blocks of w.
void launch_kv8_expand(const int32_t* list, int n, int hkv, int head_dim, const epic_kv8_cache& c, const Kv8Rows& w,
                       uint16_t* k, uint16_t* v, int32_t* table, hipStream_t stream);
// As launch_link_decode; a.k_cache and a.v_cache are not read.  Writes the private blocks of w.  once: no two work
// items read the same block.
void launch_kv8_decode(const AttnArgs& a, const epic_kv8_cache& c, const Kv8Rows& w, int head_dim, int n_work, bool once,
                       hipStream_t stream);

}  // namespace epic

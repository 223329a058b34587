// Entry points of the 8-bit cache: argument validation on the host, then kernel launches on the
// caller's stream.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "attention_call.h"
#include "kv8.h"
#include "plan_internal.h"
#include "status.h"

using namespace epic;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

size_t round_up(size_t n, size_t a) { return (n + a - 1) / a * a; }

epic_status hip_status(const char* what) {
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(EPIC_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return EPIC_OK;
}

epic_status check_cache(const epic_kv8_cache* c) {
  EPIC_CHECK_ARG(c != nullptr, "8-bit cache is NULL");
  EPIC_CHECK_ARG(c->num_blocks >= 0, "num_blocks %d < 0", c->num_blocks);
  EPIC_CHECK_ARG(c->k && c->v && c->scale && aligned16(c->k) && aligned16(c->v) && aligned16(c->scale),
                 "8-bit cache NULL or unaligned");
  return EPIC_OK;
}

// Arguments of a move between the two kinds of cache; n_src and n_dst are their pools' blocks.
epic_status check_move(const epic_attn_cfg* cfg, int32_t n, const int32_t* src, int32_t n_src, const int32_t* dst,
                       int32_t n_dst, const uint16_t* k, const uint16_t* v, const epic_kv8_cache* c) {
  epic_status st = validate_attn_cfg(cfg);
  if (st != EPIC_OK) return st;
  EPIC_CHECK_ARG(n >= 0 && n_src >= 0 && n_dst >= 0, "n %d, pools of %d and %d blocks", n, n_src, n_dst);
  EPIC_CHECK_ARG((src || n <= n_src) && (dst || n <= n_dst), "%d blocks without a list, pools of %d and %d", n, n_src, n_dst);
  if (kv8_groups(n, cfg->num_kv_heads) > kKv8MaxGroups)
    return fail(EPIC_ERR_UNSUPPORTED, "%d blocks of %d KV heads are too many", n, cfg->num_kv_heads);
  if (n == 0) return EPIC_OK;
  st = check_cache(c);
  if (st != EPIC_OK) return st;
  EPIC_CHECK_ARG(k && v && aligned16(k) && aligned16(v), "KV caches NULL or unaligned");
  return EPIC_OK;
}

// Workspace: split-KV partials as in the bf16 call, then, for wide tiles, the linked blocks in bf16 and their table.
struct Layout {
  size_t partials, k, v, table, total;
};
Layout layout(const epic_attn_cfg* cfg, const epic_plan_sizes* s) {
  Layout w{};
  w.partials = epic_link_workspace_bytes(cfg, s);
  w.k = w.v = w.table = w.total = round_up(w.partials, 256);
  if (s->tile_rows != kTileRowsTiny && s->n_s > 0) {
    const size_t cache = size_t(s->n_linked_blocks) * cfg->num_kv_heads * kBlock * cfg->head_dim * sizeof(uint16_t);
    w.v = w.k + round_up(cache, 256);
    w.table = w.v + round_up(cache, 256);
    w.total = w.table + round_up(size_t(s->n_linked_blocks) * sizeof(int32_t), 256);
  }
  return w;
}

}  // namespace

extern "C" epic_status epic_kv8_pack(const epic_attn_cfg* cfg, int32_t n, const int32_t* src_blocks,
                                     const uint16_t* k_cache, const uint16_t* v_cache, int32_t num_blocks,
                                     const int32_t* dst_blocks, const epic_kv8_cache* cache, void* stream) {
  clear_error();
  EPIC_CHECK_ARG(cache != nullptr, "8-bit cache is NULL");
  epic_status st = check_move(cfg, n, src_blocks, num_blocks, dst_blocks, cache->num_blocks, k_cache, v_cache, cache);
  if (st != EPIC_OK || n == 0) return st;
  launch_kv8_pack({src_blocks, dst_blocks, n, num_blocks, cache->num_blocks, cfg->num_kv_heads}, cfg->head_dim, k_cache,
                  v_cache, *cache, static_cast<hipStream_t>(stream));
  return hip_status("8-bit cache pack launch");
}

extern "C" epic_status epic_kv8_unpack(const epic_attn_cfg* cfg, int32_t n, const int32_t* src_blocks,
                                       const epic_kv8_cache* cache, const int32_t* dst_blocks, uint16_t* k_cache,
                                       uint16_t* v_cache, int32_t num_blocks, void* stream) {
  clear_error();
  EPIC_CHECK_ARG(cache != nullptr, "8-bit cache is NULL");
  epic_status st = check_move(cfg, n, src_blocks, cache->num_blocks, dst_blocks, num_blocks, k_cache, v_cache, cache);
  if (st != EPIC_OK || n == 0) return st;
  launch_kv8_unpack({src_blocks, dst_blocks, n, cache->num_blocks, num_blocks, cfg->num_kv_heads}, cfg->head_dim, *cache,
                    k_cache, v_cache, static_cast<hipStream_t>(stream));
  return hip_status("8-bit cache unpack launch");
}

extern "C" size_t epic_link_kv8_workspace_bytes(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes) {
  if (!cfg || !sizes || validate_attn_cfg(cfg) != EPIC_OK) return 0;
  return layout(cfg, sizes).total;
}

extern "C" epic_status epic_link_attention_kv8(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes,
                                               const epic_plan* plan_dev, const uint16_t* q_s, const uint16_t* k_s,
                                               const uint16_t* v_s, const epic_kv8_cache* cache, uint16_t* out,
                                               float* lse, void* workspace, size_t workspace_bytes, void* stream_ptr) {
  clear_error();
  epic_status st = check_attention(cfg, sizes, plan_dev);
  if (st != EPIC_OK) return st;
  if (sizes->n_s == 0 && sizes->n_private == 0) return EPIC_OK;
  st = check_cache(cache);
  if (st != EPIC_OK) return st;
  const int hkv = cfg->num_kv_heads, d = cfg->head_dim;
  // a launch has fewer than 2^32 threads: 256 per four KV heads of a block, up to 512 per KV head of a work item
  if (kv8_groups(int64_t(sizes->n_private) + sizes->n_linked_blocks, hkv) > kKv8MaxGroups ||
      2 * (int64_t(sizes->n_work) + sizes->n_private) * hkv > kKv8MaxGroups)
    return fail(EPIC_ERR_UNSUPPORTED, "%d linked and %d private blocks, %d work items of %d KV heads are too many",
                sizes->n_linked_blocks, sizes->n_private, sizes->n_work, hkv);
  hipStream_t stream = static_cast<hipStream_t>(stream_ptr);
  if (sizes->n_s > 0) {
    EPIC_CHECK_ARG(q_s && k_s && v_s && out, "NULL tensor argument");
    EPIC_CHECK_ARG(aligned16(q_s) && aligned16(k_s) && aligned16(v_s) && aligned16(out), "tensors must be 16-byte aligned");
  }
  const Layout w = layout(cfg, sizes);
  if (w.total > 0) {
    if (workspace == nullptr || workspace_bytes < w.total)
      return fail(EPIC_ERR_WORKSPACE, "workspace of %zu bytes given, %zu needed", workspace_bytes, w.total);
    EPIC_CHECK_ARG(aligned16(workspace), "workspace must be 16-byte aligned");
  }
  record_profile_event(0, stream);
  const bool tiny = sizes->tile_rows == kTileRowsTiny;
  Kv8Rows rows{plan_dev->priv_block, plan_dev->priv_src, plan_dev->priv_rows, k_s, v_s, sizes->n_private, 0};
  // Few private blocks, none turned, are written by the launch that reads them; for wide tiles where a launch counts
  // beside what is widened
  const bool joined = sizes->n_s > 0 && sizes->n_rerotated == 0 && sizes->n_private <= kKv8JoinedRows &&
                      (tiny || int64_t(sizes->n_linked_blocks) * hkv <= kKv8JoinedPairs);
  if (!joined) {
    launch_kv8_write(rows, sizes->n_rerotated > 0 ? plan_dev->priv_rot : nullptr, hkv, d, cfg->rope_theta, *cache, stream);
    rows.n = 0;
  }
  if (sizes->n_s == 0) return hip_status("8-bit link write launch");      // re-rotated copies only
  AttnArgs a = attention_args(cfg, sizes, plan_dev, q_s, nullptr, nullptr, out, lse, workspace);
  if (tiny) {
    record_profile_event(1, stream);
    // a single tile: no two work items read the same block
    launch_kv8_decode(a, *cache, rows, d, sizes->n_work, sizes->n_tiles == 1, stream);
  } else {
    // The matrix cores bound wide tiles, and every tile would widen the same keys again: they are widened once, for
    // the bf16 kernel.  Requests that share blocks link more of them than there are: the pool then, block by block.  A
    // pool that holds more than the list, of other documents, is not: there a block is widened once for each request that
    // links it (32 requests of 8 x 2000 tokens of 64 documents, 8505 distinct of 32 256 blocks: 2119 us over a pool of
    // 8704, 2729 over one of 40 704).
    char* ws = static_cast<char*>(workspace);
    uint16_t* k = reinterpret_cast<uint16_t*>(ws + w.k);
    uint16_t* v = reinterpret_cast<uint16_t*>(ws + w.v);
    int32_t* table = reinterpret_cast<int32_t*>(ws + w.table);
    a.k_cache = k, a.v_cache = v;
    if (cache->num_blocks < sizes->n_linked_blocks) {
      launch_kv8_expand(nullptr, cache->num_blocks, hkv, d, *cache, rows, k, v, nullptr, stream);
    } else {
      launch_kv8_expand(plan_dev->linked_blocks, sizes->n_linked_blocks, hkv, d, *cache, rows, k, v, table, stream);
      a.linked_blocks = table;
    }
    record_profile_event(1, stream);
    launch_link_attention(a, d, sizes->n_work, stream);
  }
  record_profile_event(2, stream);
  if (sizes->n_partials > 0) launch_link_combine(a, d, sizes->n_tiles, stream);
  record_profile_event(3, stream);
  return hip_status("8-bit link attention launch");
}

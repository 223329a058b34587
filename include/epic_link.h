/*
 * epic_link.h -- C ABI of libepic_link, the link step of LegoLink
 * position-independent caching (EPIC, arXiv 2410.15332) on AMD MI355X (gfx950).
 *
 * The link step (Sec. 2.2 "link", Sec. 4.2): per-chunk KV caches were computed
 * independently, each with positions starting at 0 (the compile step).  A request
 * names chunks (in order) and a suffix of new (mutable) tokens.  The linked
 * sequence is the chunks concatenated, then the suffix.  Only the selected set S
 * is computed: the first k tokens of every chunk except the first, plus every
 * suffix token (LegoLink-k, Sec. 4.2).  Each S row attends causally over the
 * whole linked KV, in which S rows carry their newly computed K/V at their own
 * linked positions (Eq. 1).  k < 0 selects every token (Fully Recompute, Sec. 2.3).
 *
 * Conventions used everywhere below
 *  - bf16 values are passed as uint16_t bit patterns.
 *  - Paged KV cache of one layer: fixed blocks of `block_size` (16) token slots.
 *      K cache: [num_blocks][Hkv][block_size][head_dim]   (a key's vector is contiguous)
 *      V cache: [num_blocks][Hkv][head_dim][block_size]   (a block's keys are contiguous per dim)
 *    Slot id = block * block_size + offset.
 *  - Shared chunk blocks are read only.  Every block that receives a recomputed
 *    row is a request-private block taken from the caller's free list; a private
 *    block that also holds cached rows is first copied from the shared block
 *    (copy-on-write).  The "updated linked KV" is the linked block table of the
 *    plan plus the contents of the private blocks.
 *  - Device pointers are caller-owned device memory (e.g. torch tensors).  Device
 *    entry points enqueue work on `stream` (a hipStream_t; NULL = default stream)
 *    and return without synchronising.  Argument errors are detected on the host
 *    before anything is enqueued; nothing is launched when a call fails.
 *  - No entry point allocates device memory; scratch space is the caller's
 *    `workspace` of at least the size the matching *_workspace_bytes call returns
 *    (epic_link_attention_noalloc instead uses a fixed device array of the library).
 *  - Return value: EPIC_OK or an error code; epic_last_error() gives detail
 *    (thread-local, valid until the next call on the same thread).
 */
#ifndef EPIC_LINK_H
#define EPIC_LINK_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  EPIC_OK = 0,
  EPIC_ERR_INVALID_ARG = 1,     /* malformed sizes, ids out of range, NULL where data is needed */
  EPIC_ERR_UNSUPPORTED = 2,     /* a shape the library does not implement */
  EPIC_ERR_NO_PRIVATE_BLOCKS = 3,/* free list shorter than the plan needs */
  EPIC_ERR_WORKSPACE = 4,       /* workspace smaller than required */
  EPIC_ERR_HIP = 5              /* a HIP runtime call failed (launch error) */
} epic_status;

/* Static description of a status code; never freed. */
const char* epic_status_string(int status);
/* Detail of the last failure on this thread ("" if none). */
const char* epic_last_error(void);
/* Library version string, e.g. "epic_link 0.1 gfx950". */
const char* epic_version(void);

/* Attention shape.  Supported: head_dim in {64, 128}; block_size == 16;
 * num_q_heads a multiple of num_kv_heads with G = num_q_heads / num_kv_heads a
 * power of two <= 128.  Query head h reads KV head floor(h / G).
 * softmax_scale == 0 means 1 / sqrt(head_dim).
 * kv_split_blocks: key blocks per split-KV work item (0 = library default);
 * rows whose keys span several work items are merged with a log-sum-exp combine.
 * tile_rows: query rows (S row x head) per attention workgroup, 16, 128 or 256
 * (0 = library default: 16 when every request has at most 16 / G S rows, as in
 * decode; else 256 when the rows of a tile need nearly the same keys, else 128).
 * 16-row tiles need G <= 16.
 * rope_theta: the rotary base theta (inverse frequency theta^(-2i/D), pairs (i, i + D/2))
 * that cached K was rotated with; a plan with re-rotated blocks needs it > 0. */
typedef struct {
  int32_t num_q_heads;
  int32_t num_kv_heads;
  int32_t head_dim;
  int32_t block_size;
  float softmax_scale;
  int32_t kv_split_blocks;
  int32_t tile_rows;
  float rope_theta;    /* rotary base of the cached K; used only by plans that re-rotate (else may be 0) */
} epic_attn_cfg;

/* One request, host memory, caller-owned.
 * chunk_blocks[chunk_block_off[j] .. chunk_block_off[j+1]) are the physical
 * blocks of chunk j in token order: token t of the chunk is in block t / bs at
 * offset t % bs; a chunk needs exactly ceil(chunk_len[j] / bs) blocks.
 * Chunk ids may repeat inside a request and across requests (shared caches).
 * Cached K is stored rotated at the chunk's own positions 0..L-1 (the compile
 * step).  By default the link reuses it as stored (the paper reuses cached KV
 * unchanged).  rerotate = 1 instead rotates the cached K rows of every chunk j > 0
 * by its linked offset off_j (RoPE composes, so R(off_j) R(t) = R(off_j + t)): all
 * blocks of those chunks become private copies, written by the link write with K
 * rotated in fp32 from float64 angles and rounded to bf16, V copied unchanged.
 * Chunk 0 (offset 0) stays shared.  Ignored for k < 0 (every token recomputed).
 * The rotation is that of epic_attn_cfg.rope_theta: keys that were rotated otherwise
 * (epic_rope_cfg) must not be re-rotated. */
typedef struct {
  int32_t num_chunks;
  const int32_t* chunk_len;        /* [num_chunks], each >= 1 */
  const int32_t* chunk_block_off;  /* [num_chunks + 1], CSR offsets, [0] == 0 */
  const int32_t* chunk_blocks;     /* physical block ids */
  int32_t suffix_len;              /* mutable tokens after the chunks, >= 0 */
  int32_t k;                       /* LegoLink-k; k < 0 = recompute every token */
  int32_t rerotate;                /* 1: cached K of chunk j > 0 is re-rotated to its linked positions */
} epic_link_request;

/* Sizes of a plan for a batch of requests. */
typedef struct {
  int32_t batch;
  int32_t n_s;              /* rows of S over the batch */
  int32_t n_linked_blocks;  /* entries of the linked block tables */
  int32_t n_private;        /* private blocks taken from the free list */
  int32_t n_tiles;          /* attention query tiles (per KV head) */
  int32_t n_work;           /* attention work items (per KV head), list entries among them */
  int32_t n_partials;       /* split-KV partial results (per KV head) */
  int32_t tile_rows;        /* query rows (S row x head) per tile: 16, 128 or 256 */
  int32_t max_pos;          /* 1 + largest linked position in the batch */
  int32_t n_rerotated;      /* private blocks whose copied rows are re-rotated */
  int64_t total_ints;       /* int32 entries of the plan buffer */
} epic_plan_sizes;

/* Plan arrays (all int32).  epic_plan_layout() points them into one contiguous
 * buffer of sizes.total_ints int32 so that the plan can be uploaded with a
 * single copy; the same layout call on the device copy gives the device plan.
 *   s_pos[n_s]            linked position of each S row (ascending per request)
 *   s_req[n_s]            request of each S row
 *   s_slot[n_s]           slot id receiving the row's K/V
 *   s_off[batch + 1]      S rows of request r: [s_off[r], s_off[r+1])
 *   linked_blocks[n_lb]   linked block table (physical ids, position order)
 *   block_pos0[n_lb]      linked position of slot 0 of each linked block
 *   block_len[n_lb]       valid slots of each linked block (1..block_size)
 *   blk_off[batch + 1]    linked blocks of request r
 *   priv_block[n_private] private block ids (taken from free_blocks in order)
 *   priv_src[n_private]   shared block copied into it first, or -1
 *   priv_rows[n_private * block_size]  S row stored in each slot, or -1
 *   priv_rot[n_private]   linked offset by which the rows copied from priv_src are
 *                         re-rotated (K only), or 0
 *   tiles[n_tiles * 4]    (first S row, S rows, first partial or -1, splits)
 *   work[n_work * 8]      (tile, first linked block, end linked block, partial or -1,
 *                         leading 4-block KV tiles that need no mask, 0, 0, 0).
 *                         Decode plans of requests that share chunk blocks also have items
 *                         that carry rows of several requests (last int 1: n listed S rows
 *                         over blocks all of them link) or a list of blocks (last int 2),
 *                         and list entries (first int -1)
 */
typedef struct {
  int32_t* s_pos;
  int32_t* s_req;
  int32_t* s_slot;
  int32_t* s_off;
  int32_t* linked_blocks;
  int32_t* block_pos0;
  int32_t* block_len;
  int32_t* blk_off;
  int32_t* priv_block;
  int32_t* priv_src;
  int32_t* priv_rows;
  int32_t* tiles;
  int32_t* work;
  int32_t* priv_rot;
} epic_plan;

/* Host only, integer, synchronous.  Validates the requests and computes the
 * plan sizes for a batch.  n_free is the number of free blocks the caller can
 * offer; EPIC_ERR_NO_PRIVATE_BLOCKS if the plan needs more. */
epic_status epic_plan_sizes_get(const epic_link_request* reqs, int32_t batch,
                                const epic_attn_cfg* cfg, int32_t n_free,
                                epic_plan_sizes* out);

/* Points the arrays of `plan` into `base` (host or device memory of
 * sizes->total_ints int32).  Pure pointer arithmetic; never dereferences base. */
epic_status epic_plan_layout(const epic_plan_sizes* sizes, int32_t* base, epic_plan* plan);

/* Host only, integer, synchronous: builds the plan (selection of S per
 * LegoLink-k, linked block tables, private blocks with copy sources and slot
 * map, attention tiles and split-KV work items) into host arrays laid out by
 * epic_plan_layout.  free_blocks[0..n_free) must be distinct and must not be
 * chunk blocks; private blocks are taken in order.  Block ids must be
 * < num_blocks (the pool size, used for validation only). */
epic_status epic_plan_link(const epic_link_request* reqs, int32_t batch,
                           const epic_attn_cfg* cfg, const int32_t* free_blocks,
                           int32_t n_free, int32_t num_blocks,
                           const epic_plan_sizes* sizes, epic_plan* plan);

/* Decode over the linked cache (the step after the link: each request appends
 * new tokens after its last linked position and only those are computed).
 * prev / prev_sizes: the host arrays of the previous plan of these requests (the
 * link plan, or the previous decode plan).  new_tokens[b] >= 0 tokens are
 * appended to request b: S = those, at positions n_b .. n_b + t_b - 1 where n_b is
 * the request's linked length in prev.  They fill the request's last block if the
 * previous plan wrote it (a private block) and it has free slots -- that block is
 * its own copy source, so its earlier tokens stay -- and then new blocks taken in
 * order from free_blocks (distinct, not linked by prev).  The new plan links
 * everything prev linked plus the new blocks; it lists as private only the blocks
 * that receive a new token, so epic_link_attention with it (q_s / k_s / v_s of the
 * new tokens) writes nothing else.  Requests that link the same blocks may share work
 * items (see epic_plan), so the parts that a row's softmax is merged from, and with them
 * the last bits of its result, depend on the batch; with kv_split_blocks set, or where the
 * partials of whole shared items would pass EPIC_NOALLOC_SCRATCH_BYTES, each request has
 * items of its own.  Host only, integer, synchronous. */
epic_status epic_plan_decode_sizes(const epic_plan_sizes* prev_sizes, const epic_plan* prev,
                                   const int32_t* new_tokens, const epic_attn_cfg* cfg, int32_t n_free,
                                   epic_plan_sizes* out);
epic_status epic_plan_decode(const epic_plan_sizes* prev_sizes, const epic_plan* prev, const int32_t* new_tokens,
                             const epic_attn_cfg* cfg, const int32_t* free_blocks, int32_t n_free,
                             int32_t num_blocks, const epic_plan_sizes* sizes, epic_plan* plan);

/* Compile step (Sec. 2.2): every chunk is prefilled alone, positions from 0, and
 * its K/V per layer become the chunk's cache.  LegoLink-0 (Sec. 5.4) prepends
 * n_dummy dummy tokens to every chunk for this prefill and drops their K/V, so
 * the cache holds the chunk's L tokens only (token t at block t / bs, offset
 * t % bs), rotated at their compile positions n_dummy + t.
 * chunk_blocks[chunk_block_off[j] .. chunk_block_off[j+1]): the ceil(L_j / bs)
 * blocks that receive chunk j's cache (all distinct).  n_dummy >= 0. */
typedef struct {
  int32_t num_chunks;
  const int32_t* chunk_len;        /* [num_chunks], each >= 1 */
  const int32_t* chunk_block_off;  /* [num_chunks + 1], CSR offsets, [0] == 0 */
  const int32_t* chunk_blocks;     /* physical block ids receiving the caches */
  int32_t n_dummy;                 /* dummy tokens prepended to every chunk (0 = plain compile) */
} epic_compile_batch;

/* Host only, integer, synchronous.  The compile plan has one request per chunk,
 * in order: S = its n_dummy + L_j tokens at positions 0 .. n_dummy + L_j - 1, the
 * dummies first, so the caller's S rows (hidden states) of chunk j are n_dummy
 * dummy rows then the chunk's L_j token rows.  With n_dummy == 0 the linked
 * blocks are the chunk blocks and free_blocks is not used.  With n_dummy > 0
 * the attention reads the n_dummy + L_j tokens from ceil((n_dummy + L_j) / bs)
 * staging blocks per chunk taken in order from free_blocks (distinct, not chunk
 * blocks; EPIC_ERR_NO_PRIVATE_BLOCKS if too few), and the chunk blocks are
 * private blocks outside the linked table that receive rows n_dummy .. (the
 * staging blocks hold the dummy-inclusive K/V afterwards and may be reused).
 * epic_link_model (or epic_link_attention per layer) with this plan is the
 * compile step; s_slot gives the linked (staging) slot of every row. */
epic_status epic_plan_compile_sizes(const epic_compile_batch* batch, const epic_attn_cfg* cfg, int32_t n_free,
                                    epic_plan_sizes* out);
epic_status epic_plan_compile(const epic_compile_batch* batch, const epic_attn_cfg* cfg,
                              const int32_t* free_blocks, int32_t n_free, int32_t num_blocks,
                              const epic_plan_sizes* sizes, epic_plan* plan);

/* Workspace bytes epic_link_attention needs for this plan (split-KV partials). */
size_t epic_link_workspace_bytes(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes);

/* One attention layer of the link step (Sec. 4.2, Eq. 1), on the device:
 *   1. build every private block: copy its source block (if any; K rotated by
 *      priv_rot when that is non-zero, see epic_link_request.rerotate), then
 *      store k_s / v_s of the S rows into their slots (bit-exact copies);
 *   2. for each S row r at linked position p and query head h: softmax over the
 *      linked keys at positions <= p of scale * <q, k>, times V; write out[r, h]
 *      (bf16) and lse[r, h] = natural log of the softmax denominator (fp32).
 * q_s [n_s][Hq][D], k_s / v_s [n_s][Hkv][D] (bf16, ascending S order, already
 * rotated); k_cache / v_cache: the layer's paged caches (layouts above);
 * out [n_s][Hq][D] bf16; lse [n_s][Hq] fp32 or NULL.  plan_dev: plan arrays in
 * device memory.  Empty S: EPIC_OK, nothing launched. */
epic_status epic_link_attention(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes,
                                const epic_plan* plan_dev,
                                const uint16_t* q_s, const uint16_t* k_s, const uint16_t* v_s,
                                uint16_t* k_cache, uint16_t* v_cache,
                                uint16_t* out, float* lse,
                                void* workspace, size_t workspace_bytes, void* stream);

/* epic_link_attention for callers that cannot allocate device memory (code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * steps, kernels and results, with the split-KV partials kept in a fixed array of
 * EPIC_NOALLOC_SCRATCH_BYTES of device memory that the library holds, one copy per
 * GPU, from the time its code is loaded on that GPU until the process ends.  The
 * caller still passes inputs, caches and outputs (as for epic_link_attention); no
 * device memory is allocated or freed by the call.  A plan whose partials need more
 * than EPIC_NOALLOC_SCRATCH_BYTES (epic_link_workspace_bytes) is rejected with
 * EPIC_ERR_WORKSPACE before anything is enqueued (a larger kv_split_blocks gives fewer
 * partials).  Every call on one GPU shares that GPU's array: calls whose work overlaps
 * in time on one GPU (other streams, other threads) race and give wrong results;
 * calls in one stream are ordered and safe.  Nothing in the array needs to start at
 * any value: each call writes every partial it reads. */
#define EPIC_NOALLOC_SCRATCH_BYTES (96u << 20)
epic_status epic_link_attention_noalloc(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes,
                                        const epic_plan* plan_dev,
                                        const uint16_t* q_s, const uint16_t* k_s, const uint16_t* v_s,
                                        uint16_t* k_cache, uint16_t* v_cache,
                                        uint16_t* out, float* lse, void* stream);

/* Profiling hook for callers that time the step's kernels.  events: NULL (off)
 * or 4 hipEvent_t created by the caller; each entry may be NULL.  Until the
 * next call on the same thread, every device entry point records, on its
 * stream, events[0] before the link write, events[1] before the attention
 * kernel, events[2] after it and events[3] after the split-KV combine (per
 * layer for the model entry points; each record overwrites the previous one;
 * where their Q|K|V projection leaves partial sums and nothing is re-rotated, the
 * pass that adds them up writes the private blocks itself, before events[0], so
 * nothing runs between events[0] and events[1].
 * epic_link_attention_kv8 widens the cache for wide tiles before events[1]; few private blocks
 * are written by that launch, or in 16-row tiles by its attention kernel.)
 * Never fails. */
epic_status epic_set_profile_events(void* const* events);

/* ---------------------------------------------------------------- model level */

/* Llama-style decoder (Sec. 5.1 models): pre-norm RMSNorm, rotary embedding
 * (pairs (i, i + D/2), inverse frequency theta^(-2i/D), angles in float64),
 * GQA attention, SwiGLU MLP, final RMSNorm.  hidden % 128 == 0,
 * ffn % 128 == 0 and (Hq + 2 Hkv) D % 128 == 0 are required. */
typedef struct {
  epic_attn_cfg attn;
  int32_t hidden;
  int32_t ffn;
  int32_t n_layers;
  float rope_theta;
  float rms_eps;
} epic_model_cfg;

/* Device pointers to one layer's bf16 weights, [out][in] row-major (y = x W^T):
 *   attn_norm [hidden], wqkv [(Hq + 2 Hkv) D][hidden] (rows: q | k | v),
 *   wo [hidden][Hq D], mlp_norm [hidden], w_gate_up [2 ffn][hidden] (rows: gate | up),
 *   w_down [hidden][ffn]. */
typedef struct {
  const uint16_t* attn_norm;
  const uint16_t* wqkv;
  const uint16_t* wo;
  const uint16_t* mlp_norm;
  const uint16_t* w_gate_up;
  const uint16_t* w_down;
} epic_layer_weights;

/* Workspace bytes for epic_link_layer / epic_link_model with this plan. */
size_t epic_model_workspace_bytes(const epic_model_cfg* cfg, const epic_plan_sizes* sizes);

/* One decoder layer for the S rows (Sec. 4.2 per-layer recipe): hidden_s
 * [n_s][hidden] fp32 residual stream, updated in place; the layer's K/V caches
 * receive the rotated K and the V of every S row (private blocks, as in
 * epic_link_attention). */
epic_status epic_link_layer(const epic_model_cfg* cfg, const epic_layer_weights* w,
                            const epic_plan_sizes* sizes, const epic_plan* plan_dev,
                            float* hidden_s, uint16_t* k_cache, uint16_t* v_cache,
                            void* workspace, size_t workspace_bytes, void* stream);

/* All layers, then the final RMSNorm: out_hidden [n_s][hidden] fp32.
 * layers: host array [n_layers] of device weight pointers; k_caches / v_caches:
 * host arrays [n_layers] of device cache pointers.  hidden_s holds the layer-0
 * rows (embeddings of the S tokens) on entry and is overwritten.
 * The compile step (Sec. 2.2) is this call on a request with no chunks whose
 * suffix is the chunk's tokens: positions 0..L-1, every token computed. */
epic_status epic_link_model(const epic_model_cfg* cfg, const epic_layer_weights* layers,
                            const uint16_t* final_norm,
                            const epic_plan_sizes* sizes, const epic_plan* plan_dev,
                            float* hidden_s, uint16_t* const* k_caches, uint16_t* const* v_caches,
                            float* out_hidden, void* workspace, size_t workspace_bytes,
                            void* stream);

/* ---------------------------------------------------------------- projections */

/* The projection GEMM that epic_link_layer / epic_link_model run for the S rows
 * (Sec. 4.2: Q = E W_Q, K = E W_K, V = E W_V of the selected rows, then the output
 * projection W_O; the model's SwiGLU MLP), on its own:
 *   C[i][j] = sum_t a[i][t] w[j][t]     a: bf16 [m][k]; w: bf16 [n][k] ([out][in]);
 *                                       fp32 accumulation
 * epilogue EPIC_GEMM_STORE:    c[i][j] = C[i][j]                       c: fp32 [m][n]
 *          EPIC_GEMM_RESIDUAL: c[i][j] += C[i][j]                      c: fp32 [m][n], in place
 *          EPIC_GEMM_SWIGLU:   act[i][j] = bf16(silu(C[i][j]) C[i][j + n/2]), j < n/2
 *                              (rows [0, n/2) of w: gate; [n/2, n): up)   act: bf16 [m][n/2]
 * Shapes: m >= 0, k % 64 == 0, n % 128 == 0, and with 256 rows more than m every
 * operand and output below 2^31 bytes; else EPIC_ERR_UNSUPPORTED.
 * Device pointers, 16-byte aligned.  workspace: at least epic_gemm_workspace_bytes()
 * bytes of device memory, 256-byte aligned, owned by the caller; it holds the
 * partial sums of products that are divided along k and the arrival counters of tiles
 * cut along k (cleared by this call), so calls in flight at the same time need separate
 * workspaces.
 * How a product is divided depends on its sizes alone, and its parts are added in a fixed
 * order, so results do not depend on timing:
 *   - whole tiles: one chain of additions in k order (gate and up of few rows: from a k
 *     stage of the tile's own, wrapping); with an fp32 result and less than a round of tiles, a
 *     chain for each of up to a few equal parts of k, added to c one after the other;
 *   - parts of k in separate planes (few rows, or few tiles and a long k): each part in one
 *     to four chains over its k slices, the parts in k order;
 *   - tiles cut along k: the part that holds the tile's last k stage first, then the others
 *     in k order.  The environment variable EPIC_GEMM_FINISH_POLLS (read at each launch,
 *     default 4096) bounds how long that last part's workgroup polls for the others before
 *     falling back to the last-to-arrive protocol; 0 forces the fallback (a test hook; the
 *     sums are the same either way).
 * Enqueued on `stream` (NULL: the default stream); returns after the enqueue. */
typedef enum { EPIC_GEMM_STORE = 0, EPIC_GEMM_RESIDUAL = 1, EPIC_GEMM_SWIGLU = 2 } epic_gemm_epilogue;
size_t epic_gemm_workspace_bytes(void);
epic_status epic_gemm(int32_t epilogue, const uint16_t* a, const uint16_t* w, int32_t m, int32_t n, int32_t k,
                      float* c, uint16_t* act, void* workspace, size_t workspace_bytes, void* stream);

/* ---------------------------------------------------------------- 8-bit projections */

/* The decoder layer's projections on 8-bit operands: e4m3 values (1-4-3 bits, largest 448,
 * no infinities) with one power-of-two scale per 128 values, an e8m0 byte (2^(byte - 127)),
 * which the matrix instruction applies.  For a group of values y, t is the smallest
 * integer in [-127, 127] with max |y| <= 448 * 2^t, over the finite y (t = 0 if all of them
 * are 0); the scale's byte is t + 127 and the values are y / 2^t rounded once, to nearest
 * even.  Infinities and NaN become NaN.
 *  - Rows: values [m][k], a scale per 128 consecutive values of a row, laid out
 *    [k / 128][m rounded up to 4] (a group's scales of all rows are contiguous; the padding
 *    is never used and may be written).  epic_fp8_scale_bytes(m, k) bytes (0 if m < 0 or
 *    k is not a positive multiple of 128).
 *  - Weights: values [n][k] ([out][in]), a scale per 128 x 128 block, [ceil(n / 128)][k / 128].
 * All of it contiguous device memory, k % 128 == 0; values 16-byte, row scales 4-byte
 * aligned.  Every call is deterministic: sums have a fixed order for given sizes. */
size_t epic_fp8_scale_bytes(int32_t m, int32_t k);

/* Round x (bf16 [m][k]) to q and scale: as rows (block_rows == 1), or as weights
 * (block_rows == 128; the last block may have fewer rows).  Up to 2^35 - 2^13 values, and 65535
 * blocks of rows; more are EPIC_ERR_UNSUPPORTED (a launch has fewer than 2^32 threads). */
epic_status epic_quant_fp8(const uint16_t* x, int32_t m, int32_t k, int32_t block_rows, uint8_t* q, uint8_t* scale,
                           void* stream);

/* The residual stream's addition, RMSNorm and rounding in one pass:
 *   s = x + delta;   y = s / sqrt(mean(s^2) + eps) * weight;   y -> q, scale (rows)
 * x, x_out: fp32 [m][hidden]; delta: bf16 [m][hidden] (a product of epic_gemm_fp8, say), or
 * NULL for none; weight: bf16 [hidden].  x_out receives s unless it is NULL; it may be x,
 * and else overlaps nothing.  Sums and statistics are fp32.  hidden % 128 == 0, at most
 * 32768; up to 2^22 - 1 rows at any such width (2^23 - 2 up to 16384 wide), for the same reason. */
epic_status epic_rmsnorm_fp8(const float* x, const uint16_t* delta, const uint16_t* weight, int32_t m, int32_t hidden,
                             float eps, float* x_out, uint8_t* q, uint8_t* scale, void* stream);

/* The projection GEMM on 8-bit rows a and weights w:
 *   C[i][j] = sum over blocks b of 2^(a_scale[i][b] + w_scale[j / 128][b]) sum over t in b of a[i][t] w[j][t]
 * epilogue EPIC_FP8_BF16:       out bf16 [m][n] = C
 *          EPIC_FP8_SWIGLU:     out bf16 [m][n/2] = silu(C[i][j]) C[i][j + n/2]
 *          EPIC_FP8_SWIGLU_FP8: the same as rows, out e4m3 [m][n/2] and out_scale (else unused)
 * Sums are fp32, but of each eight neighbouring t (all with t / 8 alike) the matrix cores drop
 * what lies more than 13 bits below the largest product: up to 7 * 2^-13 of that product.  With
 * operands of independent signs this is 1.5e-5 to 4e-5 of the results' 2-norm, below what
 * rounding to bf16 or e4m3 costs.  Where large products of the same eight cancel (448 w - 448 w
 * beside products of w), it is measured against those, not against what they leave: 1e-2 of the
 * results' norm then, still below the 2^-4 of each large product that e4m3 operands are rounded by.
 * Where the largest value of a group of the quantised result, summed like that, is within 2^-12 of
 * where its scale changes, its 64-bit sum decides.  The scale is that of the exact sums then,
 * unless the group's sums cancel as above, or another of its values is as near to the same place.
 * Shapes: m >= 0, k % 128 == 0, n % 128 == 0 (SwiGLU: n % 256 == 0), and with 256 rows more
 * than m every operand and a bf16 [m][n] below 2^31 bytes; else EPIC_ERR_UNSUPPORTED.
 * workspace: epic_gemm_fp8_workspace_bytes() bytes, 256-byte
 * aligned, for partial sums; calls in flight at the same time need separate ones. */
typedef enum { EPIC_FP8_BF16 = 0, EPIC_FP8_SWIGLU = 1, EPIC_FP8_SWIGLU_FP8 = 2 } epic_fp8_epilogue;
size_t epic_gemm_fp8_workspace_bytes(void);
epic_status epic_gemm_fp8(int32_t epilogue, const uint8_t* a, const uint8_t* a_scale, const uint8_t* w,
                          const uint8_t* w_scale, int32_t m, int32_t n, int32_t k, void* out, uint8_t* out_scale,
                          void* workspace, size_t workspace_bytes, void* stream);

/* One layer's weights for the 8-bit projections: norms bf16, the matrices of
 * epic_layer_weights as e4m3 with block scales (epic_quant_fp8, block_rows 128). */
typedef struct {
  const uint16_t* attn_norm;
  const uint8_t* wqkv;
  const uint8_t* wqkv_scale;
  const uint8_t* wo;
  const uint8_t* wo_scale;
  const uint16_t* mlp_norm;
  const uint8_t* w_gate_up;
  const uint8_t* w_gate_up_scale;
  const uint8_t* w_down;
  const uint8_t* w_down_scale;
} epic_layer_weights_fp8;

/* epic_link_layer and epic_link_model with their projections on 8-bit operands: the same
 * plans, caches (bf16), residual stream and outputs (fp32).  The norms' outputs, the
 * attention's and the SwiGLU's are rounded to e4m3 per 128 values before the product that
 * reads them; W_O's and W_down's products of many rows are added to the stream in bf16.
 * Hq * head_dim % 128 == 0 and hidden <= 32768 are required besides what epic_model_cfg asks. */
size_t epic_model_fp8_workspace_bytes(const epic_model_cfg* cfg, const epic_plan_sizes* sizes);
epic_status epic_link_layer_fp8(const epic_model_cfg* cfg, const epic_layer_weights_fp8* w,
                                const epic_plan_sizes* sizes, const epic_plan* plan_dev,
                                float* hidden_s, uint16_t* k_cache, uint16_t* v_cache,
                                void* workspace, size_t workspace_bytes, void* stream);
epic_status epic_link_model_fp8(const epic_model_cfg* cfg, const epic_layer_weights_fp8* layers,
                                const uint16_t* final_norm,
                                const epic_plan_sizes* sizes, const epic_plan* plan_dev,
                                float* hidden_s, uint16_t* const* k_caches, uint16_t* const* v_caches,
                                float* out_hidden, void* workspace, size_t workspace_bytes,
                                void* stream);

/* ---------------------------------------------------------------- head norm and rotation */

/* Rotary positions.  The first rot_dim dims of a head (a multiple of 16, at most head_dim; 0: none)
 * are rot_dim / 2 pairs j: dims (j, j + rot_dim / 2), or (2 j, 2 j + 1) where interleaved == 1.
 * Pair j turns by pos * f_j:
 *   f_j = theta^(-2 j / rot_dim) * (keep_j + (1 - keep_j) / factor)
 * keep_j = 0 where original_context == 0 (every frequency divided by factor), else, with
 * turns_j = original_context * theta^(-2 j / rot_dim) / 2 pi the turns that pair j makes over the
 * context the model was trained on, 0 up to low_turns, 1 from high_turns, and linear between.
 * amplitude multiplies the rotated pairs.  factor == 0 and amplitude == 0 stand for 1.
 * Plans that re-rotate cached keys (epic_link_request.rerotate) turn the whole head, pairs
 * (j, j + D / 2), by offset * rope_theta^(-2 j / D) of epic_attn_cfg, however the keys were made;
 * nothing tells it from the keys.  Such plans are for keys of rot_dim == head_dim, interleaved == 0,
 * factor 1 and theta == rope_theta, with any amplitude and norm; keys of other forms would come
 * out wrong. */
typedef struct {
  int32_t rot_dim;
  int32_t interleaved;
  float theta;
  float factor;
  int32_t original_context;
  float low_turns;
  float high_turns;
  float amplitude;
} epic_rope_cfg;

/* Host only: freqs[rot_dim / 2] = f_j (float64, radians a position).  A caller uploads them once. */
epic_status epic_rope_freqs(const epic_rope_cfg* rope, double* freqs);

/* What stands between the Q|K|V product and the attention, in one pass: of every row, each query
 * and key head is normed (y = x / sqrt(mean(x^2) + eps) * w, where its weight is given) and its
 * first rot_dim dims are rotated at the row's position; V passes.  In fp32, from float64 angles,
 * rounded to bf16 once.
 * qkv: rows of q | k | v heads, (Hq + 2 Hkv) D values, ld values apart (a multiple of 16 bytes),
 * in_type EPIC_QKV_BF16 (as epic_gemm_fp8 leaves them) or EPIC_QKV_FP32 (as epic_gemm does);
 * pos [rows] (a plan's s_pos, say); freqs [rot_dim / 2] of epic_rope_freqs, in device memory (may
 * be NULL where rot_dim == 0); q_norm, k_norm: bf16 [D] or NULL for no norm; q [rows][Hq][D], k, v
 * [rows][Hkv][D] bf16, as epic_link_attention and epic_link_attention_kv8 take them.  Device
 * pointers, 16-byte aligned (freqs 8); no two of input and outputs overlap.  Up to 2^24 - 4 rows. */
typedef enum { EPIC_QKV_BF16 = 0, EPIC_QKV_FP32 = 1 } epic_qkv_type;
epic_status epic_qk_norm_rope(const epic_attn_cfg* cfg, const epic_rope_cfg* rope, int32_t in_type, const void* qkv,
                              int64_t ld, int32_t rows, const int32_t* pos, const double* freqs,
                              const uint16_t* q_norm, const uint16_t* k_norm, float eps, uint16_t* q, uint16_t* k,
                              uint16_t* v, void* stream);

/* ---------------------------------------------------------------- cache in 8 bits */

/* A paged cache of one layer in 8 bits, 0.51 of the bf16 one: blocks of 16 tokens; a row (the D
 * values of K, or of V, of a token and KV head) is e4m3 values and one e8m0 byte by the rule of
 * the 8-bit projections, t the smallest integer in [-127, 127] with max |y| <= 448 * 2^t.  A token
 * of which a value of K or V is not finite is NaN: both bytes 255.
 *   k      [num_blocks][Hkv][D / 64][4][16][16]     dim 64 j + 16 a + e of token s at [j][a][s][e]
 *   v      [num_blocks][Hkv][D / 64][4][16][4][4]   dim 64 j + 16 t + r of token 4 a + c at [j][a][r][t][c]
 *   scale  [num_blocks][Hkv][2][16]                 bytes of K, of V
 * (the order in which the matrix cores take the values).  Device memory, 16-byte aligned.  In a
 * cache that is written other than by this library, NaN tokens hold K all 0x7F and V all 0, and
 * other tokens no NaN codes. */
typedef struct {
  uint8_t* k;
  uint8_t* v;
  uint8_t* scale;
  int32_t num_blocks;
} epic_kv8_cache;

/* Blocks of a bf16 cache (k_cache, v_cache: the layouts above, num_blocks blocks) to blocks of an
 * 8-bit one, and back: src_blocks[i] into dst_blocks[i], i < n, whole blocks.  Lists in device
 * memory; NULL stands for 0 .. n - 1.  The blocks of dst_blocks are distinct.  An entry with an id
 * outside its pool moves nothing.  Back is exact, but for results outside bf16's range; NaN tokens
 * are NaN in K and V. */
epic_status epic_kv8_pack(const epic_attn_cfg* cfg, int32_t n, const int32_t* src_blocks, const uint16_t* k_cache,
                          const uint16_t* v_cache, int32_t num_blocks, const int32_t* dst_blocks,
                          const epic_kv8_cache* cache, void* stream);
epic_status epic_kv8_unpack(const epic_attn_cfg* cfg, int32_t n, const int32_t* src_blocks, const epic_kv8_cache* cache,
                            const int32_t* dst_blocks, uint16_t* k_cache, uint16_t* v_cache, int32_t num_blocks,
                            void* stream);

/* epic_link_attention over an 8-bit cache, with any plan (link, decode, compile):
 *   1. every private block takes its source's bytes (K of re-rotated blocks: turned in fp32 and
 *      rounded to 8 bits again; see epic_rope_cfg for the keys that these may hold), then the S rows k_s / v_s, rounded; a slot with neither holds zeros;
 *   2. attention as there, over the values that the cache now holds, with fp32 sums (V of 2^119 and
 *      more may overflow them), P rounded to bf16 (in 16-row tiles times the scale of V: probabilities of
 *      tokens whose V stays below some 2^-102 lose bits there).  A row that attends to a NaN token has NaN in
 *      out, and its lse means nothing; NaN in tokens after a row, or in slots past a block's
 *      tokens, does not reach it.
 * q_s, k_s, v_s, out, lse as there.  workspace: epic_link_kv8_workspace_bytes() bytes (0 without
 * split-KV partials and wide tiles), 16-byte aligned; calls in flight at the same time need separate
 * ones.  Plans of wide tiles (128 or 256 rows) keep their linked blocks in it in bf16, 64 D Hkv
 * bytes for each entry of the linked table, for the time of the call.  That widening is a copy of the
 * linked cache, so plans of few new rows over long caches are better made with tile_rows = 16 here: of one
 * request over 131 072 cached keys of 8 heads of 128, 16 new rows of 32 heads take 88 us so, 290 by default (bf16
 * cache: 135), 32 rows 149 and 294.
 * The last bits of a row's result depend on the batch here too, by what its plan shares and splits and
 * by how many private blocks it writes.
 * The plan's block ids are below cache->num_blocks. */
size_t epic_link_kv8_workspace_bytes(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes);
epic_status epic_link_attention_kv8(const epic_attn_cfg* cfg, const epic_plan_sizes* sizes, const epic_plan* plan_dev,
                                    const uint16_t* q_s, const uint16_t* k_s, const uint16_t* v_s,
                                    const epic_kv8_cache* cache, uint16_t* out, float* lse, void* workspace,
                                    size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* EPIC_LINK_H */

// The decoder layer and the model on 8-bit projections.
//
// The layer of model.cpp with its four products on e4m3 operands (gemm8.h):
//   x = RMSNorm(h) w_attn                       e4m3 + scales
//   q, k, v = x Wqkv^T, q and k rotated           bf16, as in model.cpp
//   link write + attention over K_exp / V_exp    bf16; o rounded to e4m3
//   h += o Wo^T                                  with the next norm
//   x = RMSNorm(h) w_mlp                          e4m3
//   act = silu(x Wg^T) * (x Wu^T)                 e4m3, from the product's epilogue
//   h += act Wd^T                                with the next norm
// The residual stream stays fp32.  What W_O and W_down add to it arrives as partial sums in
// fp32 planes (few rows), which the next norm adds, or as one bf16 product.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "gemm8.h"
#include "kernels.h"
#include "model_internal.h"
#include "plan_internal.h"
#include "quant.h"
#include "status.h"

using namespace epic;

namespace {

size_t align256(size_t n) { return (n + 255) & ~size_t(255); }

struct Rows8 {
  uint8_t *q, *scale;
};

struct LayerWs8 {
  Rows8 x, o8, act;  // [n_s][hidden], [n_s][hq D], [n_s][ffn]
  uint16_t* q;       // [n_s][hq][D]
  uint16_t* k;       // [n_s][hkv][D]
  uint16_t* v;       // [n_s][hkv][D]
  uint16_t* o;       // [n_s][hq D]
  uint16_t* delta;   // [n_s][hidden]: W_O's or W_down's product
  float2* cs;        // [n_s][D/2]
  void* attn;        // split-KV partials
  float* partial;    // planes of partial sums
  size_t total;
};

LayerWs8 carve(const epic_model_cfg* c, const epic_plan_sizes* s, char* base) {
  const size_t n = size_t(s->n_s), ld = scale_ld(s->n_s);
  const size_t qd = size_t(c->attn.num_q_heads) * c->attn.head_dim, kd = size_t(c->attn.num_kv_heads) * c->attn.head_dim;
  LayerWs8 w{};
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* p = base ? base + off : nullptr;
    off += align256(bytes);
    return p;
  };
  auto rows = [&](size_t k) {
    Rows8 r;
    r.q = reinterpret_cast<uint8_t*>(take(n * k));
    r.scale = reinterpret_cast<uint8_t*>(take(k / kGroup * ld));
    return r;
  };
  w.x = rows(c->hidden);
  w.o8 = rows(qd);
  w.act = rows(c->ffn);
  w.q = reinterpret_cast<uint16_t*>(take(n * qd * 2));
  w.k = reinterpret_cast<uint16_t*>(take(n * kd * 2));
  w.v = reinterpret_cast<uint16_t*>(take(n * kd * 2));
  w.o = reinterpret_cast<uint16_t*>(take(n * qd * 2));
  w.delta = reinterpret_cast<uint16_t*>(take(n * c->hidden * 2));
  w.cs = reinterpret_cast<float2*>(take(n * size_t(c->attn.head_dim / 2) * 8));
  w.attn = take(epic_link_workspace_bytes(&c->attn, s));
  w.partial = reinterpret_cast<float*>(take(kPartial8Bytes));
  w.total = off;
  return w;
}

epic_status validate_fp8(const epic_model_cfg* c) {
  epic_status st = validate_model(c);
  if (st != EPIC_OK) return st;
  if (c->attn.num_q_heads * c->attn.head_dim % kGroup != 0)
    return fail(EPIC_ERR_UNSUPPORTED, "Hq * D must be a multiple of %d", kGroup);
  if (c->hidden > kMaxNormHidden) return fail(EPIC_ERR_UNSUPPORTED, "hidden %d above %d", c->hidden, kMaxNormHidden);
  return EPIC_OK;
}

epic_status check_weights(const epic_layer_weights_fp8* w) {
  EPIC_CHECK_ARG(w != nullptr, "layer weights are NULL");
  EPIC_CHECK_ARG(w->attn_norm && w->wqkv && w->wqkv_scale && w->wo && w->wo_scale && w->mlp_norm && w->w_gate_up &&
                     w->w_gate_up_scale && w->w_down && w->w_down_scale,
                 "a layer weight pointer is NULL");
  auto al = [](const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; };
  EPIC_CHECK_ARG(al(w->attn_norm) && al(w->wqkv) && al(w->wo) && al(w->mlp_norm) && al(w->w_gate_up) && al(w->w_down),
                 "norms and weight values must be 16-byte aligned");
  return EPIC_OK;
}

epic_status check_call(const epic_model_cfg* c, const epic_plan_sizes* s, const epic_plan* p, const float* h, void* ws,
                       size_t ws_bytes) {
  epic_status st = validate_fp8(c);
  if (st == EPIC_OK) st = check_model_call(c, s, p, h);
  if (st != EPIC_OK || s->n_s == 0) return st;
  // 31-bit byte offsets: operands and results, rows padded to a whole 256-row tile
  const int64_t rows = int64_t(s->n_s) + 256, lim = int64_t(1) << 31;
  const int64_t qkv_n = int64_t(c->attn.num_q_heads + 2 * c->attn.num_kv_heads) * c->attn.head_dim;
  const int64_t qd = int64_t(c->attn.num_q_heads) * c->attn.head_dim;
  if (rows * std::max<int64_t>(std::max(c->hidden, c->ffn), qd) >= lim || rows * std::max<int64_t>(qkv_n, c->hidden) * 2 >= lim ||
      rows * c->ffn * 2 >= lim || int64_t(2) * c->ffn * c->hidden >= lim || qkv_n * c->hidden >= lim)
    return fail(EPIC_ERR_UNSUPPORTED, "%d rows or the weights exceed the 2^31-byte GEMM operand limit", s->n_s);
  return check_workspace(ws, ws_bytes, carve(c, s, nullptr).total);
}

// What is still to be added to the residual stream: planes, a bf16 product, or nothing.
struct Pending {
  StreamSum planes;
  const uint16_t* delta;
};

Gemm8Args product(const Rows8& a, const uint8_t* w, const uint8_t* sw, int m, int n, int k, float* partial) {
  Gemm8Args g{};
  g.A = a.q, g.sa = a.scale, g.W = w, g.sw = sw, g.M = m, g.N = n, g.K = k, g.partial = partial;
  return g;
}

// The product, left pending for the norm that follows.
Pending residual_product(Gemm8Args g, uint16_t* delta, hipStream_t stream) {
  const Gemm8Plan p = gemm8_plan(g.M, g.N, g.K, kBf16Out);
  const bool whole = p.kind == Gemm8Kind::kWhole || p.kind == Gemm8Kind::kNarrow;
  if (!whole) return Pending{launch_gemm8_partial(g, p, stream), nullptr};
  g.out = delta;
  if (p.kind == Gemm8Kind::kNarrow) launch_gemm8_narrow(g, kBf16Out, p.tm, p.tn, stream);
  else launch_gemm8_wide(g, kBf16Out, p.tm, stream);
  return Pending{StreamSum{}, delta};
}

// h += what is pending.
void settle(Pending* p, float* h, int n, int hidden, hipStream_t stream) {
  if (p->planes.partial != nullptr) {
    GemmArgs g{};
    g.C = h;
    launch_stream_finish(p->planes, g, kResidual, stream);
  } else if (p->delta != nullptr) {
    launch_add_bf16(h, p->delta, size_t(n) * hidden, stream);
  }
  *p = Pending{};
}

// x = RMSNorm(h + pending) w, h updated.
void add_norm(Pending* p, float* h, const uint16_t* w, const Rows8& x, int n, int hidden, float eps, hipStream_t stream) {
  const bool adds = p->planes.partial != nullptr || p->delta != nullptr;
  launch_rmsnorm_fp8(h, p->delta, p->planes, w, n, hidden, eps, adds ? h : nullptr, x.q, x.scale, stream);
  *p = Pending{};
}

// One layer; the rotary table ws.cs is already filled.  pending: the last layer's W_down
// product on entry, this layer's on return.
epic_status run_layer(const epic_model_cfg* c, const epic_layer_weights_fp8* w, const epic_plan_sizes* s,
                      const epic_plan* p, float* h, uint16_t* kc, uint16_t* vc, const LayerWs8& ws, Pending* pending,
                      hipStream_t stream) {
  const int n = s->n_s, H = c->hidden, F = c->ffn;
  const int hq = c->attn.num_q_heads, hkv = c->attn.num_kv_heads, D = c->attn.head_dim;
  add_norm(pending, h, w->attn_norm, ws.x, n, H, c->rms_eps, stream);

  // partial sums of Q|K|V go straight into the private blocks
  Gemm8Args qkv = product(ws.x, w->wqkv, w->wqkv_scale, n, (hq + 2 * hkv) * D, H, ws.partial);
  qkv.q = ws.q, qkv.k = ws.k, qkv.v = ws.v, qkv.cs = ws.cs, qkv.hq = hq, qkv.hkv = hkv, qkv.head_dim = D;
  const Gemm8Plan qp = gemm8_plan(n, qkv.N, H, kRopeOut);
  const bool partial = qp.kind != Gemm8Kind::kWhole, write = partial && s->n_rerotated == 0;
  if (partial) {
    const StreamSum sum = launch_gemm8_partial(qkv, qp, stream);
    GemmArgs g{};
    g.q = ws.q, g.k = ws.k, g.v = ws.v, g.cs = ws.cs, g.hq = hq, g.hkv = hkv, g.head_dim = D;
    if (write)
      launch_stream_rope_write(sum, g, StreamWrite{p->priv_block, p->priv_src, p->priv_rows, s->n_private, kc, vc}, stream);
    else
      launch_stream_finish(sum, g, kRope, stream);
  } else {
    launch_gemm8_wide(qkv, kRopeOut, qp.tm, stream);
  }
  epic_attn_cfg ac = c->attn;
  ac.rope_theta = c->rope_theta;            // cached K was rotated with the model's base
  epic_status st = run_link_attention(&ac, s, p, ws.q, write ? nullptr : ws.k, write ? nullptr : ws.v, kc, vc, ws.o,
                                      nullptr, ws.attn, stream);
  if (st != EPIC_OK) return st;
  launch_quant_rows(ws.o, n, hq * D, ws.o8.q, ws.o8.scale, stream);
  *pending = residual_product(product(ws.o8, w->wo, w->wo_scale, n, H, hq * D, ws.partial), ws.delta, stream);
  add_norm(pending, h, w->mlp_norm, ws.x, n, H, c->rms_eps, stream);
  Gemm8Args gu = product(ws.x, w->w_gate_up, w->w_gate_up_scale, n, 2 * F, H, ws.partial);
  gu.out = ws.act.q, gu.out_scale = ws.act.scale;
  launch_gemm8(gu, kGluQuantOut, stream);
  *pending = residual_product(product(ws.act, w->w_down, w->w_down_scale, n, H, F, ws.partial), ws.delta, stream);
  return hip_ok("decoder layer launch");
}

}  // namespace

extern "C" size_t epic_model_fp8_workspace_bytes(const epic_model_cfg* cfg, const epic_plan_sizes* sizes) {
  if (!cfg || !sizes || validate_fp8(cfg) != EPIC_OK) return 0;
  return carve(cfg, sizes, nullptr).total;
}

extern "C" epic_status epic_link_layer_fp8(const epic_model_cfg* cfg, const epic_layer_weights_fp8* w,
                                           const epic_plan_sizes* sizes, const epic_plan* plan_dev, float* hidden_s,
                                           uint16_t* k_cache, uint16_t* v_cache, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  clear_error();
  epic_status st = check_call(cfg, sizes, plan_dev, hidden_s, workspace, workspace_bytes);
  if (st != EPIC_OK) return st;
  if (sizes->n_s == 0) return link_write_only(cfg, sizes, plan_dev, &k_cache, &v_cache, 1, stream);
  st = check_weights(w);
  if (st != EPIC_OK) return st;
  EPIC_CHECK_ARG(k_cache && v_cache, "KV cache pointers are NULL");
  hipStream_t s = static_cast<hipStream_t>(stream);
  const LayerWs8 ws = carve(cfg, sizes, static_cast<char*>(workspace));
  launch_rope_table(plan_dev->s_pos, ws.cs, sizes->n_s, cfg->attn.head_dim, cfg->rope_theta, s);
  Pending pending{};
  st = run_layer(cfg, w, sizes, plan_dev, hidden_s, k_cache, v_cache, ws, &pending, s);
  if (st != EPIC_OK) return st;
  settle(&pending, hidden_s, sizes->n_s, cfg->hidden, s);
  return hip_ok("decoder layer launch");
}

extern "C" epic_status epic_link_model_fp8(const epic_model_cfg* cfg, const epic_layer_weights_fp8* layers,
                                           const uint16_t* final_norm, const epic_plan_sizes* sizes,
                                           const epic_plan* plan_dev, float* hidden_s, uint16_t* const* k_caches,
                                           uint16_t* const* v_caches, float* out_hidden, void* workspace,
                                           size_t workspace_bytes, void* stream) {
  clear_error();
  epic_status st = check_call(cfg, sizes, plan_dev, hidden_s, workspace, workspace_bytes);
  if (st != EPIC_OK) return st;
  if (sizes->n_s == 0) return link_write_only(cfg, sizes, plan_dev, k_caches, v_caches, cfg->n_layers, stream);
  EPIC_CHECK_ARG(layers && k_caches && v_caches && final_norm && out_hidden, "NULL model argument");
  for (int l = 0; l < cfg->n_layers; ++l) {
    st = check_weights(&layers[l]);
    if (st != EPIC_OK) return st;
    EPIC_CHECK_ARG(k_caches[l] && v_caches[l], "layer %d: KV cache pointers are NULL", l);
  }
  hipStream_t s = static_cast<hipStream_t>(stream);
  const LayerWs8 ws = carve(cfg, sizes, static_cast<char*>(workspace));
  launch_rope_table(plan_dev->s_pos, ws.cs, sizes->n_s, cfg->attn.head_dim, cfg->rope_theta, s);
  Pending pending{};
  for (int l = 0; l < cfg->n_layers; ++l) {
    st = run_layer(cfg, &layers[l], sizes, plan_dev, hidden_s, k_caches[l], v_caches[l], ws, &pending, s);
    if (st != EPIC_OK) return st;
  }
  if (pending.planes.partial != nullptr) {
    launch_rmsnorm_sum(pending.planes, hidden_s, final_norm, nullptr, out_hidden, cfg->rms_eps, s);
  } else {
    settle(&pending, hidden_s, sizes->n_s, cfg->hidden, s);
    launch_rmsnorm(hidden_s, final_norm, nullptr, out_hidden, sizes->n_s, cfg->hidden, cfg->rms_eps, s);
  }
  return hip_ok("final norm launch");
}

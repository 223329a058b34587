"""The decoder layer and the model on 8-bit projections (epic_link_layer_fp8, epic_link_model_fp8).

Against the oracle (oracle.fp8.decoder_layer), a layer at a time on the same inputs:
  - recomputed K and V in the cache: the norm's e4m3 rows agree but for values within 2^-20 of a
    border of rounding (one in about 2^16, each a step of 2^-3 of one of `hidden` inputs); the
    product's dropped bits (2^-12 of its 2-norm) and the rounding to bf16 (2^-9 rms at most)
    follow: 2-norm within 2^-8.
  - what a layer adds to the stream: o differs by about 2^-8 (bf16 attention weights and its own
    rounding), so e4m3's steps (up to 2^-3) round otherwise for at most that share of a step,
    sqrt(2^-8 * 2^-3) = 2.2% rms; the MLP's input, SwiGLU output and products carry that on:
    2-norm within 6%.  A wrong scale, row or weight is off by its whole size.
The model and the layers on their own, and replays of a captured call, agree bit for bit.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle  # noqa: E402
import synth  # noqa: E402
from oracle import fp8  # noqa: E402
from synth.configs import ModelWorkload  # noqa: E402
from test_gpu_model import _bits, _f64, _linked_rows, _s_embeddings  # noqa: E402

pytestmark = pytest.mark.gpu


def _wl(name, lens, suffix, k, hidden=512, ffn=1024, hq=8, hkv=2, d=64, layers=2, seed=51):
    return ModelWorkload(name, seed, layers, hidden, ffn, hq, hkv, d, 16, 500000.0, 1e-5, lens, suffix, k)


# both head dims, an odd number of KV heads, heads of k and v in one tile; with the kernels of the
# Q|K|V product (its epilogue or its consumer rotates) and of the others (checked in test_fp8.py)
CASES = [
    _wl("streamed_d64", [37, 100, 16, 51], 23, 5),
    _wl("streamed_d128", [64, 45], 30, 16, ffn=1536, hq=4, hkv=2, d=128),
    _wl("one_row", [40], 1, 0, hidden=256, ffn=512, hq=4, hkv=4),
    _wl("split_d128", [200, 100], 150, 100, hidden=4096, ffn=1024, hq=8, hkv=2, d=128, layers=1),
    _wl("whole_d128", [700, 300], 250, 250, hidden=256, ffn=768, hq=4, hkv=2, d=128),
    _wl("whole_d64", [700, 300], 250, 250, hidden=384, ffn=512, hq=6, hkv=3),
    _wl("whole_crossing_heads", [400, 200], 150, 200, hidden=256, ffn=512, hq=2, hkv=1),
    _wl("whole192_d128", [64], 2049, 0, hidden=384, ffn=512, hq=16, hkv=8, d=128, layers=1),
    _wl("whole192_d64", [30], 2049, 0, hidden=384, ffn=512, hq=32, hkv=16, layers=1),
    _wl("whole256_d128", [64], 2049, 0, hidden=384, ffn=512, hq=32, hkv=8, d=128, layers=1),
    _wl("whole256_d64", [30], 2049, 0, hidden=384, ffn=512, hq=64, hkv=16, layers=1),
]
QKV = ["stream", "stream", "few", "split128", "whole128", "whole128", "whole128", "whole192", "whole192", "whole256", "whole256"]


def _stage(wl, **kw):
    from paper_2410_15332_amd import harness
    print(f"[gpu-test] fp8 model {wl.name} {kw}", flush=True)
    return harness.stage_model(wl, fp8=True, **kw)


def _layer_call(st, layer, hidden):
    from paper_2410_15332_amd import epic_link as el
    el.epic_link_layer_fp8(st.cfg, st.layers[layer], st.dplan, hidden, st.k_caches[layer], st.v_caches[layer],
                           st.workspace)


def _norm(x):
    return float(np.linalg.norm(x))


@pytest.mark.parametrize("wl", CASES, ids=[w.name for w in CASES])
def test_layers_against_the_oracle(wl):
    st = _stage(wl, caches="synthetic")
    s_pos = oracle.legolink_positions(wl.chunk_lens, wl.suffix_len, wl.k)
    hq, hkv, d = wl.num_q_heads, wl.num_kv_heads, wl.head_dim
    st.hidden.copy_(st.emb)
    for layer in range(wl.n_layers):
        caches = [synth.chunk_cache(wl.seed, j, n, hkv, d, 0.5, layer=layer) for j, n in enumerate(wl.chunk_lens)]
        h_in = st.hidden.double().cpu().numpy()
        _layer_call(st, layer, st.hidden)
        torch.cuda.synchronize()
        w = fp8.weights(synth.model_weights(wl.seed, layer, wl.hidden, wl.ffn, hq, hkv, d))
        h, k, v, added = fp8.decoder_layer(h_in, s_pos, w, [_f64(c[0]) for c in caches], [_f64(c[1]) for c in caches],
                                           wl.linked_len, wl.ffn, hq, hkv, d, wl.rope_theta, wl.rms_eps)
        gk, gv = _linked_rows(st, layer, s_pos)
        ek, ev = _norm(gk - k) / _norm(k), _norm(gv - v) / _norm(v)
        eh = _norm(st.hidden.double().cpu().numpy() - h) / _norm(added[0] + added[1])
        print(f"[gpu-test] layer {layer}: k {ek:.2e} v {ev:.2e} added {eh:.2e}", flush=True)
        assert ek <= 2.0 ** -8 and ev <= 2.0 ** -8 and eh <= 0.06


@pytest.mark.parametrize("wl", CASES, ids=[w.name for w in CASES])
def test_model_is_its_layers(wl):
    st = _stage(wl, caches="compile")
    st.run()
    torch.cuda.synchronize()
    out, k = st.out.clone(), [c.clone() for c in st.k_caches]
    st.hidden.copy_(st.emb)
    for layer in range(wl.n_layers):
        _layer_call(st, layer, st.hidden)
    h = st.hidden.double()
    ref = h * torch.rsqrt(h.square().mean(-1, keepdim=True) + wl.rms_eps) * st.final_norm.double()
    assert all(torch.equal(a, b) for a, b in zip(k, st.k_caches))
    assert bool(((out - ref).abs() <= 2.0 ** -20 * ref.abs()).all())


@pytest.mark.parametrize("wl", [CASES[0], CASES[2], CASES[4]], ids=lambda w: w.name)
def test_replays_of_a_captured_call(wl):
    from paper_2410_15332_amd import harness
    st = _stage(wl, caches="compile")
    st.run()
    torch.cuda.synchronize()
    ref = [st.out.clone(), st.k_caches[1].clone()]
    graph = harness.capture_graph(st.run)
    for _ in range(3):
        st.out.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(ref[0], st.out) and torch.equal(ref[1], st.k_caches[1])
        st.run()                                            # an eager step between replays
        torch.cuda.synchronize()


def test_near_the_bf16_model():
    """Compile and link in 8 bits against the same model in bf16: e4m3's rounding, 2^-4 at most and
    about 2^-5.5 rms on each operand of four products a layer, independent between values: the
    rows of the last hidden state agree to a tenth in 2-norm, and point the same way."""
    from paper_2410_15332_amd import harness
    wl = CASES[0]
    a, b = harness.stage_model(wl, caches="compile"), _stage(wl, caches="compile")
    a.run()
    b.run()
    torch.cuda.synchronize()
    x, y = a.out.double(), b.out.double()
    off = float((x - y).norm() / x.norm())
    print(f"[gpu-test] fp8 against bf16 model: {off:.3f}", flush=True)
    assert off <= 0.1
    assert float(torch.cosine_similarity(x, y, -1).min()) > 0.99


def test_re_rotated_chunks():
    """Private copies of re-rotated chunks take the other write path; with n_s = 0 they are all there is."""
    from paper_2410_15332_amd import epic_link as el
    wl = CASES[0]
    st = _stage(wl, caches="synthetic", rerotate=True)
    st.run()
    torch.cuda.synchronize()
    s_pos = oracle.legolink_positions(wl.chunk_lens, wl.suffix_len, wl.k)
    K, _ = el.read_linked_kv(_bits(st.k_caches[0]), _bits(st.v_caches[0]), st.views, 0)
    cached = [_f64(synth.chunk_cache(wl.seed, j, n, wl.num_kv_heads, wl.head_dim, 0.5, layer=0)[0])
              for j, n in enumerate(wl.chunk_lens)]
    moved = np.concatenate(oracle.rerotate_cached(cached, wl.chunk_lens, wl.rope_theta, True))
    keep = np.setdiff1d(np.arange(len(moved)), s_pos)
    assert np.abs(_f64(K[keep]) - moved[keep]).max() <= 2.0 ** -7 * np.abs(moved).max()


def test_refusals():
    """Checked before anything is enqueued."""
    from paper_2410_15332_amd import epic_link as el
    st = _stage(CASES[0], caches="none")
    for bad in (dict(workspace=None), dict(workspace=st.workspace[:-256]), dict(hidden_s=None), dict(k_cache=None)):
        args = {**dict(hidden_s=st.hidden, k_cache=st.k_caches[0], v_cache=st.v_caches[0], workspace=st.workspace), **bad}
        with pytest.raises(el.EpicError):
            el.epic_link_layer_fp8(st.cfg, st.layers[0], st.dplan, **args)
    w = el.epic_layer_weights_fp8(*(getattr(st.layers[0], n) for n, _ in el.epic_layer_weights_fp8._fields_))
    w.wo_scale = None
    with pytest.raises(el.EpicError):
        el.epic_link_layer_fp8(st.cfg, w, st.dplan, st.hidden, st.k_caches[0], st.v_caches[0], st.workspace)


# ---------------------------------------------------------------- the other plans: re-rotated chunks, none to recompute, decode

def _against_the_oracle(call, h_in, s_pos, w, cached_k, cached_v, n_total, wl, read):
    """A layer call on the stream h_in (fp32, in place) against the oracle's, by the bars above.  read() returns the
    recomputed K and V from the cache."""
    hq, hkv, d = wl.num_q_heads, wl.num_kv_heads, wl.head_dim
    before = h_in.double().cpu().numpy()
    call()
    torch.cuda.synchronize()
    h, k, v, added = fp8.decoder_layer(before, s_pos, w, cached_k, cached_v, n_total, wl.ffn, hq, hkv, d, wl.rope_theta, wl.rms_eps)
    gk, gv = read()
    ek, ev = _norm(gk - k) / _norm(k), _norm(gv - v) / _norm(v)
    eh = _norm(h_in.double().cpu().numpy() - h) / _norm(added[0] + added[1])
    print(f"[gpu-test] k {ek:.2e} v {ev:.2e} added {eh:.2e}", flush=True)
    assert ek <= 2.0 ** -8 and ev <= 2.0 ** -8 and eh <= 0.06


RE_ROTATED = [(CASES[0], "stream"), (CASES[1], "stream"), (_wl("rr_one_row", [37, 20, 50], 1, 0, hidden=256, ffn=512, hq=4, hkv=4), "few"),
              (_wl("rr_split_d128", [200, 150], 150, 100, hidden=4096, ffn=1024, hq=8, hkv=2, d=128, layers=1), "split128"), (CASES[4], "whole128"), (CASES[5], "whole128")]


@pytest.mark.parametrize("wl,kernel", RE_ROTATED, ids=[w.name for w, _ in RE_ROTATED])
def test_re_rotated_layers_against_the_oracle(wl, kernel):
    """Re-rotated plans rotate and write in two launches where others take one: the recomputed K and V, what a layer adds
    to the stream, and the rows that are only moved (within a bf16 step), of every layer."""
    from paper_2410_15332_amd import epic_link as el
    import ctypes as C
    route = el._lib.epic_gemm_fp8_route_name
    route.restype = C.c_char_p
    hq, hkv, d = wl.num_q_heads, wl.num_kv_heads, wl.head_dim
    st = _stage(wl, caches="synthetic", rerotate=True)
    assert st.sizes.n_rerotated > 0 and route(3, st.sizes.n_s, (hq + 2 * hkv) * d, wl.hidden).decode() == kernel
    s_pos = oracle.legolink_positions(wl.chunk_lens, wl.suffix_len, wl.k)
    st.hidden.copy_(st.emb)
    for layer in range(wl.n_layers):
        caches = [synth.chunk_cache(wl.seed, j, n, hkv, d, 0.5, layer=layer) for j, n in enumerate(wl.chunk_lens)]
        moved = oracle.rerotate_cached([_f64(c[0]) for c in caches], wl.chunk_lens, wl.rope_theta, True)
        w = fp8.weights(synth.model_weights(wl.seed, layer, wl.hidden, wl.ffn, hq, hkv, d))
        _against_the_oracle(lambda: _layer_call(st, layer, st.hidden), st.hidden, s_pos, w, moved, [_f64(c[1]) for c in caches],
                            wl.linked_len, wl, lambda: _linked_rows(st, layer, s_pos))
        K, V = el.read_linked_kv(_bits(st.k_caches[layer]), _bits(st.v_caches[layer]), st.views, 0)
        keep = np.setdiff1d(np.arange(sum(wl.chunk_lens)), s_pos)
        moved, v = np.concatenate(moved), np.concatenate([c[1] for c in caches])
        assert np.abs(_f64(K[keep]) - moved[keep]).max() <= 2.0 ** -7 * np.abs(moved).max()
        assert np.array_equal(V[keep], v[keep])


def test_plans_without_rows():
    """n_s = 0: the re-rotated copies are all that a call writes, by the layer, by the model, and as the bf16 entry
    points write them; without re-rotation, nothing."""
    from paper_2410_15332_amd import epic_link as el, harness
    wl = _wl("no_rows", [37, 100, 16], 0, 0)
    ref = harness.stage_model(wl, caches="synthetic", rerotate=True)
    st = _stage(wl, caches="synthetic", rerotate=True)
    assert st.sizes.n_s == 0 and st.sizes.n_rerotated > 0
    fresh = [[_bits(t).copy() for t in c] for c in (st.k_caches, st.v_caches)]
    ref.run()
    for call in ("model", "layers"):
        if call == "model":
            st.run()
        else:
            for layer in range(wl.n_layers):
                for t, bits in zip((st.k_caches[layer], st.v_caches[layer]), (fresh[0][layer], fresh[1][layer])):
                    t.view(torch.int16).copy_(torch.from_numpy(bits.view(np.int16)))
                el.epic_link_layer_fp8(st.cfg, st.layers[layer], st.dplan, None, st.k_caches[layer], st.v_caches[layer], None)
        torch.cuda.synchronize()
        for layer in range(wl.n_layers):
            k, v = _bits(st.k_caches[layer]), _bits(st.v_caches[layer])
            assert not np.array_equal(k, fresh[0][layer])
            assert np.array_equal(k, _bits(ref.k_caches[layer])) and np.array_equal(v, _bits(ref.v_caches[layer]))
    plain = _stage(wl, caches="synthetic")
    before = [_bits(t).copy() for t in plain.k_caches + plain.v_caches]
    plain.run()
    torch.cuda.synchronize()
    assert all(np.array_equal(a, _bits(t)) for a, t in zip(before, plain.k_caches + plain.v_caches))


DECODE = [_wl("decode_d64", [37, 100, 16], 25, 5, layers=1), _wl("decode_d128", [40, 21], 18, 3, ffn=512, hq=4, hkv=2, d=128, layers=1)]


@pytest.mark.parametrize("wl", DECODE, ids=[w.name for w in DECODE])
def test_decode_of_two_requests(wl):
    """Decode plans through the 8-bit layer after a link of two requests that share chunks: single tokens, then 3 and
    10 at once.  Each request's new K and V and what the layer adds, against the oracle; all other rows keep their bits."""
    from paper_2410_15332_amd import epic_link as el, harness
    print(f"[gpu-test] fp8 decode {wl.name}", flush=True)
    hq, hkv, d, H = wl.num_q_heads, wl.num_kv_heads, wl.head_dim, wl.hidden
    bits = synth.model_weights(wl.seed, 0, H, wl.ffn, hq, hkv, d)
    tw, layer = harness.quantise_layer({k: harness._bf16_tensor(v, "cuda") for k, v in bits.items()})
    w = fp8.weights(bits)
    cfg = harness.model_cfg(wl, 1)
    chunks, pool, at = [], 80, 0
    for n in wl.chunk_lens:
        chunks.append(list(range(at, at + -(-n // 16))))
        at += len(chunks[-1])
    pick = [list(range(len(wl.chunk_lens))), [1, 0]]
    reqs = [el.Request([wl.chunk_lens[j] for j in p], [chunks[j] for j in p], wl.suffix_len + 7 * i, wl.k) for i, p in enumerate(pick)]
    gen = torch.Generator(device="cuda").manual_seed(wl.seed)
    kc = torch.empty((pool, hkv, 16, d), dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=gen)
    vc = torch.empty((pool, hkv, d, 16), dtype=torch.bfloat16, device="cuda").normal_(0, 0.5, generator=gen)

    def step(sizes, host, views, cached):
        """One layer call on a plan; per request checked where cached (its K and V before the new rows) is given."""
        h = torch.randn(sizes.n_s, H, device="cuda", generator=gen)
        before = h.double().cpu().numpy()
        ws = torch.empty(max(256, el.epic_model_fp8_workspace_bytes(cfg, sizes)), dtype=torch.uint8, device="cuda")
        el.epic_link_layer_fp8(cfg, layer, el.DevicePlan(sizes, host), h, kc, vc, ws)
        torch.cuda.synchronize()
        out, linked = h.double().cpu().numpy(), []
        for b in range(2):
            K, V = el.read_linked_kv(_bits(kc), _bits(vc), views, b)
            linked.append((K, V))
            if cached is None:
                continue
            rows = slice(int(views["s_off"][b]), int(views["s_off"][b + 1]))
            pos, n = views["s_pos"][rows].astype(np.int64), len(cached[b][0])
            assert np.array_equal(pos, np.arange(n, n + rows.stop - rows.start)) and len(K) == pos[-1] + 1
            ref, k, v, added = fp8.decoder_layer(before[rows], pos, w, [_f64(cached[b][0])], [_f64(cached[b][1])], len(K), wl.ffn,
                                                 hq, hkv, d, wl.rope_theta, wl.rms_eps)
            ek, ev = _norm(_f64(K[pos]) - k) / _norm(k), _norm(_f64(V[pos]) - v) / _norm(v)
            eh = _norm(out[rows] - ref) / _norm(added[0] + added[1])
            print(f"[gpu-test] request {b}, {len(pos)} tokens: k {ek:.2e} v {ev:.2e} added {eh:.2e}", flush=True)
            assert ek <= 2.0 ** -8 and ev <= 2.0 ** -8 and eh <= 0.06
            assert np.array_equal(K[:n], cached[b][0]) and np.array_equal(V[:n], cached[b][1])
        return linked

    sizes, host, views = el.epic_plan_link(reqs, cfg.attn, list(range(at, 60)), pool)
    linked = step(sizes, host, views, None)
    free = [i for i in range(60, pool)]
    for new in ([1, 1], [3, 10], [1, 1]):
        sizes, host, views = el.epic_plan_decode(sizes, host, new, cfg.attn, free, pool)
        assert sizes.n_s == sum(new) and (sum(new) > 2 or sizes.tile_rows == 16)
        free = [i for i in free if i not in set(views["linked_blocks"].tolist())]
        linked = step(sizes, host, views, linked)


# streams longer than the norm's 4096 in registers at a time, with planes pending; and Q|K|V whose last column tile is half
# past the end, after each kind of 256-column tiles
WIDE = [
    (_wl("long_8320", [40, 33], 9, 4, hidden=8320, ffn=256, hq=4, hkv=2), "stream"),
    (_wl("long_20480", [40], 5, 0, hidden=20480, ffn=256, hq=2, hkv=1), "stream"),
    (_wl("half_tile_d128", [700, 300], 250, 250, hidden=256, ffn=768, hq=3, hkv=3, d=128), "whole128"),
    (_wl("half_tile_d64", [700, 300], 250, 250, hidden=256, ffn=512, hq=2, hkv=2), "whole128"),
    (_wl("half_tile192", [64], 2049, 0, hidden=384, ffn=512, hq=11, hkv=11, d=128, layers=1), "whole192"),
    (_wl("half_tile256", [64], 2049, 0, hidden=384, ffn=512, hq=17, hkv=17, d=128, layers=1), "whole256"),
    (_wl("half_tile_split", [200, 100], 150, 100, hidden=4096, ffn=1024, hq=3, hkv=3, d=128, layers=1), "split128"),
]


@pytest.mark.parametrize("wl,kernel", WIDE, ids=[w.name for w, _ in WIDE])
def test_wide_layers_against_the_oracle(wl, kernel):
    from paper_2410_15332_amd import epic_link as el
    import ctypes as C
    route = el._lib.epic_gemm_fp8_route_name
    route.restype = C.c_char_p
    hq, hkv, d = wl.num_q_heads, wl.num_kv_heads, wl.head_dim
    st = _stage(wl, caches="synthetic")
    assert route(3, st.sizes.n_s, (hq + 2 * hkv) * d, wl.hidden).decode() == kernel
    s_pos = oracle.legolink_positions(wl.chunk_lens, wl.suffix_len, wl.k)
    st.hidden.copy_(st.emb)
    for layer in range(wl.n_layers):
        caches = [synth.chunk_cache(wl.seed, j, n, hkv, d, 0.5, layer=layer) for j, n in enumerate(wl.chunk_lens)]
        w = fp8.weights(synth.model_weights(wl.seed, layer, wl.hidden, wl.ffn, hq, hkv, d))
        _against_the_oracle(lambda: _layer_call(st, layer, st.hidden), st.hidden, s_pos, w, [_f64(c[0]) for c in caches],
                            [_f64(c[1]) for c in caches], wl.linked_len, wl, lambda: _linked_rows(st, layer, s_pos))
    alone = st.hidden.double()
    st.run()
    torch.cuda.synchronize()
    ref = alone * torch.rsqrt(alone.square().mean(-1, keepdim=True) + wl.rms_eps) * st.final_norm.double()
    assert bool(((st.out - ref).abs() <= 2.0 ** -20 * ref.abs()).all())

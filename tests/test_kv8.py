"""The 8-bit cache and the head norm and rotation without a GPU: the oracle's cache against torch's
e4m3 and against itself, rotary frequencies, and everything that the entry points refuse (no call
here reaches a launch)."""
import ctypes as C
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp8, kv8  # noqa: E402
from oracle.link import masked_attention  # noqa: E402
from paper_2410_15332_amd import epic_link as el  # noqa: E402

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4
P = 1 << 20                                              # an aligned address that is never followed


# ---------------------------------------------------------------- the oracle

def test_rows_round_as_torch_rounds():
    rng = np.random.default_rng(1)
    k, v = (rng.normal(size=(7, 3, 64)) * np.exp(3 * rng.normal(size=(7, 3, 1))) for _ in range(2))
    k = k.astype(np.float32).astype(np.float64)          # torch rounds from float32
    v = v.astype(np.float32).astype(np.float64)
    kq, vq, ks, vs = kv8.quantise(k, v)
    for y, q, b in ((k, kq, ks), (v, vq, vs)):
        t = b.astype(int) - 127
        top = np.abs(y).max(-1)
        assert np.all(top <= 448.0 * 2.0 ** t) and np.all(top > 448.0 * 2.0 ** (t - 1))
        ref = torch.from_numpy(np.ldexp(y, -t[..., None])).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
        assert np.array_equal(q, ref)


def test_nan_tokens_are_nan_in_both():
    k, v = np.ones((4, 64)), np.ones((4, 64))
    k[1, 3], v[2, 5] = np.inf, np.nan
    kq, vq, ks, vs = kv8.quantise(k, v)
    assert list(ks == 255) == list(vs == 255) == [False, True, True, False]
    assert np.all(kq[1:3] == 0x7F) and np.all(vq[1:3] == 0)
    assert np.isnan(kv8.values(kq, ks)[1:3]).all() and np.isnan(kv8.values(vq, vs)[1:3]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_layout_round_trip(d):
    rng = np.random.default_rng(2)
    k, v = (rng.integers(0, 256, (3, 2, 16, d)).astype(np.uint8) for _ in range(2))
    a, b = kv8.layout(k, v)
    assert a.shape == el.kv8_shapes(3, 2, d)[0] and b.shape == el.kv8_shapes(3, 2, d)[1]
    assert a[1, 0, d // 64 - 1, 2, 7, 5] == k[1, 0, 7, d - 64 + 32 + 5]
    assert b[1, 0, d // 64 - 1, 2, 7, 3, 1] == v[1, 0, 9, d - 64 + 48 + 7]
    for x, y in zip(kv8.tokens(a, b), (k, v)):
        assert np.array_equal(x, y)


def test_oracle_attention_without_nan_is_masked_attention():
    rng = np.random.default_rng(3)
    q, K, V = rng.normal(size=(5, 4, 64)), rng.normal(size=(9, 2, 64)), rng.normal(size=(9, 2, 64))
    pos = np.array([0, 2, 4, 7, 8])
    out, lse, bad = kv8.attention(q, K, V, pos)
    o, l = masked_attention(q, K, V, pos)
    assert np.array_equal(out, o) and np.array_equal(lse, l) and not bad.any()
    K[5, 1] = np.nan                                     # rows from position 5 on, heads of KV head 1
    bad = kv8.attention(q, K, V, pos)[2]
    assert bad.tolist() == [[False] * 4] * 3 + [[False, False, True, True]] * 2


# ---------------------------------------------------------------- frequencies

@pytest.mark.parametrize("rot", [16, 48, 64, 128])
@pytest.mark.parametrize("theta", [10000.0, 500000.0])
def test_plain_and_divided_frequencies(rot, theta):
    f = theta ** (-2.0 * np.arange(rot // 2) / rot)
    assert np.allclose(el.epic_rope_freqs(el.rope_cfg(rot, theta)), f, rtol=1e-14)
    assert np.allclose(el.epic_rope_freqs(el.rope_cfg(rot, theta, factor=4.0)), f / 4.0, rtol=1e-14)
    assert np.allclose(el.epic_rope_freqs(el.rope_cfg(rot, theta, factor=0.0)), f, rtol=1e-14)


def test_frequencies_for_long_contexts():
    """By wavelength: short waves keep their frequency, long ones have it divided, those between are
    mixed by how many of them the original context holds."""
    rot, theta, factor, ctx, low, high = 128, 500000.0, 8.0, 8192, 1.0, 4.0
    got = el.epic_rope_freqs(el.rope_cfg(rot, theta, factor=factor, original_context=ctx, low_turns=low, high_turns=high))
    kinds = set()
    for j in range(rot // 2):
        f = theta ** (-2.0 * j / rot)
        wave = 2 * math.pi / f
        if wave < ctx / high:
            want, kind = f, "kept"
        elif wave > ctx / low:
            want, kind = f / factor, "divided"
        else:
            mix = (ctx / wave - low) / (high - low)
            want, kind = (1 - mix) * f / factor + mix * f, "mixed"
        kinds.add(kind)
        assert math.isclose(got[j], want, rel_tol=1e-12), j
    assert kinds == {"kept", "divided", "mixed"}


@pytest.mark.parametrize("kw", [dict(rot_dim=8), dict(rot_dim=-16), dict(theta=1.0), dict(theta=float("nan")),
                                dict(theta=float("inf")), dict(factor=-1.0), dict(factor=float("nan")),
                                dict(original_context=-1), dict(original_context=4096, low_turns=4.0, high_turns=4.0),
                                dict(original_context=4096, low_turns=-1.0, high_turns=4.0), dict(interleaved=2),
                                dict(original_context=4096, low_turns=1.0, high_turns=float("inf")),
                                dict(amplitude=-1.0), dict(amplitude=float("inf"))])
def test_frequencies_refuse(kw):
    r = el.rope_cfg(64, 10000.0)
    for name, x in kw.items():
        setattr(r, name, x)
    out = (C.c_double * 64)()
    assert el._rope_freqs(C.byref(r), out) == INVALID
    assert el._last_error()


# ---------------------------------------------------------------- refusals of the C entry points

def _rope(cfg=None, rope=None, kind=0, qkv=16 * P, ld=1280, rows=4, pos=P, freqs=P, qn=P, kn=P, eps=1e-6, q=17 * P,
          k=18 * P, v=19 * P):
    cfg = cfg or el.attn_cfg(8, 1, 128)
    rope = rope or el.rope_cfg(128, 10000.0)
    return el._qk_norm_rope(C.byref(cfg), C.byref(rope), kind, qkv, ld, rows, pos, freqs, qn, kn, eps, q, k, v, None)


@pytest.mark.parametrize("kw,status", [
    (dict(rows=-1), INVALID), (dict(kind=2), INVALID), (dict(kind=-1), INVALID), (dict(ld=1279), INVALID),
    (dict(ld=1284), INVALID), (dict(kind=1, ld=1282), INVALID), (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(qkv=None), INVALID), (dict(pos=None), INVALID), (dict(freqs=None), INVALID), (dict(freqs=P + 4), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(qkv=16 * P + 8), INVALID),
    (dict(q=17 * P + 8), INVALID), (dict(qn=P + 8), INVALID), (dict(kn=P + 8), INVALID),
    (dict(q=16 * P), INVALID), (dict(k=16 * P + 3 * 2560), INVALID), (dict(v=16 * P + 4 * 2560 - 16), INVALID),
    (dict(k=17 * P + 4 * 2048 - 16), INVALID), (dict(v=18 * P), INVALID),
    (dict(rope=el.rope_cfg(144, 10000.0)), INVALID), (dict(rope=el.rope_cfg(24, 10000.0)), INVALID),
    (dict(rows=1 << 24), UNSUPPORTED), (dict(ld=1 << 41), UNSUPPORTED),
    (dict(cfg=el.attn_cfg(12, 4, 128)), UNSUPPORTED), (dict(cfg=el.attn_cfg(8, 2, 96)), UNSUPPORTED)])
def test_qk_norm_rope_refuses(kw, status):
    assert _rope(**kw) == status
    assert el._last_error()


def test_no_rows_are_fine():
    assert _rope(rows=0, qkv=None, q=None, k=None, v=None, pos=None, freqs=None) == 0


def _cache(k=P, v=2 * P, scale=3 * P, n=8):
    return el.epic_kv8_cache(k, v, scale, n)


def _pack(cfg=None, n=4, src=P, k=P, v=P, blocks=8, dst=P, cache=None):
    cfg = cfg or el.attn_cfg(2, 2, 128)
    return el._kv8_pack(C.byref(cfg), n, src, k, v, blocks, dst, C.byref(cache or _cache()), None)


def _unpack(cfg=None, n=4, src=P, k=P, v=P, blocks=8, dst=P, cache=None):
    cfg = cfg or el.attn_cfg(2, 2, 128)
    return el._kv8_unpack(C.byref(cfg), n, src, C.byref(cache or _cache()), dst, k, v, blocks, None)


@pytest.mark.parametrize("call", [_pack, _unpack])
@pytest.mark.parametrize("kw,status", [
    (dict(n=-1), INVALID), (dict(blocks=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(k=P + 8), INVALID), (dict(v=P + 8), INVALID), (dict(cache=_cache(n=-1)), INVALID),
    (dict(cache=_cache(k=None)), INVALID), (dict(cache=_cache(v=None)), INVALID), (dict(cache=_cache(scale=None)), INVALID),
    (dict(cache=_cache(scale=P + 4)), INVALID), (dict(cache=_cache(k=P + 8)), INVALID),
    (dict(n=9, src=None), INVALID), (dict(n=9, dst=None), INVALID), (dict(n=1 << 24), UNSUPPORTED),
    (dict(cfg=el.attn_cfg(2, 2, 80)), UNSUPPORTED), (dict(cfg=el.attn_cfg(2, 0, 64)), INVALID)])
def test_moves_refuse(call, kw, status):
    assert call(**kw) == status
    assert el._last_error()


def test_moving_nothing_is_fine():
    assert _pack(n=0, src=None, dst=None, k=None, v=None) == 0
    assert _unpack(n=0, src=None, dst=None, k=None, v=None) == 0


def _plan(tile_rows=0, split=0):
    cfg = el.attn_cfg(8, 2, 64, 0.0, split, tile_rows)
    sizes, buf, _ = el.epic_plan_link([el.Request([40, 30], [[0, 1, 2], [3, 4]], 5, 4)], cfg, range(5, 20), 20)
    return cfg, sizes, buf


def _attend(cfg, sizes, buf, q=P, k=P, v=P, cache=None, out=P, ws=P, size=1 << 40, plan=True):
    p = el.epic_plan_layout(sizes, buf.ctypes.data)
    return el._link_attention_kv8(C.byref(cfg), C.byref(sizes), C.byref(p) if plan else None, q, k, v,
                                  C.byref(cache or _cache()), out, None, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(q=P + 8), INVALID), (dict(out=P + 2), INVALID), (dict(plan=False), INVALID),
    (dict(cache=_cache(k=None)), INVALID), (dict(cache=_cache(scale=P + 1)), INVALID),
    (dict(ws=None), WORKSPACE), (dict(size=100), WORKSPACE), (dict(ws=P + 8), INVALID)])
def test_attention_refuses(kw, status):
    assert _attend(*_plan(128), **kw) == status
    assert el._last_error()


def test_attention_refuses_rotation_without_a_base():
    cfg = el.attn_cfg(8, 2, 64)
    sizes, buf, _ = el.epic_plan_link([el.Request([40, 30], [[0, 1, 2], [3, 4]], 5, 4, True)], cfg, range(5, 20), 20)
    assert _attend(cfg, sizes, buf) == INVALID


def test_workspace():
    """16-row tiles: the bf16 call's partials; wide tiles: the linked blocks in bf16 and their table too."""
    for tile_rows in (16, 128):
        for split in (0, 2):
            cfg, sizes, _ = _plan(tile_rows, split)
            need, partials = el.epic_link_kv8_workspace_bytes(cfg, sizes), el.epic_link_workspace_bytes(cfg, sizes)
            assert (sizes.n_partials > 0) == (split > 0)
            if tile_rows == 16:
                assert need == partials
            else:
                assert need >= partials + sizes.n_linked_blocks * (2 * 2 * 16 * 64 * 2 + 4)
    assert el._link_kv8_ws(None, C.byref(sizes)) == 0
    assert el._link_kv8_ws(C.byref(el.attn_cfg(8, 2, 96)), C.byref(sizes)) == 0


# ---------------------------------------------------------------- refusals of the binding

def test_binding_refuses_other_memory():
    """Tensors of the host: the library could not tell them from the GPU's."""
    with pytest.raises(ValueError, match="current GPU"):
        k = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
        cache = el.Kv8Cache.zeros(4, 2, 64, device="cpu")
        el.epic_kv8_pack(k, k.transpose(2, 3).contiguous(), cache)


@pytest.mark.parametrize("k,v,s", [((4, 2, 1, 4, 16, 16), (4, 2, 1, 4, 16, 4, 4), (4, 2, 2, 8)),
                                   ((4, 2, 1, 4, 16, 16), (4, 2, 2, 4, 16, 4, 4), (4, 2, 2, 16)),
                                   ((4, 2, 3, 4, 16, 16), (4, 2, 3, 4, 16, 4, 4), (4, 2, 2, 16)),
                                   ((4, 2, 4, 16, 16), (4, 2, 1, 4, 16, 4, 4), (4, 2, 2, 16))])
def test_cache_shapes_are_checked(k, v, s):
    with pytest.raises(ValueError):
        el.Kv8Cache(*(torch.zeros(x, dtype=torch.uint8) for x in (k, v, s)))


def test_cache_types_and_strides_are_checked():
    k, v, s = (torch.zeros(x, dtype=torch.uint8) for x in el.kv8_shapes(4, 2, 64))
    with pytest.raises(ValueError):
        el.Kv8Cache(k.to(torch.int32), v, s)
    with pytest.raises(ValueError):
        el.Kv8Cache(k, v.transpose(3, 4), s)
    el.Kv8Cache(k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu))


def _parts(cache, hkv=2, d=64):
    c = cache.of(hkv, d, -1)._obj
    return c.k, c.v, c.scale, c.num_blocks


def _addresses(cache):
    return cache.k.data_ptr(), cache.v.data_ptr(), cache.scale.data_ptr(), cache.k.shape[0]


def test_cache_follows_its_tensors():
    """A call takes the addresses that the tensors have by then: after other tensors took their place, and after they
    were resized."""
    cache = el.Kv8Cache.zeros(4, 2, 64, device="cpu")
    assert _parts(cache) == _addresses(cache)
    old = cache.k                                        # (kept, so that its address is no other's)
    cache.k = torch.ones_like(old)
    assert cache.k.data_ptr() != old.data_ptr() and _parts(cache) == _addresses(cache)
    cache.k, cache.v, cache.scale = (torch.zeros(s, dtype=torch.uint8) for s in el.kv8_shapes(9, 2, 64))
    assert _parts(cache) == _addresses(cache) and cache.num_blocks == 9
    for n in (4096, 3):                                  # to other memory; within what it has
        for t, s in zip((cache.k, cache.v, cache.scale), el.kv8_shapes(n, 2, 64)):
            t.resize_(s)
        assert _parts(cache) == _addresses(cache) and cache.num_blocks == n
    cache.k, cache.v, cache.scale = (torch.zeros(s, dtype=torch.uint8) for s in el.kv8_shapes(4, 3, 128))
    assert _parts(cache, 3, 128) == _addresses(cache) and (cache.hkv, cache.d) == (3, 128)
    with pytest.raises(ValueError):
        cache.of(2, 64, -1)


@pytest.mark.parametrize("name", ["k", "v", "scale"])
def test_cache_of_unlike_tensors_is_refused(name):
    for change in (lambda t: t[:3], lambda t: torch.zeros((5, *t.shape[1:]), dtype=t.dtype), lambda t: t.to(torch.int16),
                   lambda t: t.transpose(0, 1)):
        cache = el.Kv8Cache.zeros(4, 4, 64, device="cpu")
        setattr(cache, name, change(getattr(cache, name)))
        for _ in range(2):
            with pytest.raises(ValueError):
                cache.of(4, 64, -1)
    cache = el.Kv8Cache.zeros(4, 4, 64, device="cpu")
    t = getattr(cache, name)
    t.resize_((6, *t.shape[1:]))                         # one of the three
    with pytest.raises(ValueError):
        cache.of(4, 64, -1)
    cache = el.Kv8Cache.zeros(4, 4, 64, device="cpu")
    parts = {"k": cache.k, "v": cache.v, "scale": cache.scale}
    with pytest.raises(ValueError, match="missing"):
        el.Kv8Cache(**{**parts, name: None})
    setattr(cache, name, None)
    with pytest.raises(ValueError, match="missing"):
        cache.of(4, 64, -1)
    setattr(cache, name, parts[name])
    assert _parts(cache, 4) == _addresses(cache)

"""GPU parity of epic_qk_norm_rope against its definition in float64.

Bars.  With y the exact normed head and u = max |a|, |b| of a pair: the norm's fp32 steps (products and
sums of 128 squares in a tree of at most 20, square root, division, two products) are off by under 32 * 2^-24
of |y|; an angle's sine and cosine by 2^-22 (2^-25 of a rest up to pi / 4, 2e-9 of a polynomial, its own
fp32 roundings: under 4 of 2^-24) and by what float64 leaves of an angle of 2^31 (five roundings of
2^-53, the reference's among them: 20 of 2^-24), the rotation by 3 roundings.  So each result is within
amplitude * (|a| + |b|) * 60 * 2^-24 of the exact one before it is rounded to bf16: then 2^-8 of itself,
or half a step of the smallest values.  Heads that are neither normed nor turned, and V, are
rounded only: bits of bf16 inputs are kept.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import oracle  # noqa: E402

pytestmark = pytest.mark.gpu

THETA = 500000.0


def _el():
    from paper_2410_15332_amd import epic_link as el
    return el


def _guarded(shape, dtype=torch.bfloat16):
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    raw = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    return raw[:n].view(dtype).view(shape), raw[n:]


def _exact(x, pos, f, rot, interleaved, amp, w, eps):
    """x [n, heads, d] float64 -> (result, the sum of magnitudes that each result is made of)."""
    if w is not None:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    y, mag = x.copy(), np.abs(x)
    if rot:
        j = np.arange(rot // 2)
        a, b = (2 * j, 2 * j + 1) if interleaved else (j, j + rot // 2)
        ang = pos[:, None].astype(np.float64) * f
        c, s = amp * np.cos(ang)[:, None], amp * np.sin(ang)[:, None]
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        both = amp * (np.abs(x[..., a]) + np.abs(x[..., b]))
        mag[..., a] = mag[..., b] = both
    return y, mag


def _check(got, y, mag, what):
    got = got.double().cpu().numpy()
    bar = 2.0 ** -8 * np.abs(y) + mag * 61 * 2.0 ** -24 + 2.0 ** -134
    over = np.abs(got - y) > bar
    assert not over.any(), f"{what}: {over.sum()} of {over.size} off, worst {np.max(np.abs(got - y) / bar):.2f} bars"


def _case(n, hq, hkv, d, rot, dtype, interleaved=False, norms="qk", pad=0, pos=None, eps=1e-6, seed=0, scale=1.0, **scaling):
    el = _el()
    print(f"[gpu-test] rope n {n} heads {hq}/{hkv}/{d} rot {rot} {dtype} inter {interleaved} norms '{norms}' pad {pad}", flush=True)
    rng = np.random.default_rng([n, hq, d, rot, seed])
    cols = (hq + 2 * hkv) * d
    x = torch.from_numpy(rng.normal(size=(n, cols + pad)) * scale * np.exp(rng.normal(size=cols + pad))).to(dtype).cuda()
    qkv = x[:, :cols]
    pos = np.arange(n) + 7 if pos is None else np.asarray(pos)
    rope = el.rope_cfg(rot, THETA, interleaved, **scaling)
    f = el.epic_rope_freqs(rope)
    w = {h: torch.from_numpy(1 + 0.2 * rng.normal(size=d)).to(torch.bfloat16).cuda() for h in norms}
    outs = [_guarded((n, h, d)) for h in (hq, hkv, hkv)]
    (q, _), (k, _), (v, _) = outs
    el.epic_qk_norm_rope(el.attn_cfg(hq, hkv, d), rope, qkv, torch.from_numpy(pos.astype(np.int32)).cuda(),
                         torch.from_numpy(f).cuda() if rot else None, q, k, v, q_norm=w.get("q"), k_norm=w.get("k"), eps=eps)
    torch.cuda.synchronize()
    for _, guard in outs:
        assert bool((guard == 0xA5).all()), "written behind the end"
    xs = qkv.double().cpu().numpy().reshape(n, hq + 2 * hkv, d)
    amp = scaling.get("amplitude", 1.0)
    for name, got, part in (("q", q, xs[:, :hq]), ("k", k, xs[:, hq:hq + hkv])):
        wt = w[name].double().cpu().numpy() if name in w else None
        _check(got, *_exact(part, pos, f, rot, interleaved, amp, wt, eps), name)
    raw = qkv.reshape(n, hq + 2 * hkv, d)[:, hq + hkv:].to(torch.bfloat16)
    assert torch.equal(v.view(torch.int16), raw.contiguous().view(torch.int16)), "v"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,rot", [(64, 64), (128, 128), (128, 64), (128, 16), (64, 48), (128, 112), (64, 0)])
def test_parts_of_the_head(d, rot, interleaved, dtype):
    _case(37, 8, 2, d, rot, dtype, interleaved)


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 8, 64), (1, 1, 64), (1, 1, 128), (128, 1, 128), (40, 5, 128), (6, 3, 64)])
@pytest.mark.parametrize("n", [1, 2, 3, 255, 256, 514])
def test_heads_and_rows(n, hq, hkv, d):
    """Heads of less than a wavefront to several passes of a workgroup, a workgroup each below 256 rows."""
    _case(n, hq, hkv, d, d, torch.bfloat16)


@pytest.mark.parametrize("hq,hkv,d,rot", [(8, 8, 64, 64), (16, 1, 64, 48), (8, 1, 128, 128), (1, 1, 64, 16), (6, 3, 128, 96)])
@pytest.mark.parametrize("dtype,interleaved", [(torch.bfloat16, False), (torch.float32, True)])
def test_short_rows(hq, hkv, d, rot, dtype, interleaved):
    """Rows of few heads, several to a workgroup, the last workgroup with fewer."""
    _case(2051, hq, hkv, d, rot, dtype, interleaved)


@pytest.mark.parametrize("norms", ["", "q", "k", "qk"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_norms_of_either(norms, dtype):
    _case(5, 8, 4, 128, 96, dtype, norms=norms)


@pytest.mark.parametrize("dtype,pad", [(torch.bfloat16, 8), (torch.bfloat16, 264), (torch.float32, 4), (torch.float32, 1284)])
@pytest.mark.parametrize("n", [1, 9, 700])
def test_rows_apart(n, dtype, pad):
    _case(n, 4, 2, 64, 32, dtype, pad=pad)


@pytest.mark.parametrize("scaling", [dict(factor=4.0), dict(factor=8.0, original_context=8192, low_turns=1.0, high_turns=4.0),
                                     dict(factor=32.0, original_context=4096, low_turns=1.0, high_turns=32.0, amplitude=1.25)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_and_negative_positions(scaling, interleaved):
    pos = [0, 1, 2 ** 31 - 1, 2 ** 24 + 1, 1000003, 131071, -1, -(2 ** 31), 77, 2 ** 30]
    _case(len(pos), 8, 2, 128, 128, torch.float32, interleaved, pos=pos, **scaling)


def test_small_and_large_values():
    for scale in (1e-30, 1e-12, 1e12):
        _case(4, 4, 2, 64, 64, torch.float32, norms="", scale=scale)
    _case(4, 4, 2, 64, 64, torch.bfloat16, scale=1e-20, eps=1e-30)   # squares below fp32's range: eps alone
    _case(4, 4, 2, 64, 64, torch.bfloat16, scale=1e14)


def test_matches_the_models_rotation():
    """Half layout, whole head, no scaling: the rotation of the decoder layers."""
    el = _el()
    rng = np.random.default_rng(9)
    n, hq, hkv, d = 33, 4, 2, 128
    qkv = torch.from_numpy(rng.normal(size=(n, (hq + 2 * hkv) * d))).to(torch.float32).cuda()
    pos = rng.integers(0, 131072, n)
    rope = el.rope_cfg(d, THETA)
    q, k, v = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    el.epic_qk_norm_rope(el.attn_cfg(hq, hkv, d), rope, qkv, torch.from_numpy(pos.astype(np.int32)).cuda(),
                         torch.from_numpy(el.epic_rope_freqs(rope)).cuda(), q, k, v)
    x = qkv.double().cpu().numpy().reshape(n, -1, d)
    ref = oracle.rope(x[:, :hq], pos, THETA)
    assert np.abs(q.double().cpu().numpy() - ref).max() <= 2.0 ** -8 * np.abs(ref).max()


def test_nan_stays_in_its_head():
    el = _el()
    n, hq, hkv, d = 3, 4, 2, 64
    x = torch.randn(n, (hq + 2 * hkv) * d, device="cuda")
    x[1, 2 * d + 5] = float("nan")
    x[2, hq * d + 1] = float("inf")
    rope = el.rope_cfg(d, THETA)
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    q, k, v = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
    el.epic_qk_norm_rope(el.attn_cfg(hq, hkv, d), rope, x, torch.arange(n, dtype=torch.int32, device="cuda"),
                         torch.from_numpy(el.epic_rope_freqs(rope)).cuda(), q, k, v, q_norm=w, k_norm=w)
    bad = torch.isnan(q).any(-1)
    assert bad.nonzero().tolist() == [[1, 2]] and bool(torch.isnan(q[1, 2]).all())
    assert torch.isnan(k).any(-1).nonzero().tolist() == [[2, 0]]
    assert not bool(torch.isnan(v).any())


def test_other_stream_and_graph():
    el = _el()
    n, hq, hkv, d = 20, 8, 2, 128
    rope = el.rope_cfg(64, THETA, True)
    f = torch.from_numpy(el.epic_rope_freqs(rope)).cuda()
    x = torch.randn(n, (hq + 2 * hkv) * d, device="cuda").to(torch.bfloat16)
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1000
    w = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    cfg = el.attn_cfg(hq, hkv, d)

    def call(outs, stream=None):
        el.epic_qk_norm_rope(cfg, rope, x, pos, f, *outs, q_norm=w, k_norm=w, stream=stream)

    def fresh():
        return [torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv)]

    ref, other, graphed = fresh(), fresh(), fresh()
    call(ref)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    call(other, s)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(graphed)
    for _ in range(3):
        for t in graphed:
            t.zero_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(ref, other, graphed))
    x.copy_(torch.randn_like(x.float()).to(torch.bfloat16))       # a replay reads what the input holds now
    g.replay()
    call(ref)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, graphed))


def test_binding_refuses():
    el = _el()
    cfg, rope = el.attn_cfg(4, 2, 64), el.rope_cfg(64, THETA)
    f = torch.from_numpy(el.epic_rope_freqs(rope)).cuda()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    good = dict(qkv=torch.zeros(3, 512, **bf), pos=torch.zeros(3, dtype=torch.int32, device="cuda"), freqs=f,
                q=torch.zeros(3, 4, 64, **bf), k=torch.zeros(3, 2, 64, **bf), v=torch.zeros(3, 2, 64, **bf))
    el.epic_qk_norm_rope(cfg, rope, **good)
    for name, bad in (("qkv", torch.zeros(3, 511, **bf)), ("qkv", torch.zeros(512, 3, **bf).t()),
                      ("qkv", torch.zeros(3, 512, dtype=torch.float16, device="cuda")), ("qkv", torch.zeros(3, 512)),
                      ("pos", torch.zeros(3, dtype=torch.int64, device="cuda")), ("pos", torch.zeros(2, dtype=torch.int32, device="cuda")),
                      ("freqs", f.float()), ("freqs", f[:31]), ("freqs", None), ("q", torch.zeros(3, 4, 64, device="cuda")),
                      ("k", torch.zeros(3, 4, 64, **bf)), ("v", torch.zeros(3, 2, 128, **bf)[..., ::2]), ("v", None)):
        with pytest.raises(ValueError):
            el.epic_qk_norm_rope(cfg, rope, **{**good, name: bad})
    x = torch.zeros(3, 8, 64, **bf)
    with pytest.raises(el.EpicError):                     # in place
        el.epic_qk_norm_rope(cfg, rope, **{**good, "qkv": x.view(3, 512), "q": x.view(-1)[:768].view(3, 4, 64)})
    torch.cuda.synchronize()

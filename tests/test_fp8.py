"""The 8-bit operators without a GPU: the oracle's e4m3 and scales against another definition,
and everything that the entry points refuse (no call here reaches a launch)."""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp8  # noqa: E402
from paper_2410_15332_amd import epic_link as el  # noqa: E402

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 4


# ---------------------------------------------------------------- the oracle

def test_e4m3_values_are_torchs():
    codes = np.arange(256, dtype=np.uint8)
    ref = torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(fp8.e4m3_decode(codes), ref, equal_nan=True)


def test_e4m3_rounding_is_torchs():
    rng = np.random.default_rng(3)
    y = np.concatenate([rng.uniform(-448, 448, 20000), rng.normal(0, 0.02, 20000), fp8.POSITIVE[:127],
                        (fp8.POSITIVE[:126] + fp8.POSITIVE[1:127]) / 2, [0.0, -0.0, 2.0 ** -10, -2.0 ** -10]])
    y = y.astype(np.float32)
    ref = torch.from_numpy(y).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(fp8.e4m3_encode(y), ref)
    assert list(fp8.e4m3_encode(np.array([np.nan, np.inf, -np.inf]))) == [0x7F] * 3


@pytest.mark.parametrize("top,t", [(448.0, 0), (448.0 * (1 + 2.0 ** -20), 1), (224.0, -1), (1.75, -8), (1.7500001, -7),
                                   (1.0, -8), (0.0, 0), (2.0 ** -149, -127), (3.0e38, 120)])
def test_scale_exponent(top, t):
    assert fp8.scale_exponent(top) == t
    if 0 < t < 127 or -127 < t < 0:
        assert top <= 448 * 2.0 ** t and top > 448 * 2.0 ** (t - 1)


def test_quantise_keeps_half_a_step():
    rng = np.random.default_rng(4)
    y = rng.normal(size=(5, 256)) * np.exp(rng.normal(size=(5, 256)))
    q, t = fp8.quantise(y)
    s = np.ldexp(1.0, fp8.spread(t, 5, 256))
    assert np.all(np.abs(fp8.dequantise(q, t) - y) <= np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * s))


# ---------------------------------------------------------------- refusals of the C entry points

P = 1 << 20                                              # an aligned address that is never followed


def _quant(x=P, m=4, k=128, rows=1, q=P, scale=P):
    return el._quant_fp8(x, m, k, rows, q, scale, None)


def _norm(x=P, delta=P, w=P, m=4, k=128, eps=1e-5, out=P, q=P, scale=P):
    return el._rmsnorm_fp8(x, delta, w, m, k, eps, out, q, scale, None)


def _gemm(epi=0, a=P, sa=P, w=P, sw=P, m=4, n=256, k=128, out=P, ss=P, ws=P, size=64 << 20):
    return el._gemm_fp8(epi, a, sa, w, sw, m, n, k, out, ss, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), INVALID), (dict(k=0), INVALID), (dict(rows=2), INVALID), (dict(rows=0), INVALID),
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(x=P + 8), INVALID),
    (dict(q=P + 4), INVALID), (dict(k=64), UNSUPPORTED), (dict(k=192), UNSUPPORTED),
    (dict(m=(1 << 31) - 1, k=128), UNSUPPORTED), (dict(m=1 << 30, k=1024), UNSUPPORTED),
    (dict(m=1 << 28, k=128), UNSUPPORTED),
    (dict(m=65536 * 128, rows=128), UNSUPPORTED)])
def test_quant_refuses(kw, status):
    assert _quant(**kw) == status
    assert el._last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(m=-1), INVALID), (dict(k=0), INVALID), (dict(eps=0.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(x=None), INVALID), (dict(w=None), INVALID),
    (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(out=P + 4), INVALID), (dict(delta=P + 8), INVALID),
    (dict(k=130), UNSUPPORTED), (dict(k=32768 + 128), UNSUPPORTED), (dict(m=(1 << 31) - 1), UNSUPPORTED),
    (dict(m=1 << 23, k=4096), UNSUPPORTED)])
def test_norm_refuses(kw, status):
    assert _norm(**kw) == status
    assert el._last_error()


@pytest.mark.parametrize("kw,status", [
    (dict(epi=3), INVALID), (dict(epi=-1), INVALID), (dict(m=-1), INVALID), (dict(n=0), INVALID), (dict(k=-128), INVALID),
    (dict(a=None), INVALID), (dict(sa=None), INVALID), (dict(w=None), INVALID), (dict(sw=None), INVALID),
    (dict(out=None), INVALID), (dict(epi=2, ss=None), INVALID), (dict(sa=P + 2), INVALID), (dict(a=P + 8), INVALID),
    (dict(w=P + 8), INVALID), (dict(out=P + 4), INVALID), (dict(epi=2, ss=P + 1), INVALID), (dict(ws=P + 128), INVALID),
    (dict(k=64), UNSUPPORTED), (dict(k=200), UNSUPPORTED), (dict(n=200), UNSUPPORTED), (dict(epi=1, n=384), UNSUPPORTED),
    (dict(epi=2, n=128), UNSUPPORTED), (dict(m=1 << 24, k=128), UNSUPPORTED), (dict(n=1 << 24, k=128), UNSUPPORTED),
    (dict(m=1 << 20, n=1024), UNSUPPORTED), (dict(ws=None), WORKSPACE), (dict(size=(64 << 20) - 1), WORKSPACE)])
def test_gemm_refuses(kw, status):
    assert _gemm(**kw) == status
    assert el._last_error()


def test_no_rows_is_no_work():
    assert _quant(m=0, x=None, q=None, scale=None) == 0
    assert _norm(m=0, x=None, w=None, q=None, scale=None) == 0
    assert _gemm(m=0, a=None, sa=None, out=None, ws=None) == 0


def test_scale_bytes():
    assert el.epic_fp8_scale_bytes(5, 256) == 2 * 8 == int(np.prod(el.fp8_row_scale_shape(5, 256)))
    assert el.epic_fp8_scale_bytes(0, 256) == 0
    assert el.epic_fp8_scale_bytes(5, 100) == 0 and el.epic_fp8_scale_bytes(-1, 128) == 0
    assert el.fp8_block_scale_shape(300, 256) == (3, 2)


# ---------------------------------------------------------------- refusals of the binding

def test_binding_refuses_what_the_kernels_cannot_read():
    x = torch.zeros(4, 256, dtype=torch.bfloat16)
    q, s = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(2, 4, dtype=torch.uint8)
    for bad in (dict(x=x.float()), dict(x=x.t().contiguous().t()), dict(q=q[:, :128]), dict(q=q.to(torch.int8)),
                dict(scale=s[:, :3]), dict(scale=None), dict()):                      # the last: not on a GPU
        with pytest.raises(ValueError):
            el.epic_quant_fp8(**{**dict(x=x, q=q, scale=s), **bad})
    with pytest.raises(ValueError):
        el.epic_rmsnorm_fp8(torch.zeros(4, 256), torch.zeros(128, dtype=torch.bfloat16), 1e-5, q, s)
    with pytest.raises(ValueError):
        el.epic_gemm_fp8(el.FP8_BF16, q, s, torch.zeros(128, 128, dtype=torch.uint8), torch.zeros(1, 2, dtype=torch.uint8),
                         torch.zeros(4, 128, dtype=torch.bfloat16))


class _Elsewhere:
    """A workspace of 64 MB of another device, aligned: everything that the library itself looks at is right."""

    device, nbytes = "another device", 64 << 20

    def get_device(self):
        return 7

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return P

    def stride(self):
        return (1,)

    def numel(self):
        return self.nbytes

    def element_size(self):
        return 1


def _workspaces():
    """What may not reach a kernel: memory of another device, and a view with one byte behind its 64 MB."""
    return [_Elsewhere(), torch.zeros(1, dtype=torch.uint8).expand(64 << 20)]


@pytest.mark.parametrize("bad", [0, 1])
def test_gemm_refuses_workspaces_of_other_memory(bad, monkeypatch):
    """With host tensors in the place of the GPU's, and no call past the binding."""
    calls = []
    monkeypatch.setattr(el, "_device_of", lambda name, t: t.get_device())
    monkeypatch.setattr(el, "_raw_stream", lambda stream, device: None)
    monkeypatch.setattr(el, "_gemm_fp8", lambda *args: calls.append(args) or 0)
    u8 = lambda *s: torch.zeros(s, dtype=torch.uint8)  # noqa: E731
    args = (el.FP8_BF16, u8(4, 256), u8(2, 4), u8(128, 256), u8(1, 2), torch.zeros(4, 128, dtype=torch.bfloat16))
    el.epic_gemm_fp8(*args, workspace=u8(64 << 20))
    assert len(calls) == 1
    with pytest.raises(ValueError, match="workspace"):
        el.epic_gemm_fp8(*args, workspace=_workspaces()[bad])
    assert len(calls) == 1


class _Plan:
    sizes, plan = el.epic_plan_sizes(), el.epic_plan()


def _model_args(n=2):
    """Arguments of a model call on host tensors; a layer call's are the first of each list."""
    t = lambda *s, dtype=torch.float32: torch.zeros(s, dtype=dtype)  # noqa: E731
    bf16 = torch.bfloat16
    return dict(cfg=el.epic_model_cfg(el.attn_cfg(2, 1, 64), 128, 128, n, 1e4, 1e-5),
                layers=[el.epic_layer_weights_fp8() for _ in range(n)], final_norm=t(128, dtype=bf16), dplan=_Plan(),
                hidden_s=t(3, 128), k_caches=[t(4, 1, 16, 64, dtype=bf16) for _ in range(n)],
                v_caches=[t(4, 1, 64, 16, dtype=bf16) for _ in range(n)], out_hidden=t(3, 128),
                workspace=t(512, dtype=torch.uint8))


def _layer_args(**kw):
    a = {**_model_args(1), **kw}
    return dict(cfg=a["cfg"], weights=a["layers"][0], dplan=a["dplan"], hidden_s=a["hidden_s"], k_cache=a["k_caches"][0],
                v_cache=a["v_caches"][0], workspace=a["workspace"])


@pytest.fixture
def on_host(monkeypatch):
    """Layer and model calls on host tensors, up to the library; returns the calls that got there."""
    calls = []
    monkeypatch.setattr(el, "_current_device", lambda: -1, raising=False)
    for name in ("_stream", "_raw_stream"):
        monkeypatch.setattr(el, name, lambda *args: None)
    for name in ("_link_layer_fp8", "_link_model_fp8"):
        monkeypatch.setattr(el, name, lambda *args: calls.append(args) or 0)
    return calls


def test_layer_and_model_refuse_tensors_of_other_memory(on_host):
    """A workspace of another device or with nothing behind it, and tensors whose rows lie apart."""
    el.epic_link_layer_fp8(**_layer_args())
    el.epic_link_model_fp8(**_model_args())
    assert len(on_host) == 2
    wide = torch.zeros(3, 256)[:, :128]
    k = torch.zeros(4, 16, 1, 64, dtype=torch.bfloat16)[:, ::2]
    for bad in [dict(workspace=w) for w in _workspaces()] + [dict(hidden_s=wide), dict(hidden_s=_Elsewhere()),
                                                             dict(k_caches=[k, k]), dict(v_caches=[_Elsewhere()] * 2)]:
        with pytest.raises(ValueError, match=next(iter(bad))[:7]):
            el.epic_link_layer_fp8(**_layer_args(**bad))
        with pytest.raises(ValueError, match=next(iter(bad))[:7]):
            el.epic_link_model_fp8(**{**_model_args(), **bad})
    for bad in (dict(out_hidden=wide), dict(final_norm=_Elsewhere())):
        with pytest.raises(ValueError):
            el.epic_link_model_fp8(**{**_model_args(), **bad})
    assert len(on_host) == 2


def test_model_refuses_other_numbers_of_layers(on_host):
    """The library reads cfg.n_layers entries of each list."""
    good = _model_args()
    for name in ("layers", "k_caches", "v_caches"):
        for n in (0, 1, 3):
            with pytest.raises(ValueError, match="2 layers"):
                el.epic_link_model_fp8(**{**good, name: (good[name] * 2)[:n]})
    with pytest.raises(ValueError, match="3 layers"):
        el.epic_link_model_fp8(**{**good, "cfg": _model_args(3)["cfg"]})
    assert not on_host


# ---------------------------------------------------------------- the kernel chosen by sizes

def route(epi, m, n, k):
    f = el._lib.epic_gemm_fp8_route_name
    f.restype = C.c_char_p
    return f(epi, m, n, k).decode()


@pytest.mark.parametrize("m,n,k", [(1, 128, 128), (4, 6144, 4096), (100, 28672, 4096), (128, 4096, 14336),
                                   (501, 4096, 4096), (736, 28672, 4096), (20560, 4096, 14336), (129, 256, 128)])
def test_every_size_has_a_kernel(m, n, k):
    for epi in range(3):
        assert route(epi, m, n, k) != ""


def test_gpu_cases_take_the_kernels_they_name():
    import test_gpu_fp8 as gpu
    for (m, n, k), kernels in gpu.ROUTES:
        assert tuple(route(e, m, n, k) for e in range(3)) == kernels, (m, n, k)
    seen = {name for _, kernels in gpu.ROUTES for name in kernels}
    assert seen == {"few", "stream", "narrow64x64", "narrow64x128", "narrow128x128", "narrow64x256", "whole128", "whole192",
                    "whole256", "split128", "split192", "split256"}


def test_model_cases_take_the_kernels_they_name():
    import oracle
    import test_gpu_fp8_model as gpu
    for wl, kernel in zip(gpu.CASES, gpu.QKV):
        rows = len(oracle.legolink_positions(wl.chunk_lens, wl.suffix_len, wl.k))
        assert route(3, rows, (wl.num_q_heads + 2 * wl.num_kv_heads) * wl.head_dim, wl.hidden) == kernel, wl.name


def test_plans_keep_within_what_they_need():
    """Row limits of the short-row kernels; and no planes where they would not fit the workspace."""
    rng = np.random.default_rng(9)
    for _ in range(3000):
        m, n, k = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (5000, 200, 130))
        n, k = 256 * n, 128 * k
        for e in range(4):
            name = route(e, m, n, k)
            assert name and (name != "few" or m <= 32) and (name != "stream" or m <= 128)
    for m in (1, 16, 32, 33, 128, 500):
        for n in (1 << 19, 1 << 20, 1 << 23):
            for e in range(4):
                name = route(e, m, n, 128)
                planes = {"few": 1, "stream": 2}.get(name, 2 if name.startswith("split") else 0)
                assert planes * 4 * m * n <= 64 << 20, (m, n, name)


def planes(epi, m, n, k):
    return el._lib.epic_gemm_fp8_planes(epi, m, n, k)


@pytest.mark.parametrize("epi,m,n,k", [(1, 100, 384, 256), (2, 4, 128, 128), (0, 1 << 24, 1024, 128), (0, 4, 128, 64), (0, 4, 64, 128),
                                       (0, 1, 1 << 24, 128), (0, (1 << 19) - 256, 128, 4096), (1, -1, 256, 128)])
def test_refused_sizes_have_no_planes(epi, m, n, k):
    """The query about partial sums and the entry point have one opinion on sizes."""
    assert planes(epi, m, n, k) == -1
    assert _gemm(epi=epi, m=m, n=n, k=k) in (INVALID, UNSUPPORTED)


def test_largest_row_count():
    """With 256 rows more the operands are below 2^31 bytes; of one row more they are not."""
    m = (1 << 19) - 257
    assert planes(0, m, 128, 4096) == 0 and planes(0, m + 1, 128, 4096) == -1


def test_partial_sums_fit_the_workspace():
    """Every plan's planes, whatever the sizes: many parts of a long k, many columns, all row counts of the kernels that
    leave planes."""
    rng = np.random.default_rng(10)
    most, size = {}, el.epic_gemm_fp8_workspace_bytes()
    for i in range(20000):
        m = int(np.exp(rng.uniform(0, np.log(150 if i % 2 else 5000))))
        n = 256 * int(np.exp(rng.uniform(0, np.log(1 << 14))))
        k = 128 * int(np.exp(rng.uniform(0, np.log(2000))))
        for e in range(4):
            p = planes(e, m, n, k)
            if p >= 0:
                kind = route(e, m, n, k).rstrip("0123456789x")
                assert p * 4 * m * n <= size, (e, m, n, k, kind, p)
                assert (p == 0) == (kind in ("whole", "narrow")) and (kind != "split" or 2 <= p <= 16)
                most[kind] = max(most.get(kind, 0), p)
    assert most["few"] == 1 and most["split"] == 16 and most["stream"] > 2

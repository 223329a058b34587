"""GPU parity of the 8-bit operators (epic_quant_fp8, epic_rmsnorm_fp8, epic_gemm_fp8) against
their definition in float64 (oracle.fp8).

Bars, fixed by the number formats:
  quant   the rounding is exact arithmetic: bytes and scales equal.
  norm    y differs from float64's by e = 2^-20 |y| (a fp32 sum of squares over up to 32768
          values in chains of at most 64, one square root, one division, two products: under
          16 roundings of 2^-24), then a half step of e4m3: 2^-4 |y|, or 2^-10 of the scale
          below the smallest normal value.  The scale may differ where the maximum is within e of
          a border.
  gemm    the matrix cores form a dot product of eight neighbouring values first, dropping of each
          product what is 13 bits below the largest one's exponent: at most 7 * 2^-13 of the
          largest, for each eight.  The fp32 sums above add at most K roundings of 2^-24 of
          the sum of magnitudes.  With both as e: bf16 |err| <= 2^-8 |y| + e, e4m3 the norm's bars.
          Over a whole result the dropped bits are independent of sign and size: 2^-12 of its
          2-norm beside the rounding of bf16.
Rows behind the last one, and bytes behind the last scale, stay as they were.
"""
import ctypes as C

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp8  # noqa: E402

pytestmark = pytest.mark.gpu

EPS = 1e-5


def _el():
    from paper_2410_15332_amd import epic_link as el
    return el


def _say(*what):
    print("[gpu-test] fp8", *what, flush=True)


def _guarded(shape, dtype=torch.uint8):
    """A tensor whose allocation goes on for 4 KB of 0xA5 behind it, and that guard."""
    n = int(np.prod(shape)) * torch.empty((), dtype=dtype).element_size()
    raw = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    return raw[:n].view(dtype).view(shape), raw[n:]


def _untouched(*guards):
    for g in guards:
        assert bool((g == 0xA5).all()), "written behind the end"


def _row_exponents(scale, m):
    return scale.cpu().numpy()[:, :m].T.astype(np.int64) - 127


def _activations(rng, m, k):
    size = np.exp(0.5 * rng.normal(size=k)) * np.where(rng.random(k) < 1 / 64, 12.0, 1.0)
    return rng.normal(size=(m, k)) * size


def _bf16(y):
    return torch.from_numpy(np.ascontiguousarray(y, np.float32)).to(torch.bfloat16)


# ---------------------------------------------------------------- quant

QUANT = [(1, 128), (2, 256), (3, 384), (5, 4096), (37, 640), (129, 1152), (300, 14336), (2049, 4096)]


def _quant(x, block_rows):
    el = _el()
    m, k = x.shape
    q, gq = _guarded((m, k))
    shape = el.fp8_row_scale_shape(m, k) if block_rows == 1 else el.fp8_block_scale_shape(m, k)
    s, gs = _guarded(shape)
    el.epic_quant_fp8(x.cuda(), q, s, block_rows=block_rows)
    torch.cuda.synchronize()
    _untouched(gq, gs)
    t = _row_exponents(s, m) if block_rows == 1 else s.cpu().numpy().astype(np.int64) - 127
    return q.cpu().numpy(), t


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("m,k", QUANT)
def test_quant(m, k, block_rows):
    _say("quant", m, k, block_rows)
    rng = np.random.default_rng([m, k])
    x = _bf16(_activations(rng, m, k))
    q, t = _quant(x, block_rows)
    rq, rt = fp8.quantise(x.double().numpy(), block_rows)
    assert np.array_equal(t, rt)
    assert np.array_equal(q, rq)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant_of_odd_values(block_rows):
    """Groups of zeros, of signed zeros, of the largest and the smallest bf16 values, borders of a
    scale, ties of the rounding, infinities and NaN."""
    _say("quant odd values", block_rows)
    rng = np.random.default_rng(8)
    m, k = 140, 512
    x = rng.normal(size=(m, k))
    x[0] = 0.0
    x[1] = -0.0
    x[2, :128] = 3.38e38 * np.where(rng.random(128) < 0.5, 1, -1)
    x[3, :128] = 2.0 ** -133 * rng.integers(-9, 9, 128)
    x[4, :128] = 448.0
    x[5, 128:256] = 450.0
    x[6] = rng.integers(-64, 65, k) * 2.0 ** -6 * 7
    x[7, 5], x[7, 200], x[7, 300] = np.nan, np.inf, -np.inf
    x[8] = np.nan
    x[9, 128:256] = np.inf
    x = _bf16(x)
    with np.errstate(invalid="ignore"):
        ref = x.double().numpy()
    q, t = _quant(x, block_rows)
    rq, rt = fp8.quantise(ref, block_rows)
    assert np.array_equal(t, rt)
    bad = (rq & 0x7F) == 0x7F
    assert np.array_equal((q & 0x7F) == 0x7F, bad)
    assert np.array_equal(q[~bad], rq[~bad])


# ---------------------------------------------------------------- norm

def _check_rounded(q, t, y, e):
    """Bytes q and exponents t against values y known to within e (elementwise), by the bars above."""
    m, k = y.shape
    top, slack = fp8.group_top(y), fp8.group_top(np.broadcast_to(e, y.shape))
    lo, hi = fp8.scale_exponent(np.maximum(top - slack, 0.0)), fp8.scale_exponent(top + slack)
    assert np.all((t >= lo) & (t <= hi)), "scale"
    step = np.ldexp(1.0, fp8.spread(t, m, k))
    bar = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * step) * (1 + 2.0 ** -4) + e
    off = np.abs(fp8.dequantise(q, t) - y)
    assert np.all(off <= bar), f"off by {np.max(off / bar):.3f} of the bar"


def _norm(x, delta, w, in_place=False, keep=True):
    el = _el()
    m, k = x.shape
    q, gq = _guarded((m, k))
    s, gs = _guarded(el.fp8_row_scale_shape(m, k))
    xd = torch.from_numpy(x).cuda()
    out, go = (xd, s[:0]) if in_place else _guarded((m, k), torch.float32) if keep else (None, s[:0])
    el.epic_rmsnorm_fp8(xd, w.cuda(), EPS, q, s, delta=None if delta is None else delta.cuda(), x_out=out)
    torch.cuda.synchronize()
    _untouched(gq, gs, go)
    if not in_place:
        assert np.array_equal(xd.cpu().numpy(), x, equal_nan=True)
    return q.cpu().numpy(), _row_exponents(s, m), None if out is None else out.cpu().numpy()


def _normed(x, w):
    return x / np.sqrt(np.mean(x * x, -1, keepdims=True) + EPS) * w.double().numpy()


NORM = [(1, 128, 0), (1, 4096, 1), (2, 256, 1), (3, 384, 1), (7, 1152, 0), (33, 8192, 1), (511, 640, 0), (512, 4096, 1),
        (700, 8320, 1), (130, 32768, 1), (1025, 128, 1), (600, 2048, 0)]


@pytest.mark.parametrize("m,k,add", NORM)
def test_norm(m, k, add):
    _say("norm", m, k, add)
    rng = np.random.default_rng([m, k, add])
    x = _activations(rng, m, k).astype(np.float32)
    delta = _bf16(rng.normal(size=(m, k))) if add else None
    w = _bf16(1 + 0.1 * rng.normal(size=k))
    q, t, s = _norm(x, delta, w)
    assert np.array_equal(s, x + delta.float().numpy() if add else x)     # one fp32 addition
    y = _normed(s.astype(np.float64), w)
    _check_rounded(q, t, y, 2.0 ** -20 * np.abs(y))


def test_norm_in_place_and_without_the_sum():
    _say("norm in place")
    rng = np.random.default_rng(5)
    x = rng.normal(size=(9, 1024)).astype(np.float32)
    delta = _bf16(rng.normal(size=(9, 1024)))
    w = _bf16(1 + 0.1 * rng.normal(size=1024))
    a, b, c = _norm(x, delta, w), _norm(x, delta, w, in_place=True), _norm(x, delta, w, keep=False)
    for i in range(3):
        assert np.array_equal(a[i], b[i])
    assert np.array_equal(a[0], c[0]) and np.array_equal(a[1], c[1])


def test_norm_of_odd_rows():
    """Rows of zeros, tiny and huge rows, and rows with NaN or an infinity, which touch no other row."""
    _say("norm odd rows")
    rng = np.random.default_rng(6)
    x = rng.normal(size=(8, 512)).astype(np.float32)
    x[1] = 0.0
    x[2] *= 1e-30
    x[3] *= 1e15
    x[4, 7] = np.nan
    x[5, 9] = np.inf
    w = _bf16(1 + 0.1 * rng.normal(size=512))
    q, t, _ = _norm(x, None, w)
    good = [0, 1, 2, 3, 6, 7]
    y = _normed(x[good].astype(np.float64), w)
    _check_rounded(q[good], t[good], y, 2.0 ** -20 * np.abs(y))
    assert np.all((q[4] & 0x7F) == 0x7F)                    # NaN everywhere
    assert (q[5, 9] & 0x7F) == 0x7F and np.all((np.delete(q[5], 9) & 0x7F) == 0)   # 1 / inf


# ---------------------------------------------------------------- gemm

EPI = {"bf16": 0, "swiglu": 1, "swiglu_fp8": 2}


def _operands(rng, m, n, k):
    """Quantised rows and weights, and what they stand for."""
    qa, ta = fp8.quantise(_activations(rng, m, k))
    qw, tw = fp8.quantise(rng.normal(size=(n, k)) * np.exp(rng.normal(size=(n, 1))) * 0.5 / np.sqrt(k), 128)
    return qa, ta, qw, tw


def _device(codes):
    return torch.from_numpy(codes).cuda()


def _device_rows(t):
    """Row exponents [m, k / 128] in the library's layout; the padding is NaN's byte."""
    m, g = t.shape
    s = np.full((g, -(-m // 4) * 4), 0xFF, np.uint8)
    s[:, :m] = (t + 127).T
    return torch.from_numpy(s).cuda()


def _products(a, w):
    """a w^T in float64 and the bar e of every sum: see above."""
    a, w = torch.from_numpy(a).cuda(), torch.from_numpy(w).cuda()
    (m, k), n = a.shape, w.shape[0]
    y = a @ w.t().contiguous()
    e = k * 2.0 ** -24 * (a.abs() @ w.abs().t().contiguous())
    step = max(1, int(1e8) // (n * k))
    for r in range(0, m, step):
        p = (a[r:r + step, None].abs() * w[None].abs()).view(-1, n, k // 8, 8)
        e[r:r + step] += 7 * 2.0 ** -13 * p.amax(-1).sum(-1)
    return y.cpu().numpy(), e.cpu().numpy()


def _run_gemm(epi, qa, ta, qw, tw, stale=0xAB):
    el = _el()
    (m, k), n = qa.shape, qw.shape[0]
    ws, gw = _guarded((el.epic_gemm_fp8_workspace_bytes(),))
    ws.fill_(stale)                                         # stale contents must not matter
    out, go = _guarded((m, n if epi == "bf16" else n // 2), torch.uint8 if epi == "swiglu_fp8" else torch.bfloat16)
    ss, gs = _guarded(el.fp8_row_scale_shape(m, n // 2)) if epi == "swiglu_fp8" else (None, gw)
    el.epic_gemm_fp8(EPI[epi], _device(qa), _device_rows(ta), _device(qw), _device((tw + 127).astype(np.uint8)), out,
                     out_scale=ss, workspace=ws)
    torch.cuda.synchronize()
    _untouched(gw, go, gs)
    if ss is None:
        return out.float().cpu().numpy()
    return out.cpu().numpy(), _row_exponents(ss, m)


def _silu(x):
    return x / (1 + np.exp(-x))


def _check_gemm(epi, m, n, k, seed=0):
    rng = np.random.default_rng([m, n, k, seed])
    qa, ta, qw, tw = _operands(rng, m, n, k)
    y, e = _products(fp8.dequantise(qa, ta), fp8.dequantise(qw, tw, 128))
    got = _run_gemm(epi, qa, ta, qw, tw)
    if epi != "bf16":
        gate, up, eg, eu = y[:, :n // 2], y[:, n // 2:], e[:, :n // 2], e[:, n // 2:]
        y = _silu(gate) * up
        # silu has slope at most 1.1; its own arithmetic (exp2, reciprocal, products) is below 2^-19
        e = 1.1 * eg * (np.abs(up) + eu) + np.abs(_silu(gate)) * eu + 2.0 ** -19 * np.abs(y)
    if epi == "swiglu_fp8":
        _check_rounded(got[0], got[1], y, e)
    else:
        assert np.all(np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -8) * e)
        rounded = torch.from_numpy(y).to(torch.bfloat16).double().numpy()
        assert np.linalg.norm(got - y) <= 1.1 * np.linalg.norm(rounded - y) + 2.0 ** -12 * np.linalg.norm(y)


ROWS = [1, 2, 3, 5, 16, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 385, 513, 736]


@pytest.mark.parametrize("epi", list(EPI))
@pytest.mark.parametrize("m", ROWS)
def test_gemm_rows(m, epi):
    _say("gemm rows", m, epi)
    _check_gemm(epi, m, 512, 640)


SHAPES = [(1, 256, 128), (4, 256, 14336), (17, 2304, 256), (33, 768, 1920), (100, 4096, 1024), (96, 8192, 128),
          (150, 256, 8192), (300, 1280, 384), (129, 256, 128), (260, 4096, 4096), (1000, 768, 1024), (2000, 6144, 512)]


@pytest.mark.parametrize("epi", list(EPI))
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_gemm_shapes(m, n, k, epi):
    _say("gemm shapes", m, n, k, epi)
    _check_gemm(epi, m, n, k)


@pytest.mark.parametrize("m,n,k", [(7, 128, 128), (70, 384, 256), (200, 128, 512), (300, 1408, 384)])
def test_gemm_odd_block_counts(m, n, k):
    """n a multiple of 128 but not of 256."""
    _say("gemm odd blocks", m, n, k)
    _check_gemm("bf16", m, n, k)


@pytest.mark.parametrize("m", [3, 50, 120, 300])
def test_gemm_scales_are_applied_blockwise(m):
    """Every group and block at a scale of its own, far apart: a misplaced scale is off by powers of two."""
    _say("gemm scales", m)
    rng = np.random.default_rng(m)
    n, k = 512, 1024
    qa, qw = (fp8.e4m3_encode(rng.integers(-8, 9, s).astype(np.float64)) for s in ((m, k), (n, k)))
    ta = rng.integers(-20, 21, (m, k // 128))
    tw = rng.integers(-20, 21, (n // 128, k // 128))
    y, e = _products(fp8.dequantise(qa, ta), fp8.dequantise(qw, tw, 128))
    got = _run_gemm("bf16", qa, ta, qw, tw)
    assert np.all(np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + (1 + 2.0 ** -8) * e)


@pytest.mark.parametrize("m", [1, 40, 90, 300])
def test_gemm_of_small_integers_is_exact(m):
    """Products of up to 2^6 and sums below 2^24: every addition is exact, and so any layout or index fault shows."""
    _say("gemm integers", m)
    rng = np.random.default_rng(m)
    n, k = 768, 1152
    ia, iw = rng.integers(-8, 9, (m, k)), rng.integers(-8, 9, (n, k))
    zeros = lambda r: np.zeros((r, k // 128), np.int64)  # noqa: E731
    got = _run_gemm("bf16", fp8.e4m3_encode(ia.astype(float)), zeros(m), fp8.e4m3_encode(iw.astype(float)), zeros(n // 128))
    assert np.array_equal(got, _bf16(ia @ iw.T).float().numpy())


@pytest.mark.parametrize("m", [5, 100, 400])
def test_gemm_every_e4m3_value(m):
    """All 254 finite codes, subnormal ones among them, against weights of a single 1 per row."""
    _say("gemm every value", m)
    n = k = 256
    qa = np.tile(np.where((np.arange(256) & 0x7F) == 0x7F, 0, np.arange(256)).astype(np.uint8), (m, 1))
    qa = np.stack([np.roll(r, i) for i, r in enumerate(qa)])
    qw = fp8.e4m3_encode(np.eye(n, k))
    got = _run_gemm("bf16", qa, np.zeros((m, 2), np.int64), qw, np.zeros((2, 2), np.int64))
    assert np.array_equal(got, fp8.e4m3_decode(qa).astype(np.float32))


@pytest.mark.parametrize("m", [4, 70, 300])
def test_gemm_nan_stays_in_its_row_and_column(m):
    _say("gemm nan", m)
    rng = np.random.default_rng(m)
    qa, ta, qw, tw = _operands(rng, m, 256, 384)
    clean = _run_gemm("bf16", qa, ta, qw, tw)
    qa[m // 2, 200], qw[17, 5] = 0x7F, 0xFF
    got = _run_gemm("bf16", qa, ta, qw, tw)
    bad = np.zeros(got.shape, bool)
    bad[m // 2], bad[:, 17] = True, True
    assert np.all(np.isnan(got[bad])) and np.array_equal(got[~bad], clean[~bad])

"""8-bit operands of the projections, from their definition (NumPy, float64).

e4m3: sign, 4 exponent bits (bias 7), 3 fraction bits; the largest finite value is 448,
the smallest positive one 2^-9; there are no infinities and S.1111.111 is NaN.  A group
(128 consecutive values of a row, or a 128 x 128 block of weights) has one power-of-two
scale 2^t, t the smallest integer with max |y| <= 448 * 2^t over the group's finite values
(0 where they are all 0), kept within [-127, 127].
"""
import numpy as np

GROUP = 128
TOP = 448.0


def _table():
    v = np.empty(128)
    for b in range(128):
        e, f = b >> 3, b & 7
        v[b] = f / 8.0 * 2.0 ** -6 if e == 0 else (1 + f / 8.0) * 2.0 ** (e - 7)
    v[127] = np.nan
    return v


POSITIVE = _table()


def e4m3_decode(codes):
    """The values of e4m3 bytes."""
    codes = np.asarray(codes, np.uint8)
    return np.where(codes & 0x80, -1.0, 1.0) * POSITIVE[codes & 0x7F]


def e4m3_encode(y):
    """The e4m3 bytes nearest to y (|y| <= 448; ties to the even code); NaN and infinities give 0x7F."""
    y = np.asarray(y, np.float64)
    a = np.where(np.isfinite(y), np.abs(y), 0.0)
    assert np.all(a <= TOP)
    hi = np.searchsorted(POSITIVE[:127], a)                  # first value >= a
    lo = np.maximum(hi - 1, 0)
    up, down = POSITIVE[hi] - a, a - POSITIVE[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = (code | np.where(np.signbit(y), 0x80, 0)).astype(np.uint8)
    return np.where(np.isfinite(y), code, 0x7F).astype(np.uint8)


def scale_exponent(top):
    """t of a group whose largest finite magnitude is top."""
    f, x = np.frexp(np.asarray(top, np.float64))             # top = f 2^x, 0.5 <= f < 1;  448 = 0.875 * 2^9
    t = np.where(f <= 0.875, x - 9, x - 8)
    return np.clip(np.where(np.asarray(top) > 0, t, 0), -127, 127)


def group_top(y, block_rows=1):
    """Largest finite magnitude of every group of y [m, k]: [ceil(m / block_rows), k / 128]."""
    m, k = y.shape
    top = np.where(np.isfinite(y), np.abs(y), 0.0).reshape(m, k // GROUP, GROUP).max(-1)
    return np.stack([top[r:r + block_rows].max(0) for r in range(0, m, block_rows)])


def spread(t, m, k, block_rows=1):
    """A value per group as one per element."""
    return np.repeat(np.repeat(t, block_rows, 0)[:m], GROUP, 1)[:, :k]


def quantise(y, block_rows=1):
    """y [m, k] -> (e4m3 bytes [m, k], exponents t per group)."""
    m, k = y.shape
    t = scale_exponent(group_top(y, block_rows))
    return e4m3_encode(np.ldexp(y, -spread(t, m, k, block_rows))), t


def dequantise(codes, t, block_rows=1):
    """What bytes and exponents stand for."""
    m, k = codes.shape
    return np.ldexp(e4m3_decode(codes), spread(t, m, k, block_rows))


# ---------------------------------------------------------------- the decoder layer on 8-bit projections

def rows(y):
    """What the rows y stand for after rounding to e4m3 with their scales."""
    return dequantise(*quantise(y))


def weights(w):
    """A layer's bf16 matrices (bit patterns) rounded to e4m3 in 128 x 128 blocks; norms as they are."""
    from .model import _bf16_to_f64

    out = {}
    for name, bits in w.items():
        v = _bf16_to_f64(bits)
        out[name] = v if v.ndim == 1 else dequantise(*quantise(v, GROUP), GROUP)
    return out


def decoder_layer(h, s_pos, w, cached_k, cached_v, n_total, ffn, hq, hkv, d, theta, eps):
    """model.decoder_layer with every product's input rows rounded to e4m3 (w: weights()'s);
    q, k, v and the attention output are bf16 before that, the residual stream is not rounded.
    Returns (h, k, v, and what the layer's two branches added to h)."""
    from .link import _round_bf16, expand_kv, masked_attention, rope
    from .model import _silu, rmsnorm

    n, h = len(s_pos), np.asarray(h, np.float64)
    qkv = rows(rmsnorm(h, w["attn_norm"], eps)) @ w["wqkv"].T
    q = _round_bf16(rope(qkv[:, :hq * d].reshape(n, hq, d), s_pos, theta))
    k = _round_bf16(rope(qkv[:, hq * d:(hq + hkv) * d].reshape(n, hkv, d), s_pos, theta))
    v = _round_bf16(qkv[:, (hq + hkv) * d:].reshape(n, hkv, d))
    K, V = expand_kv(cached_k, cached_v, s_pos, k, v, n_total)
    o = _round_bf16(masked_attention(q, K, V, s_pos)[0].reshape(n, hq * d))
    attn = rows(o) @ w["wo"].T
    gu = rows(rmsnorm(h + attn, w["mlp_norm"], eps)) @ w["w_gate_up"].T
    mlp = rows(_silu(gu[:, :ffn]) * gu[:, ffn:]) @ w["w_down"].T
    return h + attn + mlp, k, v, (attn, mlp)

"""The 8-bit cache, from its definition (NumPy, float64).

A row (the D values of K or of V of a token and KV head) is e4m3 values and a scale byte t + 127,
t the smallest integer in [-127, 127] with max |y| <= 448 * 2^t (0 for a row of zeros).  A token
with a value of K or V that is not finite is NaN: bytes 255 in both, K codes 0x7F, V codes 0.

A cache here is a dict of token-major arrays: k, v [blocks, Hkv, 16, D] codes and ks, vs
[blocks, Hkv, 16] bytes; ``layout`` gives the stored order of k and v.
"""
import numpy as np

from . import fp8

NAN = 255
CODES = fp8.e4m3_decode(np.arange(256))


def quantise(k, v):
    """K and V rows [..., D] -> (k codes, v codes, k bytes, v bytes)."""
    nan = ~(np.isfinite(k).all(-1) & np.isfinite(v).all(-1))
    out = []
    for y, code in ((k, 0x7F), (v, 0)):
        y = np.where(nan[..., None], 0.0, y)
        t = fp8.scale_exponent(np.abs(y).max(-1))
        q = fp8.e4m3_encode(np.ldexp(y, -t[..., None]))
        out.append((np.where(nan[..., None], np.uint8(code), q), np.where(nan, NAN, t + 127).astype(np.uint8)))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def values(codes, byte):
    """What codes [..., D] and scale bytes [...] stand for."""
    y = np.ldexp(CODES[codes], byte.astype(np.int64)[..., None] - 127)
    return np.where((byte == NAN)[..., None], np.nan, y)


def layout(k, v):
    """Token-major codes [blocks, Hkv, 16, D] in the stored order, element by element."""
    n, h, _, d = k.shape
    ks, vs = np.empty((n, h, d // 64, 4, 16, 16), np.uint8), np.empty((n, h, d // 64, 4, 16, 4, 4), np.uint8)
    for dim in range(d):
        j, i = divmod(dim, 64)
        for s in range(16):
            ks[:, :, j, i // 16, s, i % 16] = k[:, :, s, dim]
            vs[:, :, j, s // 4, i % 16, i // 16, s % 4] = v[:, :, s, dim]
    return ks, vs


def tokens(ks, vs):
    """The reverse of layout."""
    n, h, j_n = ks.shape[:3]
    k, v = np.empty((n, h, 16, 64 * j_n), np.uint8), np.empty((n, h, 16, 64 * j_n), np.uint8)
    for dim in range(64 * j_n):
        j, i = divmod(dim, 64)
        for s in range(16):
            k[:, :, s, dim] = ks[:, :, j, i // 16, s, i % 16]
            v[:, :, s, dim] = vs[:, :, j, s // 4, i % 16, i // 16, s % 4]
    return k, v


def copy(c):
    return {name: x.copy() for name, x in c.items()}


def write(c, views, k_s, v_s, theta=None):
    """The link write on cache c, in place: every private block of the plan takes its source's rows (K turned by
    priv_rot), then the rows k_s, v_s [n, Hkv, D] of S; a slot with neither is a row of zeros."""
    from .link import rope

    k, v, ks, vs = quantise(k_s, v_s)
    old = copy(c)
    for i, (dst, src) in enumerate(zip(views["priv_block"], views["priv_src"])):
        for name, fill in (("k", 0), ("v", 0), ("ks", 127), ("vs", 127)):
            c[name][dst] = old[name][src] if src >= 0 else fill
        rot = int(views["priv_rot"][i])
        if rot and src >= 0:
            y = values(old["k"][src], old["ks"][src])                     # [Hkv, 16, D]
            nan = old["ks"][src] == NAN
            y = rope(np.where(nan[..., None], 0.0, y).transpose(1, 0, 2), np.full(16, rot), theta).transpose(1, 0, 2)
            q, _, b, _ = quantise(y, np.zeros_like(y))
            c["k"][dst] = np.where(nan[..., None], old["k"][src], q)
            c["ks"][dst] = np.where(nan, NAN, b)
        for s, r in enumerate(views["priv_rows"][16 * i:16 * i + 16]):
            if r >= 0:
                c["k"][dst, :, s], c["v"][dst, :, s] = k[r], v[r]
                c["ks"][dst, :, s], c["vs"][dst, :, s] = ks[r], vs[r]


def linked(c, views, req):
    """K and V [N, Hkv, D] of request req through its linked block table."""
    at = slice(int(views["blk_off"][req]), int(views["blk_off"][req + 1]))
    blocks = views["linked_blocks"][at]
    held = np.arange(16) < views["block_len"][at][:, None]
    return [values(c[name][blocks].swapaxes(1, 2)[held], c[byte][blocks].swapaxes(1, 2)[held])
            for name, byte in (("k", "ks"), ("v", "vs"))]


def attention(q, K, V, pos, scale=None):
    """Masked attention of rows q at positions pos over K and V that may hold NaN tokens: (out, lse, NaN rows [n, Hq]).
    A row that attends to a NaN token is one; its out and lse here are those without such tokens' values."""
    from .link import masked_attention

    nan = np.isnan(K).any(-1) | np.isnan(V).any(-1)                      # [N, Hkv]
    bad = np.stack([nan[:p + 1].any(0) for p in pos]) if len(pos) else np.zeros((0, K.shape[1]), bool)
    out, lse = masked_attention(q, np.where(nan[..., None], 0.0, K), np.where(nan[..., None], 0.0, V), pos, scale)
    return out, lse, np.repeat(bad, q.shape[1] // K.shape[1], 1)

"""GPU parity of the 8-bit cache (epic_kv8_pack, epic_kv8_unpack, epic_link_attention_kv8) against its
definition in float64 (oracle.kv8).

Bars.  Moving blocks and the link write are exact arithmetic: codes and scale bytes equal, every other block as it
was.  Re-rotated keys are fp32 sums of two products off by 2^-22 of the sum of their magnitudes: their codes
may differ by one where that is next to a border, scales by one likewise; most are equal.
Attention, against float64 over the same cache: with e = (D + 8) 2^-24 scale |q| max |k| what fp32 sums leave of a
score, n keys and A = sum p |v|, the weights are off by 2 e + 2^-22 + 2 n 2^-24 of themselves before they are
rounded to bf16 (2^-8), their sum likewise without the rounding, and the result is rounded (2^-8); lse by
e + 2^-22 + n 2^-24, and 2^-22 of itself.
"""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import fp8, kv8  # noqa: E402
from oracle.link import masked_attention, rope as rope_at  # noqa: E402

pytestmark = pytest.mark.gpu

THETA = 500000.0


def _el():
    from paper_2410_15332_amd import epic_link as el
    return el


def _say(*what):
    print("[gpu-test] kv8", *what, flush=True)


def _bf16(x):
    """float64 array -> (bf16 tensor on the GPU, the values it holds)."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float64)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


def _rows(rng, *shape):
    """Values with channels of unlike size."""
    return rng.normal(size=shape) * np.exp(0.7 * rng.normal(size=shape[-1]))


def _cache(rng, blocks, hkv, d):
    k, v, ks, vs = kv8.quantise(_rows(rng, blocks, hkv, 16, d), _rows(rng, blocks, hkv, 16, d))
    return {"k": k, "v": v, "ks": ks, "vs": vs}


def _upload(c):
    k, v = kv8.layout(c["k"], c["v"])
    scale = np.stack((c["ks"], c["vs"]), 2)
    return _el().Kv8Cache(*(torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (k, v, scale)))


def _download(cache):
    k, v = kv8.tokens(cache.k.cpu().numpy(), cache.v.cpu().numpy())
    s = cache.scale.cpu().numpy()
    return {"k": k, "v": v, "ks": s[:, :, 0].copy(), "vs": s[:, :, 1].copy()}


def _equal(got, want, what=""):
    for name in want:
        diff = got[name] != want[name]
        assert not diff.any(), f"{what} {name}: {diff.sum()} of {diff.size} differ, first at {np.argwhere(diff)[0]}"


# ---------------------------------------------------------------- blocks between the two kinds of cache

def _special(rng, blocks, hkv, d):
    """Tokens at borders: zeros, the smallest and largest bf16, maxima at 448 2^t and next to it, ties of the
    rounding, and values that are not finite in K alone, in V alone, in both."""
    x = _rows(rng, 2, blocks, hkv, 16, d)
    n = 0
    for b in range(blocks):
        for g in range(hkv):
            for s in range(16):
                for y in (x[0, b, g, s], x[1, b, g, s]):
                    kind, n = n % 17, n + 1
                    if kind == 0:
                        y[:] = 0.0
                    elif kind == 1:
                        y[:] = 0.0
                        y[rng.integers(d)] = -2.0 ** -133
                    elif kind == 2:
                        y *= 2.0 ** -125
                    elif kind == 3:
                        y[:] = rng.choice([-1, 1], d) * rng.integers(0, 128, d) * 2.0 ** -133
                    elif kind == 4:
                        y *= 2.0 ** 122 / np.abs(y).max()
                        y[0] = 255 * 2.0 ** 120
                    elif kind == 5:
                        y /= np.abs(y).max() / 200.0
                        y[3] = 448.0
                    elif kind == 6:
                        y /= np.abs(y).max() / 200.0
                        y[3] = -450.0
                    elif kind == 7:                      # ties: half steps of every binade
                        y[:] = (rng.integers(8, 16, d) + 0.5) * 2.0 ** rng.integers(-9, 5, d)
                        y[0] = 448.0
                    elif kind == 8:                      # and below the normal values
                        y[:] = (rng.integers(0, 8, d) + 0.5) * 2.0 ** -9
                        y[0] = 256.0
                    elif kind == 9 and b % 3 == 1:
                        y[rng.integers(d)] = rng.choice([np.inf, -np.inf, np.nan])
                    elif kind == 10:
                        y *= np.exp(20 * rng.normal(size=d))
                    elif kind == 11:
                        y *= np.exp(-30 * rng.random())
    return x


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 3, 4, 8, 9])
def test_pack_is_the_definition(hkv, d):
    el = _el()
    _say("pack", hkv, d)
    rng = np.random.default_rng([hkv, d])
    n = 11
    x = _special(rng, n, hkv, d)
    kt, k = _bf16(x[0])
    vt, v = _bf16(x[1].swapaxes(-1, -2))
    assert np.isfinite(k).sum() < k.size and np.abs(k[np.isfinite(k)]).max() > 2.0 ** 127
    cache = el.Kv8Cache.zeros(n, hkv, d)
    el.epic_kv8_pack(kt, vt, cache)
    kq, vq, ks, vs = kv8.quantise(k, v.swapaxes(-1, -2))
    _equal(_download(cache), {"k": kq, "v": vq, "ks": ks, "vs": vs})
    assert (ks == 255).any() and (ks < 3).any() and ks[ks < 255].max() >= 246


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 5, 8])
def test_unpack_is_the_values(hkv, d):
    el = _el()
    _say("unpack", hkv, d)
    rng = np.random.default_rng([hkv, d, 1])
    n = 7
    kq, vq, ks, vs = kv8.quantise(*_special(rng, n, hkv, d))
    # every code, and every scale
    kq[0, 0] = np.resize(np.r_[0:0x7F, 0x80:0xFF], (16, d))
    ks[0, 0] = np.arange(16) * 16
    vq[1, 0] = np.resize(np.r_[0:0x7F, 0x80:0xFF], (16, d))
    vs[1, 0] = 254 - np.arange(16)
    nan = (ks == 255) | (vs == 255)
    ks[nan], vs[nan], kq[nan], vq[nan] = 255, 255, 0x7F, 0
    cache = _upload({"k": kq, "v": vq, "ks": ks, "vs": vs})
    k = torch.zeros((n, hkv, 16, d), dtype=torch.bfloat16, device="cuda")
    v = torch.zeros((n, hkv, d, 16), dtype=torch.bfloat16, device="cuda")
    el.epic_kv8_unpack(cache, k, v)
    for got, q, b in ((k, kq, ks), (v.transpose(-1, -2), vq, vs)):
        want = torch.from_numpy(kv8.values(q, b)).float().to(torch.bfloat16).float()
        assert torch.equal(torch.isnan(got.float().cpu()), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(got.float().cpu(), 0.0, posinf=1.0, neginf=-1.0),
                           torch.nan_to_num(want, 0.0, posinf=1.0, neginf=-1.0))


@pytest.mark.parametrize("n", [1, 2, 63, 1000])
def test_moves_by_lists(n):
    """Lists in any order, ids outside either pool, one block of the source twice: the listed blocks move,
    the others stay; and a block that went to 8 bits and back stands for the same values when packed again.
    (Not by the same bytes: a row whose largest value was rounded down, 225 2^t to 224 2^t = 448 2^(t-1), has the
    scale 2^(t-1) then, over which its values are e4m3 too, twice as large.)"""
    el = _el()
    _say("lists", n)
    rng = np.random.default_rng(n)
    hkv, d, pool_a, pool_b = 3, 64, n + 5, n + 9
    kt, k = _bf16(_rows(rng, pool_a, hkv, 16, d))
    vt, v = _bf16(_rows(rng, pool_a, hkv, d, 16))
    start = _cache(rng, pool_b, hkv, d)
    cache = _upload(start)
    src, dst = rng.integers(0, pool_a, n), rng.permutation(pool_b)[:n]
    if n > 10:
        src[3], src[4], dst[5], dst[6], src[7] = -1, pool_a, pool_b, -5, 2 ** 31 - 1
    st, dt = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (src, dst))
    el.epic_kv8_pack(kt, vt, cache, st, dt)
    want = kv8.copy(start)
    ok = (src >= 0) & (src < pool_a) & (dst >= 0) & (dst < pool_b)
    for name, x in zip(("k", "v", "ks", "vs"), kv8.quantise(k[src[ok]], v[src[ok]].swapaxes(-1, -2))):
        want[name][dst[ok]] = x
    got = _download(cache)
    _equal(got, want, "pack")
    back_k, back_v = torch.full_like(kt, 3.0), torch.full_like(vt, 3.0)
    back = rng.permutation(pool_a)[:n]
    bt = torch.from_numpy(back.astype(np.int32)).cuda()
    el.epic_kv8_unpack(cache, back_k, back_v, dt, bt)
    wk, wv = np.full(k.shape, 3.0), np.full(v.shape, 3.0)
    fine = (dst >= 0) & (dst < pool_b)
    wk[back[fine]] = kv8.values(want["k"], want["ks"])[dst[fine]]
    wv[back[fine]] = kv8.values(want["v"], want["vs"])[dst[fine]].swapaxes(-1, -2)
    assert np.array_equal(back_k.double().cpu().numpy(), wk) and np.array_equal(back_v.double().cpu().numpy(), wv)
    again = el.Kv8Cache.zeros(pool_b, hkv, d)
    el.epic_kv8_pack(back_k, back_v, again, bt, dt)
    a, at = _download(again), dst[fine]
    for x, scale in (("k", "ks"), ("v", "vs")):
        assert np.array_equal(kv8.values(a[x][at], a[scale][at]), kv8.values(want[x][at], want[scale][at]))


def test_moves_refuse():
    el = _el()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    k, v, cache = torch.zeros(4, 2, 16, 64, **bf), torch.zeros(4, 2, 64, 16, **bf), el.Kv8Cache.zeros(6, 2, 64)
    i = torch.zeros(3, dtype=torch.int32, device="cuda")
    for args, kw in (((k, v, cache), {}), ((k, v[:3], cache), dict(src_blocks=i, dst_blocks=i)),
                     ((k.float(), v, cache), dict(src_blocks=i)), ((k, v, el.Kv8Cache.zeros(6, 4, 64)), dict(src_blocks=i)),
                     ((k, v, cache), dict(src_blocks=i.long())), ((k, v, cache), dict(src_blocks=i, dst_blocks=i[:2])),
                     ((k, v, cache), dict(src_blocks=i.cpu())), ((k.transpose(1, 2).contiguous().transpose(1, 2), v, cache), dict(src_blocks=i))):
        with pytest.raises(ValueError):
            el.epic_kv8_pack(*args, **kw)
    with pytest.raises(el.EpicError):                    # five blocks without a list, a pool of four
        el.epic_kv8_pack(k, v, cache, dst_blocks=torch.zeros(5, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()


def test_moves_follow_the_caches_tensors():
    """After its tensors were replaced by larger ones, and after those were resized, a cache is read and written where they
    are, and the memory that they left stays as it is."""
    el = _el()
    rng = np.random.default_rng(8)
    hkv, d = 2, 64
    kt, k = _bf16(_rows(rng, 30, hkv, 16, d))
    vt, v = _bf16(_rows(rng, 30, hkv, d, 16))
    cache = el.Kv8Cache.zeros(5, hkv, d)
    first = cache.k, cache.v, cache.scale
    for n in (5, 9, 30, 7):
        if n == 9:
            cache.k, cache.v, cache.scale = (torch.zeros(s, dtype=torch.uint8, device="cuda") for s in el.kv8_shapes(n, hkv, d))
            for t in first:
                t.fill_(0x11)
        elif n != 5:
            for t, s in zip((cache.k, cache.v, cache.scale), el.kv8_shapes(n, hkv, d)):
                t.resize_(s)
        kn, vn = kt[30 - n:], vt[30 - n:]
        el.epic_kv8_pack(kn, vn, cache)
        kq, vq, ks, vs = kv8.quantise(k[30 - n:], v[30 - n:].swapaxes(-1, -2))
        _equal(_download(cache), {"k": kq, "v": vq, "ks": ks, "vs": vs}, f"{n} blocks")
        back_k, back_v = torch.empty_like(kn), torch.empty_like(vn)
        el.epic_kv8_unpack(cache, back_k, back_v)
        assert np.array_equal(back_k.double().cpu().numpy(), kv8.values(kq, ks))
        assert np.array_equal(back_v.double().cpu().numpy(), kv8.values(vq, vs).swapaxes(-1, -2))
    assert all(bool((t == 0x11).all()) for t in first)


# ---------------------------------------------------------------- attention

class Requests:
    """Requests over chunks in an 8-bit pool, and the oracle's copy of it, through link, decode and compile plans."""

    def __init__(self, hq, hkv, d, picks, lens, suffix, k, seed=0, rerotate=False, split=0, tile_rows=0, spare=40,
                 scale=0.0, garbage=True):
        el = _el()
        self.rng = np.random.default_rng([hq, hkv, d, seed, len(picks)])
        self.heads, self.cfg = (hq, hkv, d), el.attn_cfg(hq, hkv, d, scale, split, tile_rows, THETA)
        nb = [-(-n // 16) for n in lens]
        private = sum(sum(nb[c] if rerotate or k < 0 else min(nb[c], -(-k // 16)) for c in r) + -(-s // 16)
                      for r, s in zip(picks, suffix))
        self.blocks = sum(nb) + private + spare
        perm = self.rng.permutation(self.blocks)
        first = np.cumsum([0] + nb)
        self.ids = [[int(b) for b in perm[first[c]:first[c + 1]]] for c in range(len(lens))]
        self.free = [int(b) for b in perm[first[-1]:]]
        self.c = _cache(self.rng, self.blocks, hkv, d)
        if garbage:                                      # slots past a chunk's end, and free blocks, hold any bits
            for c, n in enumerate(lens):
                for s in range(n % 16, 16 if n % 16 else 0):
                    self._spoil(self.ids[c][-1], s)
            for b in self.free:
                for s in range(16):
                    self._spoil(b, s)
        reqs = [el.Request([lens[c] for c in r], [self.ids[c] for c in r], s, k, rerotate) for r, s in zip(picks, suffix)]
        self.rerotate = rerotate
        self._took(*el.epic_plan_link(reqs, self.cfg, self.free, self.blocks))
        self.cache = _upload(self.c)

    def _spoil(self, b, s):
        for name in ("k", "v", "ks", "vs"):
            x = self.c[name][b, :, s]
            x[...] = self.rng.choice(np.array([0x7F, 0xFF, 0x7E, 3], np.uint8), x.shape)

    def _took(self, sizes, host, views):
        self.sizes, self.host, self.views = sizes, host, views
        used = set(views["linked_blocks"].tolist()) | set(views["priv_block"].tolist())
        self.free = [b for b in self.free if b not in used]

    def decode(self, new):
        self._took(*_el().epic_plan_decode(self.sizes, self.host, new, self.cfg, self.free, self.blocks))
        return self

    def draw(self, spoil=()):
        """Rows of S: (q, k, v) tensors and values; rows in `spoil` get a value that is not finite in K, V or both."""
        hq, hkv, d = self.heads
        n = self.sizes.n_s
        q, k, v = (_rows(self.rng, n, h, d) for h in (hq, hkv, hkv))
        for i, r in enumerate(spoil):
            for y in ((k,), (v,), (k, v))[i % 3]:
                y[r, self.rng.integers(hkv), self.rng.integers(d)] = self.rng.choice([np.nan, np.inf, -np.inf])
        return [_bf16(x) for x in (q, k, v)]

    def run(self, rows=None, lse=True, stream=None, what=""):
        """The call, checked: the whole cache, and what the rows of S attend to."""
        el = _el()
        hq, hkv, d = self.heads
        n = self.sizes.n_s
        _say(what, f"heads {hq}/{hkv}/{d} rows {n} blocks {self.sizes.n_linked_blocks} tile rows {self.sizes.tile_rows} "
             f"partials {self.sizes.n_partials} private {self.sizes.n_private}")
        rows = rows or self.draw()
        (qt, q), (kt, k), (vt, v) = rows
        out = torch.full((n, hq, d), 7.0, dtype=torch.bfloat16, device="cuda")
        lt = torch.full((n, hq), 7.0, device="cuda") if lse else None
        ws = torch.full((max(256, el.epic_link_kv8_workspace_bytes(self.cfg, self.sizes)) + 4096,), 0xA5, dtype=torch.uint8,
                        device="cuda")
        guard = ws[-4096:]
        el.epic_link_attention_kv8(self.cfg, el.DevicePlan(self.sizes, self.host), qt, kt, vt, self.cache, out, lt,
                                   ws[:-4096], stream)
        torch.cuda.synchronize()
        assert bool((guard == 0xA5).all()), "written behind the workspace"
        got = _download(self.cache)
        want = kv8.copy(self.c)
        kv8.write(want, self.views, k, v, THETA)
        if self.rerotate and (self.views["priv_rot"] != 0).any():
            self._near(got, want)
            want = got                                   # attention is checked over what the cache holds
        else:
            _equal(got, want, what)
        self.c = want
        self.check(q, out, lt)
        return out, lt

    def _near(self, got, want):
        """Re-rotated keys: scales and codes next to each other, nearly all equal; everything else equal.  (Slots past a
        block's tokens held NaN codes beside any scale, which is no row of a cache: what turning leaves there is not
        compared.)"""
        dst = self.views["priv_block"][(self.views["priv_rot"] != 0) & (self.views["priv_src"] >= 0)]
        _equal({x: got[x] for x in ("v", "vs")}, {x: want[x] for x in ("v", "vs")})
        other = np.setdiff1d(np.arange(self.blocks), dst)
        _equal({x: got[x][other] for x in ("k", "ks")}, {x: want[x][other] for x in ("k", "ks")})
        length = dict(zip(self.views["linked_blocks"].tolist(), self.views["block_len"].tolist()))
        held = np.arange(16) < np.array([length[b] for b in dst.tolist()])[:, None]                      # [blocks, 16]
        g, w = ({x: c[x][dst].swapaxes(1, 2)[held] for x in ("k", "ks")} for c in (got, want))
        same = g["ks"] == w["ks"]
        assert np.abs(g["ks"].astype(int) - w["ks"]).max() <= 1 and same.mean() > 0.999
        a, b = (np.where(x["k"] & 0x80, -1, 1) * (x["k"] & 0x7F).astype(int) for x in (g, w))
        step = np.abs(a - b)[same]
        assert step.max() <= 1 and (step > 0).mean() < 1e-3, (step.max(), (step > 0).mean())

    every = 1                                            # requests are checked by this stride

    def check(self, q, out, lse):
        hq, hkv, d = self.heads
        out = out.double().cpu().numpy()
        lse = None if lse is None else lse.double().cpu().numpy()
        scale = self.cfg.softmax_scale or 1.0 / np.sqrt(d)
        for r in range(0, self.sizes.batch, self.every):
            a, b = int(self.views["s_off"][r]), int(self.views["s_off"][r + 1])
            if a == b:
                continue
            K, V = kv8.linked(self.c, self.views, r)
            pos = self.views["s_pos"][a:b]
            ref, l, bad = kv8.attention(q[a:b], K, V, pos, scale)
            fine = ~bad
            assert np.isnan(out[a:b][bad]).all(), "a row that attends to a NaN token"
            size = masked_attention(q[a:b], np.nan_to_num(K), np.abs(np.nan_to_num(V)), pos, scale)[0]
            n = (pos + 1)[:, None]
            far = np.abs(np.nan_to_num(K)).max(-1) * 0 + np.linalg.norm(np.nan_to_num(K), axis=-1)      # [N, Hkv]
            most = np.maximum.accumulate(far, 0)[pos]                                                      # [rows, Hkv]
            e = (d + 8) * 2.0 ** -24 * scale * np.linalg.norm(q[a:b], axis=-1) * np.repeat(most, hq // hkv, 1)
            weights = 2 * e + 2.0 ** -22 + 2 * n * 2.0 ** -24
            bar = (size * (2.0 ** -8 + 2 * weights[..., None])) * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(ref) + 2.0 ** -126
            err = np.abs(out[a:b] - ref)
            assert np.isfinite(out[a:b][fine]).all(), f"request {r}: not finite"
            worst = (err / bar)[fine].max() if fine.any() else 0.0
            assert worst <= 1.0, f"request {r}: {worst:.2f} bars"
            if lse is not None and fine.any():
                lbar = e + 2.0 ** -22 + n * 2.0 ** -24 + 2.0 ** -22 * np.abs(l)
                assert (np.abs(lse[a:b] - l) / lbar)[fine].max() <= 1.0, f"request {r}: lse"


HEADS = [(8, 8, 64), (32, 8, 128), (16, 1, 64), (16, 1, 128), (6, 3, 64), (4, 4, 128), (20, 5, 128), (64, 8, 64)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("rerotate", [False, True])
def test_link_then_decode(hq, hkv, d, rerotate):
    """A link step, then decode steps that fill a block, open blocks, skip a request, bring several tokens."""
    r = Requests(hq, hkv, d, [[0, 1, 2], [2, 0], [1]], [100, 37, 160], [5, 16, 1], 7, rerotate=rerotate)
    r.run(what="link")
    few = max(1, 16 // (hq // hkv))
    r.rerotate = False
    for new in ([1, 1, 1], [0, 3, 1], [min(few, 11), 1, 0], [1, 18, 2], [1, 0, 1]):
        r.decode(new).run(what=f"decode {new}")


@pytest.mark.parametrize("hq,hkv,d", [(32, 1, 64), (128, 1, 128), (16, 16, 64), (9, 9, 128)])
def test_other_head_counts(hq, hkv, d):
    """Groups too large for 16-row tiles, whose decode has wide ones; more KV heads than the wavefronts of a workgroup."""
    r = Requests(hq, hkv, d, [[0, 1], [1]], [100, 37], [5, 1], 7)
    r.run(what="link")
    for new in ([1, 1], [0, 13], [1, 0]):
        r.decode(new).run(what=f"decode {new}")


@pytest.mark.parametrize("d", [64, 128])
def test_turned_blocks_without_rows(d):
    """No row of S, but private blocks of turned keys: they are written, and nothing else is."""
    r = Requests(8, 2, d, [[0, 1], [1, 0, 0]], [100, 37], [0, 0], 0, rerotate=True)
    assert r.sizes.n_s == 0 and r.sizes.n_private > 0
    r.run(what="turned blocks alone")
    r.rerotate = False
    r.decode([1, 2]).run(what="decode")


@pytest.mark.parametrize("tile_rows", [16, 128, 256])
@pytest.mark.parametrize("split", [0, 1, 3, 8])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (32, 8, 128)])
def test_tiles_and_splits(hq, hkv, d, split, tile_rows):
    """Every tile size, whole and cut into items of few blocks, of odd numbers of blocks among them."""
    r = Requests(hq, hkv, d, [[0, 1], [1, 0]], [333, 47], [21, 3], 4, tile_rows=tile_rows, split=split)
    assert r.sizes.tile_rows == tile_rows
    if split:
        assert r.sizes.n_partials > 0
    r.run(what="link")
    r.decode([2, 1]).run(what="decode")


@pytest.mark.parametrize("k", [0, 1, 16, 17, -1])
@pytest.mark.parametrize("suffix", [0, 1, 16, 33])
def test_selections(k, suffix):
    """No rows at all (k = 0 without a suffix), the suffix alone, part of chunks, whole blocks, everything."""
    r = Requests(8, 2, 128, [[0, 1, 2], [1]], [31, 64, 1], [suffix, suffix], k)
    r.run(what=f"k {k} suffix {suffix}")


@pytest.mark.parametrize("length", [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 511, 513, 1025, 2047])
@pytest.mark.parametrize("d", [64, 128])
def test_decode_lengths(length, d):
    """One request of a chunk of that many tokens: a single block to many pairs per wavefront."""
    r = Requests(8, 2, d, [[0]], [length], [0], 0, seed=length)
    assert r.sizes.n_s == 0
    r.decode([1]).run(what=f"length {length}")
    r.decode([1]).run(what=f"length {length} + 1")


@pytest.mark.parametrize("k", [17, -1])
def test_decode_into_a_chunks_last_block(k):
    """Without a suffix the first new token goes to the copy of a chunk's last block."""
    r = Requests(8, 2, 64, [[0, 1], [1, 0]], [40, 20], [0, 0], k)
    r.run(what=f"k {k}")
    for new in ([1, 2], [0, 1], [20, 1]):
        r.decode(new).run(what=f"decode {new}")


@pytest.mark.parametrize("rerotate", [False, True])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 64), (16, 2, 128)])
def test_many_private_blocks_in_small_tiles(hq, hkv, d, rerotate):
    """More private blocks than the attention launch writes itself, and turned ones, in 16-row tiles."""
    n = 37
    r = Requests(hq, hkv, d, [[i % 3, (i + 1) % 3] for i in range(n)], [50, 33, 70], [1 + i % 19 for i in range(n)], 5,
                 rerotate=rerotate, tile_rows=16, spare=2 * n)
    assert r.sizes.n_private > 64
    r.run(what="link")
    r.rerotate = False
    r.decode([1] * n).run(what="decode")


def test_many_requests_decode():
    """70 requests: more private blocks than one wavefront looks through; then 64 of them."""
    n = 70
    r = Requests(8, 2, 64, [[i % 4] for i in range(n)], [20, 33, 17, 64], [1 + i % 17 for i in range(n)], 0, spare=3 * n)
    r.run(what="link")
    for new in ([1] * n, [1] * 64 + [0] * 6, [0] * 69 + [1]):
        r.decode(new)
        print(f"[gpu-test] private {r.sizes.n_private}", flush=True)
        r.run(what="decode")


@pytest.mark.parametrize("tile_rows", [128, 256])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (16, 8, 64)])
def test_wide_tiles_over_shared_chunks(hq, hkv, d, tile_rows):
    """Requests that link more blocks than the pool has: the pool is widened, not the list; the private blocks with
    it, or before it."""
    n = 9
    r = Requests(hq, hkv, d, [[0, 1, 2], [2, 1, 0], [1, 2, 0]] * 3, [200, 133, 170], [3] * n, 2, tile_rows=tile_rows, spare=4)
    assert r.sizes.n_linked_blocks > r.blocks
    spoil = [4, int(r.views["s_off"][2]) + 1]
    r.run(r.draw(spoil), what="shared")


def test_requests_without_chunks():
    r = Requests(8, 2, 64, [[], [0], []], [40], [3, 2, 20], 4)
    r.run(what="no chunks")
    r.decode([1, 1, 1]).run(what="decode")


@pytest.mark.parametrize("hq,hkv,d", [(8, 8, 64), (32, 8, 128), (64, 8, 64)])
def test_decode_over_shared_chunks(hq, hkv, d):
    """Requests enough that their work items carry rows of several requests and lists of blocks.  The link step is not
    run: its private blocks hold what they hold."""
    some = [[0, 1, 2], [1, 0, 2], [2, 2, 3], [0, 3], [3, 1, 0], [1, 4], [0, 1, 4], [4, 0, 3]]
    n = 40
    r = Requests(hq, hkv, d, [some[i % 8] for i in range(n)], [1533, 1800, 47, 1200, 1000],
                 [5 + 3 * i % 41 for i in range(n)], 16, spare=60, garbage=False)
    r.decode([1 + i % 2 if hq // hkv < 8 else 1 for i in range(n)])      # two rows of eight heads each fill a tile
    work = r.views["work"].reshape(-1, 8)
    assert {1, 2} <= set(work[work[:, 0] >= 0, 7].tolist()), "item kinds of the plan"
    r.every = 5                                          # every kind of request
    out, lse = r.run(what="shared")
    assert bool(torch.isfinite(out).all()) and bool(torch.isfinite(lse).all())


def _workgroups(r, waves):
    """Workgroups of a launch of 16-row tiles at `waves` wavefronts: up to 256 take eight, more four."""
    hkv = r.heads[1]
    return r.sizes.n_work * hkv + r.sizes.n_private * -(-hkv // waves)


def _item_blocks(r):
    work = r.views["work"].reshape(-1, 8)
    work = work[work[:, 0] >= 0]
    return work[:, 2] - work[:, 1]


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (16, 8, 64)])
@pytest.mark.parametrize("split", [4, 20])
def test_decode_of_one_long_request(hq, hkv, d, split):
    """A single tile in more workgroups than CUs: its blocks are read past the caches, by four wavefronts each."""
    r = Requests(hq, hkv, d, [[0, 1]], [16 * 18 * split - 5, 16 * 17 * split + 3], [0], 0, split=split)
    for new in ([1], [1 if hq // hkv > 2 else 3], [1]):
        r.decode(new)
        assert r.sizes.tile_rows == 16 and r.sizes.n_tiles == 1 and _workgroups(r, 8) > 256 and r.sizes.n_private <= 64
        r.run(what=f"one request, items of {split} blocks")


@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 64), (8, 8, 128)])
@pytest.mark.parametrize("length", [16 * 257, 16 * 300 - 7])
def test_long_items_of_four_wavefronts(hq, hkv, d, length):
    """Items of more blocks than four wavefronts take the ids of at once; the last blocks, a private one among them, are
    of the second lot, and their number is odd."""
    n = 40
    r = Requests(hq, hkv, d, [[i % 2] for i in range(n)], [length, length + 32], [5 + i % 12 for i in range(n)], 0, split=4096,
                 spare=2 * n, garbage=False)
    for new in ([1] * n, [1 + i % 2 for i in range(n)]):
        r.decode(new)
        assert r.sizes.tile_rows == 16 and _workgroups(r, 8) > 256 and 0 < r.sizes.n_private <= 64
        blocks = _item_blocks(r)
        assert blocks.min() > 256 and (blocks % 2 == 1).any()
        r.every = 13
        r.run(what="long items")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [16 * 513 - 3, 16 * 530])
def test_long_items_of_eight_wavefronts(d, length):
    r = Requests(4, 1, d, [[0]], [length], [7], 0, split=4096)
    for new in ([1], [4], [3]):
        r.decode(new)
        assert r.sizes.tile_rows == 16 and _workgroups(r, 8) <= 256 and _item_blocks(r).min() > 512
        r.run(what="long item")


@pytest.mark.parametrize("hq,hkv,d", [(16, 8, 64), (16, 8, 128)])
def test_copied_blocks_in_many_small_tiles(hq, hkv, d):
    """Private blocks that keep tokens of a shared block, written by the attention launch of more workgroups than CUs."""
    n = 10
    r = Requests(hq, hkv, d, [[i % 3, (i + 1) % 3] for i in range(n)], [90, 57, 131], [9 + i % 3 for i in range(n)], 20,
                 tile_rows=16)
    src = r.views["priv_src"]
    assert _workgroups(r, 8) > 256 and r.sizes.n_private <= 64 and ((src >= 0) & (src != r.views["priv_block"])).any()
    r.run(what="copied blocks")


@pytest.mark.parametrize("hq,hkv,d", [(16, 4, 64), (32, 4, 128), (16, 1, 128)])
def test_decode_of_many_tokens_in_small_tiles(hq, hkv, d):
    """Several 16-row tiles of a request, each over the blocks that the others' rows go to: the last block's free slots, whole
    new blocks and part of another."""
    r = Requests(hq, hkv, d, [[0, 1], [1]], [350, 219], [7, 16], 5, tile_rows=16, spare=60)
    r.run(what="link")
    for new in ([21, 5], [33, 0], [1, 48]):
        r.decode(new)
        assert r.sizes.tile_rows == 16 and r.sizes.n_tiles >= sum(n * (hq // hkv) // 16 for n in new)
        r.run(what=f"decode {new}")


@pytest.mark.parametrize("tile_rows", [16, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_in_a_chunk(d, tile_rows):
    """A cached token that is NaN, of one KV head, with a thousand tokens before it and behind it: rows before it and rows of
    requests that do not link its chunk stay finite, rows behind it are NaN in that head's."""
    r = Requests(8, 4, d, [[0, 1], [1, 0], [0]], [1400, 2300], [20, 9, 3], 6, tile_rows=tile_rows)
    b, s = r.ids[1][1111 // 16], 1111 % 16               # token 1111 of chunk 1
    r.c["k"][b, 2, s], r.c["v"][b, 2, s], r.c["ks"][b, 2, s], r.c["vs"][b, 2, s] = 0x7F, 0, 255, 255
    r.cache = _upload(r.c)
    out, _ = r.run(what="NaN in a chunk")
    bad = torch.isnan(out).any(-1).cpu().numpy()
    off = r.views["s_off"]
    want = np.zeros_like(bad)
    for req, at in ((0, 1400 + 1111), (1, 1111)):
        rows = slice(int(off[req]), int(off[req + 1]))
        want[rows, 4:6] = (r.views["s_pos"][rows] >= at)[:, None]
    assert np.array_equal(bad, want) and want.any() and not want[:, 4].all()


@pytest.mark.parametrize("amplitude", [1.0, 1.25])
def test_turned_keys_after_the_rotation(amplitude):
    """Keys of epic_qk_norm_rope in the form that re-rotating plans turn (the whole head, half pairs, the plan's base, no
    scaled frequencies): compiled into 8-bit blocks at their chunks' positions, then linked with rerotate, they are the normed
    keys turned at their linked positions.  Bars, with p = |(a, b)| of a value's pair, which no turn changes, and m the row's
    largest |y| before the first turn: a turned row's largest is at most sqrt(2) m (1.1 of that after its rounding), its scale 2^t
    at most 1 / 224 of it =: s.  Rounding to bf16 and to 8 bits leaves 2^-8 and 2^-4 of a value or half the smallest step, 2^-10
    2^t; two such errors of a pair come out of a turn as at most e = (2^-8 + 2^-4) p + sqrt(2) 2^-10 s.  The second rounding
    to 8 bits adds 2^-4 (|y| + e) + 2^-10 s; fp32 stays under 2^-12 p in all."""
    el = _el()
    hq, hkv, d = 8, 2, 128
    lens, dev = [75, 130, 48], "cuda"
    r = Requests(hq, hkv, d, [[0, 1, 2]], lens, [11], 4, rerotate=True, spare=60, garbage=False)
    link = (r.sizes, r.host, r.views)
    sizes, host, views = el.epic_plan_compile(lens, r.ids, 0, r.cfg, r.free, r.blocks)
    n, rope = sizes.n_s, el.rope_cfg(d, THETA, amplitude=amplitude)
    x = torch.from_numpy(_rows(r.rng, n, (hq + 2 * hkv) * d)).float().to(dev)
    w = torch.from_numpy(1 + 0.2 * r.rng.normal(size=d)).to(torch.bfloat16).to(dev)
    q, k, v = (torch.empty((n, h, d), dtype=torch.bfloat16, device=dev) for h in (hq, hkv, hkv))
    el.epic_qk_norm_rope(r.cfg, rope, x, torch.from_numpy(views["s_pos"].copy()).to(dev),
                         torch.from_numpy(el.epic_rope_freqs(rope)).to(dev), q, k, v, q_norm=w, k_norm=w)
    ws = torch.empty(max(256, el.epic_link_kv8_workspace_bytes(r.cfg, sizes)), dtype=torch.uint8, device=dev)
    el.epic_link_attention_kv8(r.cfg, el.DevicePlan(sizes, host), q, k, v, r.cache, torch.empty_like(q), None, ws)
    torch.cuda.synchronize()
    r.c = _download(r.cache)
    r.sizes, r.host, r.views = link
    r.run(what="link of turned keys")
    y = x.double().cpu().numpy().reshape(n, -1, d)[:, hq:hq + hkv]
    y = amplitude * y / np.sqrt((y * y).mean(-1, keepdims=True) + 1e-6) * w.double().cpu().numpy()
    K, _ = kv8.linked(r.c, r.views, 0)
    first = np.cumsum([0] + lens)
    rows = set(r.views["s_pos"].tolist())                # of S, not cached
    for c in range(3):
        pos = np.array([p for p in range(first[c], first[c + 1]) if p not in rows])
        part = y[pos]
        want = rope_at(part, pos, THETA)
        pair = np.hypot(part, np.roll(part, d // 2, -1))  # |(a, b)| of each dim's pair
        top = np.abs(part).max(-1, keepdims=True)
        step = 2.0 ** -10 * np.sqrt(2) * 1.1 * top / 224
        e = (2.0 ** -8 + 2.0 ** -4) * pair + np.sqrt(2) * step
        bar = e + 2.0 ** -4 * (np.abs(want) + e) + step + 2.0 ** -12 * pair
        err = np.abs(K[pos] - want)
        assert (err <= bar).all(), f"chunk {c}: {np.max(err / bar):.2f} bars"


@pytest.mark.parametrize("tile_rows", [16, 128, 256])
@pytest.mark.parametrize("d", [64, 128])
def test_nan_where_it_is_masked(d, tile_rows):
    """Rows of S that are not finite, in K, in V, in both: rows before them stay finite, rows from them on are NaN, in
    their heads; and what is stored of them is NaN in both."""
    r = Requests(8, 4, d, [[0, 1], [1]], [40, 90], [37, 20], 6, tile_rows=tile_rows)
    n = r.sizes.n_s
    off = [int(x) for x in r.views["s_off"]]
    spoil = [off[1] - 20, off[1] - 11, off[1] - 1, off[1] + 9, n - 3]
    rows = r.draw(spoil)
    out, _ = r.run(rows, what="NaN rows")
    assert 0 < int(torch.isnan(out).any(-1).sum()) < out.shape[0] * 8
    k, v = (torch.empty((r.blocks, 4, *s), dtype=torch.bfloat16, device="cuda") for s in ((16, d), (d, 16)))
    _el().epic_kv8_unpack(r.cache, k, v)
    slot = int(r.views["s_slot"][spoil[1]])              # NaN in V alone
    assert torch.equal(torch.isnan(k[slot // 16, :, slot % 16]).any(-1), torch.isnan(v[slot // 16, :, :, slot % 16]).any(-1))
    assert int(torch.isnan(k[slot // 16, :, slot % 16]).all(-1).sum()) == 1


def test_infinite_queries_stay_in_their_rows():
    r = Requests(8, 2, 128, [[0]], [200], [30], 0, tile_rows=16)
    rows = r.draw()
    q = rows[0][0].clone()
    q[3, 1, 5], q[7, 0, 0] = float("inf"), float("nan")
    ref, ref_lse = r.run(rows, what="finite")
    el = _el()
    out, lse = torch.empty_like(ref), torch.empty_like(ref_lse)
    ws = torch.empty(max(256, el.epic_link_kv8_workspace_bytes(r.cfg, r.sizes)), dtype=torch.uint8, device="cuda")
    el.epic_link_attention_kv8(r.cfg, el.DevicePlan(r.sizes, r.host), q, rows[1][0], rows[2][0], r.cache, out, lse, ws)
    bad = torch.zeros(out.shape[:2], dtype=torch.bool, device="cuda")
    bad[3, 1] = bad[7, 0] = True
    assert torch.equal(out[~bad], ref[~bad]) and torch.equal(lse[~bad], ref_lse[~bad])
    assert bool(torch.isnan(out[bad]).all())


@pytest.mark.parametrize("tile_rows", [16, 128])
def test_scales_of_any_size(tile_rows):
    """Keys and values whose scales lie far apart, down to the smallest."""
    r = Requests(4, 2, 64, [[0]], [70], [20], 0, tile_rows=tile_rows, garbage=False)
    hq, hkv, d = r.heads
    (qt, q), (kt, k), (vt, v) = r.draw()
    size = np.exp(r.rng.uniform(-60, 3, (r.sizes.n_s, hkv, 1)))
    kt, k = _bf16(k * size)
    vt, v = _bf16(v * np.exp(r.rng.uniform(-8, 8, size.shape)))
    r.run([(qt, q), (kt, k), (vt, v)], what="far scales")
    # one token: its V comes back as it is, whatever its scale
    one = Requests(4, 2, 64, [[]], [], [1], 0, tile_rows=tile_rows, garbage=False)
    for e in (-110, -40, 0, 60, 119):
        (qt, q), (kt, k), (vt, v) = one.draw()
        vt, v = _bf16(v * 2.0 ** e)
        out, _ = one.run([(qt, q), (kt, k), (vt, v)], what=f"one token 2^{e}")
        held = kv8.linked(one.c, one.views, 0)[1][0]
        assert np.array_equal(out.double().cpu().numpy()[0].reshape(2, 2, 64)[:, 0], held)


def test_softmax_scale_and_no_lse():
    r = Requests(8, 2, 64, [[0]], [300], [3], 0, scale=0.3)
    r.run(lse=False, what="scale 0.3")
    r.decode([1]).run(lse=False, what="decode")


def test_compile_plans():
    """Chunks compiled into 8-bit blocks, after dummy tokens and without; then linked."""
    el = _el()
    hq, hkv, d = 8, 2, 64
    for dummy in (0, 4):
        r = Requests(hq, hkv, d, [[0, 1, 2]], [50, 16, 131], [9], 4, spare=60)
        link = (r.sizes, r.host, r.views)
        r._took(*el.epic_plan_compile([50, 16, 131], r.ids, dummy, r.cfg, r.free, r.blocks))
        r.run(what=f"compile, {dummy} dummies")
        r.sizes, r.host, r.views = link
        r.run(what="link after it")


def test_far_blocks():
    """Ids whose values lie past 2^32 bytes of the pool."""
    el = _el()
    hq, hkv, d = 8, 8, 128
    blocks = 300000                                      # 4.9 GB of K, as much of V
    if torch.cuda.mem_get_info()[0] < 20 << 30:
        pytest.skip("not enough memory")
    r = Requests(hq, hkv, d, [[0, 1]], [100, 60], [5], 3, spare=20)
    near = r.cache
    far = el.Kv8Cache(*(torch.empty(s, dtype=torch.uint8, device="cuda") for s in el.kv8_shapes(blocks, hkv, d)))
    move = blocks - r.blocks
    for a, b in ((far.k, near.k), (far.v, near.v), (far.scale, near.scale)):
        b_ = b.clone()
        a[move:] = b_
    lens, ids = [100, 60], [[b + move for b in x] for x in r.ids]
    free = [b + move for b in list(r.views["priv_block"]) + r.free]
    sizes, host, _ = el.epic_plan_link([el.Request(lens, ids, 5, 3)], r.cfg, free, blocks)
    rows = r.draw()
    out, lse = r.run(rows, what="near")
    for tile_rows in (0, 16):
        cfg = el.attn_cfg(hq, hkv, d, tile_rows=tile_rows)
        sizes, host, views = el.epic_plan_link([el.Request(lens, ids, 5, 3)], cfg, free, blocks)
        o, l = torch.empty_like(out), torch.empty_like(lse)
        ws = torch.empty(max(256, el.epic_link_kv8_workspace_bytes(cfg, sizes)), dtype=torch.uint8, device="cuda")
        el.epic_link_attention_kv8(cfg, el.DevicePlan(sizes, host), *(x[0] for x in rows), far, o, l, ws)
        torch.cuda.synchronize()
        r.check(rows[0][1], o, l)
        assert torch.equal(far.k[move:], near.k) and torch.equal(far.v[move:], near.v) and torch.equal(far.scale[move:], near.scale)
    i = torch.arange(move, blocks, dtype=torch.int32, device="cuda")
    k, v = (torch.empty((r.blocks, hkv, *s), dtype=torch.bfloat16, device="cuda") for s in ((16, d), (d, 16)))
    el.epic_kv8_unpack(far, k, v, src_blocks=i)
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    el.epic_kv8_unpack(near, k2, v2)
    assert torch.equal(k.view(torch.int16), k2.view(torch.int16)) and torch.equal(v.view(torch.int16), v2.view(torch.int16))


# ---------------------------------------------------------------- streams, graphs, runs of several operators

def _call(r, rows, out, lse, ws, plan, stream=None):
    _el().epic_link_attention_kv8(r.cfg, plan, rows[0][0], rows[1][0], rows[2][0], r.cache, out, lse, ws, stream)


@pytest.mark.parametrize("kind", ["decode", "wide"])
def test_graphs_and_streams(kind):
    """Captured calls replayed between eager ones; two graphs and two streams with a workspace each."""
    el = _el()
    runs = []
    for i in range(2):
        r = Requests(32, 8, 128, [[0, 1], [0]], [700, 900], [20, 3], 16, seed=i, split=16)
        r.run(what="link")
        if kind == "decode":
            r.decode([1, 2])
        rows = r.draw()
        ref = r.run(rows, what=kind)
        out, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
        ws = torch.empty(el.epic_link_kv8_workspace_bytes(r.cfg, r.sizes), dtype=torch.uint8, device="cuda")
        plan = el.DevicePlan(r.sizes, r.host)
        stream = torch.cuda.Stream()
        assert r.sizes.n_partials > 0
        torch.cuda.synchronize()
        _call(r, rows, out, lse, ws, plan, stream)
        stream.synchronize()
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            _call(r, rows, out, lse, ws, plan)
        runs.append((r, rows, ref, out, lse, ws, plan, g, stream))
    for i in range(3):
        for _, _, _, out, lse, *_ in runs:
            out.zero_()
            lse.zero_()
        torch.cuda.synchronize()
        for *_, g, stream in runs:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for r, rows, ref, out, lse, ws, plan, *_ in runs:
            assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1]), f"replay {i}"
            _call(r, rows, out, lse, ws, plan)           # eager work between the replays
        torch.cuda.synchronize()
        for _, _, ref, out, lse, *_ in runs:
            assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


def test_same_results_every_time():
    r = Requests(32, 8, 128, [[0, 1, 2]], [2000, 1500, 900], [40], 16)
    r.run(what="link")
    r.decode([1])
    rows = r.draw()
    ref = r.run(rows, what="decode")
    el = _el()
    ws = torch.empty(max(256, el.epic_link_kv8_workspace_bytes(r.cfg, r.sizes)), dtype=torch.uint8, device="cuda")
    for _ in range(10):
        out, lse = torch.empty_like(ref[0]), torch.empty_like(ref[1])
        _call(r, rows, out, lse, ws, el.DevicePlan(r.sizes, r.host))
        assert torch.equal(out, ref[0]) and torch.equal(lse, ref[1])


def test_a_layers_attention_from_its_projections():
    """As a model uses them: Q|K|V rows of the 8-bit product are normed and turned, chunks that were compiled in
    bf16 move to the 8-bit pool, a link step and a decode step attend over it, and a block is read back."""
    el = _el()
    hq, hkv, d, hidden = 8, 2, 128, 512
    rng = np.random.default_rng(5)
    lens, suffix, k = [75, 130], 11, 8
    nb = [-(-n // 16) for n in lens]
    blocks = sum(nb) + 20
    bk, _ = _bf16(_rows(rng, blocks, hkv, 16, d))
    bv, _ = _bf16(_rows(rng, blocks, hkv, d, 16))
    cache = el.Kv8Cache.zeros(blocks, hkv, d)
    chunk = torch.arange(sum(nb), dtype=torch.int32, device="cuda")
    el.epic_kv8_pack(bk, bv, cache, src_blocks=chunk, dst_blocks=chunk)
    ids = [list(range(nb[0])), list(range(nb[0], sum(nb)))]
    cfg, rope = el.attn_cfg(hq, hkv, d, rope_theta=THETA), el.rope_cfg(64, THETA, factor=4.0)
    freqs = torch.from_numpy(el.epic_rope_freqs(rope)).cuda()
    n_qkv = (hq + 2 * hkv) * d
    w, ws = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in ((n_qkv, hidden), el.fp8_block_scale_shape(n_qkv, hidden)))
    el.epic_quant_fp8((torch.randn(n_qkv, hidden, device="cuda") / hidden ** 0.5).to(torch.bfloat16), w, ws, block_rows=128)
    qn, kn = ((1 + 0.1 * torch.randn(d, device="cuda")).to(torch.bfloat16) for _ in range(2))
    scratch = torch.empty(el.epic_gemm_fp8_workspace_bytes(), dtype=torch.uint8, device="cuda")
    norm = torch.ones(hidden, dtype=torch.bfloat16, device="cuda")
    free = list(range(sum(nb), blocks))
    sizes, host, views = el.epic_plan_link([el.Request(lens, ids, suffix, k)], cfg, free, blocks)
    c = _download(cache)
    for step in ("link", "decode"):
        if step == "decode":
            taken = sizes.n_private
            sizes, host, views = el.epic_plan_decode(sizes, host, [1], cfg, free[taken:], blocks)
        n = sizes.n_s
        plan = el.DevicePlan(sizes, host)
        a, sa = (torch.empty(s, dtype=torch.uint8, device="cuda") for s in ((n, hidden), el.fp8_row_scale_shape(n, hidden)))
        el.epic_rmsnorm_fp8(torch.randn(n, hidden, device="cuda"), norm, 1e-5, a, sa)
        qkv = torch.empty((n, n_qkv), dtype=torch.bfloat16, device="cuda")
        el.epic_gemm_fp8(el.FP8_BF16, a, sa, w, ws, qkv, workspace=scratch)
        q, kk, v = (torch.empty((n, h, d), dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        pos = torch.from_numpy(views["s_pos"].copy()).cuda()
        el.epic_qk_norm_rope(cfg, rope, qkv, pos, freqs, q, kk, v, q_norm=qn, k_norm=kn)
        out, lse = torch.empty_like(q), torch.empty((n, hq), device="cuda")
        room = torch.empty(max(256, el.epic_link_kv8_workspace_bytes(cfg, sizes)), dtype=torch.uint8, device="cuda")
        el.epic_link_attention_kv8(cfg, plan, q, kk, v, cache, out, lse, room)
        torch.cuda.synchronize()
        x = qkv.double().cpu().numpy().reshape(n, -1, d)
        y = x[:, :hq] / np.sqrt((x[:, :hq] ** 2).mean(-1, keepdims=True) + 1e-6) * qn.double().cpu().numpy()
        ang = views["s_pos"][:, None] * (THETA ** (-2.0 * np.arange(32) / 64) / 4.0)
        cs, sn = np.cos(ang)[:, None], np.sin(ang)[:, None]
        ref = np.concatenate([y[..., :32] * cs - y[..., 32:64] * sn, y[..., 32:64] * cs + y[..., :32] * sn, y[..., 64:]], -1)
        assert np.abs(q.double().cpu().numpy() - ref).max() <= 2.0 ** -8 * np.abs(ref).max()
        kv8.write(c, views, kk.double().cpu().numpy(), v.double().cpu().numpy())
        _equal(_download(cache), c, step)
        K, V = kv8.linked(c, views, 0)
        o, l, _ = kv8.attention(q.double().cpu().numpy(), K, V, views["s_pos"])
        assert np.abs(out.double().cpu().numpy() - o).max() <= 2.0 ** -6 * np.abs(V).max()
        assert np.abs(lse.double().cpu().numpy() - l).max() <= 1e-3
    el.epic_kv8_unpack(cache, bk, bv, src_blocks=chunk, dst_blocks=chunk)
    want = kv8.values(c["k"], c["ks"])[:sum(nb)]
    assert np.array_equal(bk[:sum(nb)].double().cpu().numpy(), want)


def test_attention_binding_refuses():
    el = _el()
    r = Requests(8, 2, 64, [[0]], [40], [3], 0)
    (q, _), (k, _), (v, _) = r.draw()
    out, lse = torch.empty_like(q), torch.empty((3, 8), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    plan = el.DevicePlan(r.sizes, r.host)
    good = [r.cfg, plan, q, k, v, r.cache, out, lse, ws]
    el.epic_link_attention_kv8(*good)
    for i, bad in ((2, q[:2]), (2, q.float()), (2, q.cpu()), (3, q), (4, v.transpose(1, 2).contiguous().transpose(1, 2)),
                   (5, el.Kv8Cache.zeros(4, 4, 64)), (5, el.Kv8Cache.zeros(4, 2, 64, device="cpu")), (6, out.float()),
                   (7, lse.half()), (8, ws.cpu()), (1, el.DevicePlan(r.sizes, r.host, device="cpu"))):
        with pytest.raises(ValueError):
            el.epic_link_attention_kv8(*good[:i], bad, *good[i + 1:])
    torch.cuda.synchronize()

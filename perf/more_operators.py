"""Operators of a cache in 8 bits as timed cases, with their plain forms.

Between the Q|K|V product and the attention's output, for a linked cache that is stored in
8 bits:

    rope    Q|K|V rows -> RMS norm of each query and key head -> rotation  epic_qk_norm_rope
    pack    blocks of a bf16 cache -> blocks of an 8-bit cache             epic_kv8_pack
    unpack  the way back                                                   epic_kv8_unpack
    attend  rows of S written in 8 bits, then attention over the linked    epic_link_attention_kv8
            8-bit cache (link and decode plans)

    own                 False: plain torch; True: the library's kernels
    listed()            the named cases
    draw(rng)           one more case of the same ranges
    prepare(case, seed) inputs and buffers in device memory
    run(state)          one pass; returns its outputs
    work(case)          bytes and operations the pass cannot do without
    exact(case, seed)   the same outputs from the definition in float64

The 8-bit cache has blocks of 16 tokens.  A row (the D values of K or of V of a token and KV
head) is e4m3 values and one power-of-two scale, a byte of e8m0 (2 ** (byte - 127), 255: the row
is NaN).  Values lie in the order in which the matrix cores take them:

    k      [blocks][Hkv][D / 64][4][16][16]    dim 64 j + 16 a + e of token s at [j][a][s][e]
    v      [blocks][Hkv][D / 64][4][16][4][4]  dim 64 j + 16 t + r of token 4 a + c at [j][a][r][t][c]
    scale  [blocks][Hkv][2][16]                of K, of V
"""
import math

import numpy as np
import torch

own = False

BLOCK = 16
TOP = 448.0                      # largest e4m3 value
EPS = 1e-6
THETA = 500000.0
# (query heads, KV heads, head dim)
HEADS = [(32, 8, 128), (32, 8, 128), (8, 8, 64), (16, 4, 64), (16, 8, 128), (32, 4, 128), (8, 1, 128), (16, 1, 64)]
# (factor, original context, turns below and above which a frequency is divided or kept, amplitude)
PLAIN, LINEAR, RAMP = (1.0, 0, 0.0, 0.0, 1.0), (4.0, 0, 0.0, 0.0, 1.0), (8.0, 8192, 1.0, 4.0, 1.0)
RAMP_LOUD = (32.0, 4096, 1.0, 32.0, 0.1 * math.log(32.0) + 1.0)
ROWS_COMPILE = 20560             # tokens of a compile step: 20 chunks of 1024 after 4 dummy tokens each
POOL_BLOCKS = 8192               # 64 chunks of 2048 tokens


def _rope(name, rows, heads, rot, dtype, interleaved=False, norm=True, scaling=PLAIN, far=0):
    factor, context, low, high, amplitude = scaling
    return {"name": name, "what": "rope", "rows": rows, "heads": heads[0], "kv_heads": heads[1], "dim": heads[2],
            "rot": rot, "dtype": dtype, "interleaved": interleaved, "norm": norm, "factor": factor, "context": context,
            "low": low, "high": high, "amplitude": amplitude, "far": far}


def _blocks_case(name, what, blocks, kv_heads, dim):
    return {"name": name, "what": what, "blocks": blocks, "kv_heads": kv_heads, "dim": dim}


def _attend_case(name, heads, requests, chunks, chunk_len, pool, suffix, k, mode="link", new=1, ragged=False,
                 rerotate=False):
    return {"name": name, "what": "attend", "mode": mode, "heads": heads[0], "kv_heads": heads[1], "dim": heads[2],
            "requests": requests, "chunks": chunks, "chunk_len": chunk_len, "pool": pool, "suffix": suffix, "k": k,
            "new": new, "ragged": ragged, "rerotate": rerotate}


def listed():
    return [
        # one request decoding: the Q|K|V row of a token, from the 8-bit product
        _rope("rope_decode1", 1, (32, 8, 128), 128, "bf16", far=131072),
        # a link step of 736 rows, from the fp32 product; half of each head rotated, pairs side by side
        _rope("rope_link736", 736, (32, 8, 128), 64, "fp32", interleaved=True, scaling=LINEAR, far=20000),
        # a compile step, frequencies scaled for a long context
        _rope("rope_compile", ROWS_COMPILE, (32, 8, 128), 128, "bf16", scaling=RAMP, far=131072),
        # one compiled chunk of 1000 tokens enters the 8-bit pool
        _blocks_case("pack_chunk", "pack", 63, 8, 128),
        # a pool of 64 chunks of 2048 tokens is converted
        _blocks_case("pack_pool", "pack", POOL_BLOCKS, 8, 128),
        # ten 512-token passages of a small model are read back
        _blocks_case("unpack_rag", "unpack", 320, 4, 64),
        # a whole pool is read back
        _blocks_case("unpack_pool", "unpack", POOL_BLOCKS, 8, 128),
        # a small multi-head model decoding after four short passages: launch latency
        _attend_case("attend_decode_small", (8, 8, 64), 1, 4, 128, 4, 16, 4, mode="decode"),
        # decode after a link: one token of one long request
        _attend_case("attend_decode_long", (32, 8, 128), 1, 64, 2048, 64, 250, 32, mode="decode"),
        # decode after a link: two tokens of each request of a serving batch whose documents are shared
        _attend_case("attend_decode_serving", (32, 8, 128), 32, 8, 2000, 64, 121, 32, mode="decode", new=2, ragged=True),
        # one retrieval request: ten 512-token passages and a question
        _attend_case("attend_link_rag", (32, 8, 128), 1, 10, 512, 10, 64, 16),
        # long context: 64 documents of 2048 tokens, the first 32 of each recomputed
        _attend_case("attend_link_long", (32, 8, 128), 1, 64, 2048, 64, 256, 32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["rope", "rope", "pack", "unpack", "attend", "attend", "attend"])
    hq, hkv, d = rng.choice(HEADS)
    if what == "rope":
        rows = _log(rng, 1, ROWS_COMPILE)
        case = _rope("", rows, (hq, hkv, d), 16 * rng.randint(1, d // 16), rng.choice(["bf16", "fp32"]),
                     rng.random() < 0.5, rng.random() < 0.8, rng.choice([PLAIN, LINEAR, RAMP, RAMP_LOUD]),
                     _log(rng, rows, 1 << 20))
        del case["name"]
        return case
    if what != "attend":
        return {"what": what, "blocks": _log(rng, 1, POOL_BLOCKS), "kv_heads": hkv, "dim": d}
    mode = rng.choice(["link", "decode", "decode"])
    case = _attend_case("", (hq, hkv, d), _log(rng, 1, 32), _log(rng, 1, 64), _log(rng, 17, 2048), 0, _log(rng, 1, 256),
                        rng.choice([0, 4, 16, 32, 32]), mode, rng.randint(1, 4) if mode == "decode" else 0,
                        rng.random() < 0.6, mode == "link" and rng.random() < 0.2)
    del case["name"]
    share = rng.randint(1, 4)
    while True:                                  # no more than the largest listed cases
        case["pool"] = case["chunks"] * min(share, case["requests"])
        g = _geometry(case)
        pool = g["n_chunk_blocks"] + g["n_private"]
        linked = sum(len(x["block"]) for x in g["requests"])
        if pool <= 16000 and linked <= 34000 and _attention_flops(case, g) <= 2.0e12:
            return case
        key = "requests" if case["requests"] > 1 else "chunks" if case["chunks"] > 1 else "chunk_len"
        case[key] = max(1, case[key] * 2 // 3)


# ---------------------------------------------------------------- linked sequences

def _blocks(n):
    return -(-n // BLOCK)


def _geometry(case):
    """A function of the case alone.  Physical blocks 0 .. n_chunk_blocks - 1 are the chunks', in order; the
    private ones follow, taken in order, request by request.  Per request the blocks of its linked sequence with
    their first position and tokens, the positions of its rows of S, and the private blocks it writes:
    (block, block copied into it first or -1, row of S of each slot or -1, offset that copied keys are moved by)."""
    rng = np.random.default_rng([case["pool"], case["chunk_len"], case["requests"], case["chunks"]])
    lens = np.full(case["pool"], case["chunk_len"])
    if case["ragged"]:
        lens = rng.integers((case["chunk_len"] + 1) // 2, case["chunk_len"] + 1, case["pool"])
    first = np.concatenate(([0], np.cumsum(_blocks(lens))))
    picks = [[int(c) for c in rng.permutation(case["pool"])[:case["chunks"]]] for _ in range(case["requests"])]
    free, row, out = int(first[-1]), 0, []
    for r in picks:
        block, pos0, count, rows, priv, off = [], [], [], [], [], 0
        for j, c in enumerate(r):
            n = int(lens[c])
            sel = 0 if j == 0 else min(case["k"], n)
            moved = case["rerotate"] and j > 0
            t = np.arange(0, n, BLOCK)
            ids = first[c] + t // BLOCK
            for i in range(_blocks(n) if moved else _blocks(sel)):
                slot = np.arange(16 * i, 16 * i + 16)
                fresh = np.where(slot < sel, row + slot, -1)
                keeps = sel < min(n, 16 * i + 16)                 # a cached token stays in this block
                priv.append((free, int(ids[i]) if keeps else -1, fresh, off if moved else 0))
                ids[i] = free
                free += 1
            block.append(ids)
            pos0.append(off + t)
            count.append(np.minimum(n - t, BLOCK))
            rows.append(off + np.arange(sel))
            row += sel
            off += n
        t = np.arange(0, case["suffix"], BLOCK)
        for i in range(len(t)):
            slot = np.arange(16 * i, 16 * i + 16)
            priv.append((free + i, -1, np.where(slot < case["suffix"], row + slot, -1), 0))
        block.append(free + t // BLOCK)
        pos0.append(off + t)
        count.append(np.minimum(case["suffix"] - t, BLOCK))
        rows.append(off + np.arange(case["suffix"]))
        free += len(t)
        row += case["suffix"]
        out.append({"pick": r, "block": np.concatenate(block), "pos0": np.concatenate(pos0),
                    "count": np.concatenate(count), "rows": np.concatenate(rows), "priv": priv})
    taken = free - int(first[-1])                # private blocks of the link plan
    if case["mode"] == "decode":                 # everything so far is in place; new tokens follow
        row = 0
        for x in out:
            end = int(x["pos0"][-1] + x["count"][-1])
            held, left, at, x["priv"] = int(x["count"][-1]), case["new"], row, []
            x["rows"] = end + np.arange(case["new"])
            row += case["new"]
            while left:
                if held in (0, BLOCK):
                    x["block"], x["pos0"] = np.append(x["block"], free), np.append(x["pos0"], end)
                    x["count"], held, src, free = np.append(x["count"], 0), 0, -1, free + 1
                else:
                    src = int(x["block"][-1])
                n = min(left, BLOCK - held)
                slot = np.arange(BLOCK)
                fresh = np.where((slot >= held) & (slot < held + n), at + slot - held, -1)
                x["priv"].append((int(x["block"][-1]), src, fresh, 0))
                x["count"][-1] += n
                held, left, at, end = held + n, left - n, at + n, end + n
    return {"lens": [int(n) for n in lens], "first": first, "requests": out, "n_chunk_blocks": int(first[-1]),
            "n_private": free - int(first[-1]), "taken": taken, "n_s": sum(len(x["rows"]) for x in out)}


def _attention_flops(case, g):
    return 4.0 * case["heads"] * case["dim"] * float(sum(int((x["rows"] + 1).sum()) for x in g["requests"]))


def work(case):
    hkv, d = case["kv_heads"], case["dim"]
    if case["what"] == "rope":
        values = case["rows"] * (case["heads"] + 2 * hkv) * d
        turned = case["rows"] * (case["heads"] + hkv)
        flops = turned * (3.0 * case["rot"] + (4.0 * d if case["norm"] else 0.0))
        return {"bytes": values * ((2 if case["dtype"] == "bf16" else 4) + 2) + 4 * case["rows"], "flops": flops}
    if case["what"] != "attend":
        rows = case["blocks"] * BLOCK * hkv * 2
        return {"bytes": rows * (3 * d + 1) + 8 * case["blocks"], "flops": (3.0 if case["what"] == "pack" else 1.0) * rows * d}
    g = _geometry(case)
    cached = len(set(np.concatenate([x["block"] for x in g["requests"]]).tolist()) - {p[0] for x in g["requests"] for p in x["priv"]})
    copied = sum(p[1] >= 0 and p[0] != p[1] for x in g["requests"] for p in x["priv"])
    written = sum(len(x["priv"]) for x in g["requests"])
    block = BLOCK * hkv * 2 * (d + 1)
    rows = g["n_s"] * (case["heads"] * (4 * d + 4) + 4 * hkv * d)
    return {"bytes": (cached + copied + written) * block + rows, "flops": _attention_flops(case, g)}


# ---------------------------------------------------------------- the definition

def _exponent(top):
    """Smallest t with top <= 448 * 2 ** t (0 where top is 0), in the range of an e8m0 byte."""
    f, x = torch.frexp(top)                                   # top = f 2^x, 0.5 <= f < 1; 448 = 0.875 * 2^9
    t = torch.where(f > TOP / 512.0, x - 8, x - 9)
    return torch.where(top > 0, t, torch.zeros_like(t)).clamp(-127, 127)


def _to_rows8(y):
    """Rows y [..., D] -> (y over the scale, unrounded, scale bytes [...])."""
    fine = torch.isfinite(y).all(-1)
    y = torch.where(fine[..., None], y, torch.zeros_like(y))
    t = _exponent(y.abs().amax(-1))
    byte = torch.where(fine, t + 127, torch.full_like(t, 255)).to(torch.uint8)
    return torch.ldexp(y, -t[..., None]), byte


def _of_rows8(y, byte):
    """What values y [..., D] and scale bytes [...] stand for."""
    s = torch.ldexp(torch.ones((), dtype=y.dtype, device=y.device), byte.to(torch.int32) - 127)
    return torch.where((byte == 255)[..., None], torch.full_like(y, math.nan), y * s[..., None])


def _k_order(y):
    """Tokens [..., 16, D] -> the K order."""
    y = y.unflatten(-1, (-1, 4, 16))
    n = y.dim()
    return y.permute(*range(n - 4), n - 3, n - 2, n - 4, n - 1)


def _k_tokens(y):
    """K order [..., D / 64, 4, 16, 16] -> tokens [..., 16, D]."""
    n = y.dim()
    return y.permute(*range(n - 4), n - 2, n - 4, n - 3, n - 1).flatten(-3)


def _v_order(y):
    """Tokens [..., 16, D] -> the V order."""
    y = y.unflatten(-1, (-1, 4, 16)).unflatten(-4, (4, 4))   # a c j t r
    n = y.dim()
    return y.permute(*range(n - 5), n - 3, n - 5, n - 1, n - 2, n - 4)


def _v_tokens(y):
    """V order [..., D / 64, 4, 16, 4, 4] -> tokens [..., 16, D]."""
    n = y.dim()                                               # j a r t c
    return y.permute(*range(n - 5), n - 4, n - 1, n - 5, n - 2, n - 3).flatten(-3).flatten(-3, -2)


def _e4m3(y):
    return y.to(torch.float32).to(torch.float8_e4m3fn)


def _frequencies(case):
    j = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
    f = THETA ** (-2.0 * j / case["rot"])
    if case["context"] == 0:
        return f / case["factor"]
    g = ((case["context"] * f / (2 * math.pi) - case["low"]) / (case["high"] - case["low"])).clamp(0.0, 1.0)
    return f * (g + (1.0 - g) / case["factor"])


def _pairs(x, rot, interleaved):
    a = x[..., :rot]
    return (a[..., 0::2], a[..., 1::2]) if interleaved else (a[..., :rot // 2], a[..., rot // 2:])


def _turn(x, angle, rot, interleaved, amplitude):
    """x [n, heads, d] with its first rot dims turned by angle [n, rot / 2] (float64)."""
    c, s = ((amplitude * f(angle)).to(x.dtype)[:, None] for f in (torch.cos, torch.sin))
    a, b = _pairs(x, rot, interleaved)
    y, z = a * c - b * s, b * c + a * s
    turned = torch.stack((y, z), -1).flatten(-2) if interleaved else torch.cat((y, z), -1)
    return torch.cat((turned, x[..., rot:]), -1)


# ---------------------------------------------------------------- inputs

def _loud(gen, *shape):
    """Values as keys have them: channels of unlike size, one in 32 much larger."""
    d = shape[-1]
    size = torch.exp(0.5 * torch.empty(d, device="cuda").normal_(generator=gen))
    loud = torch.rand(d, device="cuda", generator=gen) < 1.0 / 32
    return torch.empty(shape, device="cuda").normal_(generator=gen) * torch.where(loud, 4.0 * size, size)


def _normal(gen, *shape):
    return torch.empty(shape, device="cuda").normal_(generator=gen)


def _empty_cache(blocks, hkv, d):
    def empty(*shape):
        return torch.zeros(shape, dtype=torch.uint8, device="cuda")

    return {"k": empty(blocks, hkv, d // 64, 4, 16, 16), "v": empty(blocks, hkv, d // 64, 4, 16, 4, 4),
            "scale": empty(blocks, hkv, 2, 16)}


def _drawn_cache(gen, blocks, hkv, d):
    c = _empty_cache(blocks, hkv, d)
    for a in range(0, blocks, 1024):
        b = min(blocks, a + 1024)
        for i, (name, order, y) in enumerate((("k", _k_order, _loud(gen, b - a, hkv, 16, d)),
                                              ("v", _v_order, _normal(gen, b - a, hkv, 16, d)))):
            y, byte = _to_rows8(y)
            c[name][a:b] = order(_e4m3(y).view(torch.uint8))
            c["scale"][a:b, :, i] = byte
    return c


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    hkv, d = case["kv_heads"], case["dim"]
    st = {"case": case}
    bf16 = torch.bfloat16
    if case["what"] == "rope":
        n, hq = case["rows"], case["heads"]
        dtype = bf16 if case["dtype"] == "bf16" else torch.float32
        st["qkv"] = _loud(gen, n, hq + 2 * hkv, d).to(dtype).view(n, -1)
        lead = torch.randint(0, max(1, case["far"] - n + 1), (1,), device="cuda", generator=gen)
        st["pos"] = (lead + torch.arange(n, device="cuda")).to(torch.int32)
        for name in ("q_norm", "k_norm"):
            st[name] = (1.0 + 0.1 * _normal(gen, d)).to(bf16) if case["norm"] else None
        for name, h in (("q", hq), ("k", hkv), ("v", hkv)):
            st[name] = torch.empty((n, h, d), dtype=bf16, device="cuda")
        return st
    if case["what"] in ("pack", "unpack"):
        n = case["blocks"]
        for name in ("src", "dst"):
            st[name] = torch.randperm(n, device="cuda", generator=gen).to(torch.int32)
        if case["what"] == "pack":
            st["k"] = _loud(gen, n, hkv, 16, d).to(bf16)
            st["v"] = _normal(gen, n, hkv, d, 16).to(bf16)
            st["cache"] = _empty_cache(n, hkv, d)
        else:
            st["cache"] = _drawn_cache(gen, n, hkv, d)
            st["k"] = torch.empty((n, hkv, 16, d), dtype=bf16, device="cuda")
            st["v"] = torch.empty((n, hkv, d, 16), dtype=bf16, device="cuda")
        return st
    g = st["geometry"] = _geometry(case)
    # chunks' blocks lie anywhere in the pool; private ones at its end, so that a view of the end is what a pass writes
    perm = np.random.default_rng([seed, 1]).permutation(g["n_chunk_blocks"])
    place = st["place"] = np.concatenate((perm, g["n_chunk_blocks"] + np.arange(g["n_private"])))
    st["cache"] = _drawn_cache(gen, len(place), hkv, d)
    n = g["n_s"]
    st["q_s"] = _normal(gen, n, case["heads"], d).to(bf16)
    st["k_s"], st["v_s"] = _loud(gen, n, hkv, d).to(bf16), _normal(gen, n, hkv, d).to(bf16)
    st["out"] = torch.empty((n, case["heads"], d), dtype=bf16, device="cuda")
    st["lse"] = torch.empty((n, case["heads"]), dtype=torch.float32, device="cuda")

    def put(x):
        return torch.as_tensor(np.asarray(x), device="cuda")

    # the plain form's tables: linked blocks and rows of S per request, padded
    reqs = g["requests"]
    most_blocks, most_rows = max(len(x["block"]) for x in reqs), max(len(x["rows"]) for x in reqs)
    blocks = np.zeros((len(reqs), most_blocks), np.int64)
    key_pos = np.full((len(reqs), most_blocks, BLOCK), 1 << 40)
    rows, row_pos, at = np.zeros((len(reqs), most_rows), np.int64), np.zeros((len(reqs), most_rows), np.int64), 0
    for i, x in enumerate(reqs):
        blocks[i, :len(x["block"])] = place[x["block"]]
        slot = np.arange(BLOCK)
        key_pos[i, :len(x["block"])] = np.where(slot < x["count"][:, None], x["pos0"][:, None] + slot, 1 << 40)
        rows[i, :len(x["rows"])] = at + np.arange(len(x["rows"]))
        row_pos[i, :len(x["rows"])] = x["rows"]
        at += len(x["rows"])
    priv = [p for x in reqs for p in x["priv"]]
    st["tables"] = {"blocks": put(blocks), "key_pos": put(key_pos.reshape(len(reqs), -1)), "rows": put(rows),
                    "row_pos": put(row_pos), "real": put(row_pos >= 0) & (put(np.arange(most_rows)) < put(
                        [len(x["rows"]) for x in reqs])[:, None]),
                    "dst": put([place[p[0]] for p in priv]), "src": put([place[p[1]] if p[1] >= 0 else -1 for p in priv]),
                    "fresh": put(np.stack([p[2] for p in priv])), "moved": put([p[3] for p in priv])}
    return st


# ---------------------------------------------------------------- one pass

def _plan(st, el):
    """The plan a program keeps for the batch, and the workspace for it."""
    case, g, place = st["case"], st["geometry"], st["place"]
    cfg = el.attn_cfg(case["heads"], case["kv_heads"], case["dim"], rope_theta=THETA)
    ids = [[int(b) for b in place[g["first"][c]:g["first"][c + 1]]] for c in range(case["pool"])]
    free = [int(b) for b in place[g["n_chunk_blocks"]:]]
    reqs = [el.Request([g["lens"][c] for c in x["pick"]], [ids[c] for c in x["pick"]], case["suffix"], case["k"],
                       case["rerotate"]) for x in g["requests"]]
    sizes, host, _ = el.epic_plan_link(reqs, cfg, free, len(place))
    if case["mode"] == "decode":
        sizes, host, _ = el.epic_plan_decode(sizes, host, [case["new"]] * case["requests"], cfg, free[g["taken"]:],
                                             len(place))
    need = max(256, el.epic_link_kv8_workspace_bytes(cfg, sizes))
    return cfg, el.DevicePlan(sizes, host), torch.empty(need, dtype=torch.uint8, device="cuda")


def _written(st):
    """The private blocks, as the values they hold."""
    base, c = st["geometry"]["n_chunk_blocks"], st["cache"]
    return {"k": c["k"][base:].view(torch.float8_e4m3fn), "v": c["v"][base:].view(torch.float8_e4m3fn),
            "scale": c["scale"][base:].view(torch.float8_e8m0fnu)}


def _held(c):
    return {"k": c["k"].view(torch.float8_e4m3fn), "v": c["v"].view(torch.float8_e4m3fn),
            "scale": c["scale"].view(torch.float8_e8m0fnu)}


def _run_own(st):
    from paper_2410_15332_amd import epic_link as el

    case = st["case"]
    if case["what"] == "rope":
        if "rope" not in st:                     # a program keeps these for its model
            st["attn"] = el.attn_cfg(case["heads"], case["kv_heads"], case["dim"])
            st["rope"] = el.rope_cfg(case["rot"], THETA, interleaved=case["interleaved"], factor=case["factor"],
                                     original_context=case["context"], low_turns=case["low"], high_turns=case["high"],
                                     amplitude=case["amplitude"])
            st["freqs"] = torch.from_numpy(el.epic_rope_freqs(st["rope"])).cuda()
        el.epic_qk_norm_rope(st["attn"], st["rope"], st["qkv"], st["pos"], st["freqs"], st["q"], st["k"], st["v"],
                             q_norm=st["q_norm"], k_norm=st["k_norm"], eps=EPS)
        return {"q": st["q"], "k": st["k"], "v": st["v"]}
    if "kv8" not in st:
        st["kv8"] = el.Kv8Cache(st["cache"]["k"], st["cache"]["v"], st["cache"]["scale"])
    if case["what"] == "pack":
        el.epic_kv8_pack(st["k"], st["v"], st["kv8"], src_blocks=st["src"], dst_blocks=st["dst"])
        return _held(st["cache"])
    if case["what"] == "unpack":
        el.epic_kv8_unpack(st["kv8"], st["k"], st["v"], src_blocks=st["src"], dst_blocks=st["dst"])
        return {"k": st["k"], "v": st["v"]}
    if "plan" not in st:
        st["plan"] = _plan(st, el)
    cfg, plan, workspace = st["plan"]
    el.epic_link_attention_kv8(cfg, plan, st["q_s"], st["k_s"], st["v_s"], st["kv8"], st["out"], st["lse"], workspace)
    return {"out": st["out"], "lse": st["lse"], **_written(st)}


def _heads(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.to(x.dtype)


def _rope_pass(st, dtype):
    case = st["case"]
    hq, hkv = case["heads"], case["kv_heads"]
    q, k, v = st["qkv"].to(dtype).view(case["rows"], hq + 2 * hkv, case["dim"]).split((hq, hkv, hkv), 1)
    angle = st["pos"].to(torch.float64)[:, None] * _frequencies(case)
    turn = (angle, case["rot"], case["interleaved"], case["amplitude"])
    return {"q": _turn(_heads(q, st["q_norm"]), *turn), "k": _turn(_heads(k, st["k_norm"]), *turn), "v": v}


def _block_rows(c, blocks, dtype):
    """K and V [..., Hkv, 16, D] that listed blocks of an 8-bit cache stand for."""
    f8 = torch.float8_e4m3fn
    return (_of_rows8(_k_tokens(c["k"][blocks].view(f8).to(dtype)), c["scale"][blocks][..., 0, :]),
            _of_rows8(_v_tokens(c["v"][blocks].view(f8).to(dtype)), c["scale"][blocks][..., 1, :]))


def _write_private(st):
    """The private blocks: what their source holds, its keys turned where they move, then the rows of S."""
    case, c, t = st["case"], st["cache"], st["tables"]
    hkv, d = case["kv_heads"], case["dim"]
    fresh = t["fresh"]
    is_row, has_src = (fresh >= 0)[:, None, :], (t["src"] >= 0)[:, None, None]
    src = t["src"].clamp(min=0)
    for i, (name, order, tokens, rows) in enumerate((("k", _k_order, _k_tokens, st["k_s"]),
                                                     ("v", _v_order, _v_tokens, st["v_s"]))):
        old, old_byte = tokens(c[name][src]), c["scale"][src][:, :, i]
        y, byte = _to_rows8(rows.float())
        new = _e4m3(y).view(torch.uint8)[fresh.clamp(min=0)].transpose(1, 2)
        new_byte = byte[fresh.clamp(min=0)].transpose(1, 2)
        if name == "k" and case["rerotate"]:
            x = _of_rows8(old.view(torch.float8_e4m3fn).float(), old_byte)
            f = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
            x = _turn(x.flatten(1, 2), t["moved"].to(torch.float64)[:, None] * f, d, False, 1.0)
            y, b = _to_rows8(x.unflatten(1, (hkv, BLOCK)))
            moves = (t["moved"] != 0)[:, None, None]
            old = torch.where(moves[..., None], _e4m3(y).view(torch.uint8), old)
            old_byte = torch.where(moves, b, old_byte)
        none, none_byte = torch.zeros_like(old), torch.full_like(old_byte, 127)
        keep = torch.where(has_src[..., None], old, none)
        keep_byte = torch.where(has_src, old_byte, none_byte)
        c[name][t["dst"]] = order(torch.where(is_row[..., None], new, keep))
        c["scale"][t["dst"], :, i] = torch.where(is_row, new_byte, keep_byte)


def _attend(st):
    case, c, t = st["case"], st["cache"], st["tables"]
    hq, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    B, S = t["rows"].shape
    G = hq // hkv
    k, v = (x.transpose(1, 2).flatten(2, 3) for x in _block_rows(c, t["blocks"], torch.float32))   # [B, Hkv, N, D]
    real = (t["key_pos"] < 1 << 40)[:, None, :, None]
    v = torch.where(real, v, torch.zeros_like(v)).contiguous()
    kt = torch.where(real, k, torch.zeros_like(k)).transpose(2, 3).contiguous()
    q = st["q_s"].float()[t["rows"]].view(B, S, hkv, G, d).permute(0, 2, 1, 3, 4).contiguous()
    out = torch.empty((B, hkv, S, G, d), device="cuda")
    lse = torch.empty((B, hkv, S, G), device="cuda")
    step = max(1, (1 << 30) // (B * hq * kt.shape[-1]))          # rows whose scores fit 4 GB
    for a in range(0, S, step):
        b = min(S, a + step)
        s = ((q[:, :, a:b].flatten(2, 3) @ kt) / math.sqrt(d)).view(B, hkv, b - a, G, -1)
        s.masked_fill_((t["key_pos"][:, None, :] > t["row_pos"][:, a:b, None])[:, None, :, None], -math.inf)
        top = s.amax(-1, keepdim=True)
        s.sub_(top).exp_()
        total = s.sum(-1, keepdim=True)
        out[:, :, a:b] = (s.flatten(2, 3) @ v).view(B, hkv, b - a, G, d) / total
        lse[:, :, a:b] = (top + total.log())[..., 0]
    out, lse = out.permute(0, 2, 1, 3, 4).reshape(B, S, hq, d), lse.permute(0, 2, 1, 3).reshape(B, S, hq)
    return out[t["real"]].to(torch.bfloat16), lse[t["real"]]


def run(st):
    if own:
        return _run_own(st)
    case = st["case"]
    if case["what"] == "rope":
        return {name: x.to(torch.bfloat16) for name, x in _rope_pass(st, torch.float32).items()}
    src, dst = (st["src"].long(), st["dst"].long()) if case["what"] != "attend" else (None, None)
    if case["what"] == "pack":
        c = st["cache"]
        for i, (name, order, y) in enumerate((("k", _k_order, st["k"][src].float()),
                                              ("v", _v_order, st["v"][src].float().transpose(-1, -2)))):
            y, byte = _to_rows8(y)
            c[name][dst] = order(_e4m3(y).view(torch.uint8))
            c["scale"][dst, :, i] = byte
        return _held(c)
    if case["what"] == "unpack":
        k, v = _block_rows(st["cache"], src, torch.float32)
        st["k"][dst] = k.to(torch.bfloat16)
        st["v"][dst] = v.transpose(-1, -2).to(torch.bfloat16)
        return {"k": st["k"], "v": st["v"]}
    _write_private(st)
    out, lse = _attend(st)
    return {"out": out, "lse": lse, **_written(st)}


# ---------------------------------------------------------------- the same in float64

def _exact_row(y):
    """A row [..., D] in float64 -> (its values over the scale without their last rounding, the same rounded, the scale)."""
    top = y.abs().amax(-1)
    t = torch.ceil(torch.log2(top.clamp(min=2.0 ** -140) / TOP)).clamp(-127, 127)
    t = torch.where(top > TOP * torch.exp2(t), t + 1, torch.where(top <= TOP * torch.exp2(t - 1), t - 1, t)).clamp(-127, 127)
    scale = torch.exp2(torch.where(top > 0, t, torch.zeros_like(t)))
    y = y / scale[..., None]
    return y, _e4m3(y).double(), scale


def _exact_turn(x, pos, f, rot, interleaved, amplitude):
    """x [n, heads, d] in float64: pairs as complex numbers times amplitude e^(i pos f)."""
    h = rot // 2
    first = torch.arange(h, device="cuda") * 2 if interleaved else torch.arange(h, device="cuda")
    second = first + (1 if interleaved else h)
    z = torch.complex(x[..., first], x[..., second])
    z = z * torch.polar(torch.full_like(f, amplitude).expand(len(pos), -1).contiguous(), pos.double()[:, None] * f)[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def _dims(d):
    """[j, a, e] -> dim of K's order; [j, t, r] -> dim of V's."""
    return torch.arange(d, device="cuda").view(-1, 4, 16)


def _exact_block(k, v):
    """Tokens' K and V [..., 16, D] laid out in the two orders."""
    d = k.shape[-1]
    at = _dims(d)
    s = torch.arange(16, device="cuda")
    kk = k[..., s[None, None, :, None], at[:, :, None, :]]
    vv = v[..., s.view(1, 4, 1, 1, 4), at.permute(0, 2, 1)[:, None, :, :, None]]
    return kk, vv


def _exact_rows(c, block):
    """K and V [Hkv, n, D] in float64 of the tokens of listed blocks."""
    d = 64 * c["k"].shape[2]
    at, s = _dims(d), torch.arange(16, device="cuda")
    k8 = c["k"][block].view(torch.float8_e4m3fn).double()
    v8 = c["v"][block].view(torch.float8_e4m3fn).double()
    n, hkv = k8.shape[:2]
    k = torch.empty((n, hkv, 16, d), dtype=torch.float64, device="cuda")
    v = torch.empty_like(k)
    k[..., s[None, None, :, None], at[:, :, None, :]] = k8
    v[..., s.view(1, 4, 1, 1, 4), at.permute(0, 2, 1)[:, None, :, :, None]] = v8
    scale = torch.exp2(c["scale"][block].double() - 127)
    k, v = k * scale[:, :, 0, :, None], v * scale[:, :, 1, :, None]
    return k.transpose(0, 1).reshape(hkv, -1, d), v.transpose(0, 1).reshape(hkv, -1, d)


def _exact_attend(st):
    case, g, c, place = st["case"], st["geometry"], st["cache"], st["place"]
    hq, hkv, d = case["heads"], case["kv_heads"], case["dim"]
    G, base, n_s = hq // hkv, g["n_chunk_blocks"], g["n_s"]
    out = torch.empty((n_s, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((n_s, hq), dtype=torch.float64, device="cuda")
    held = {k: v.double() for k, v in _written(st).items()}
    new = [_exact_row(st[x].double().transpose(0, 1)) for x in ("k_s", "v_s")]       # [Hkv, n_s, D]
    real = [y * s[..., None] for _, y, s in new]
    f = THETA ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    row = 0
    for x in g["requests"]:
        K, V = _exact_rows(c, torch.as_tensor(place[x["block"]], device="cuda"))
        at = {int(b): i for i, b in enumerate(x["block"])}
        for dst, src, fresh, moved in x["priv"]:
            i = slice(16 * at[dst], 16 * at[dst] + 16)
            if src >= 0:
                k, v = _exact_rows(c, torch.as_tensor([place[src]], device="cuda"))
                s = torch.exp2(c["scale"][place[src]].double() - 127)
            else:
                k, v = K.new_zeros((hkv, 16, d)), K.new_zeros((hkv, 16, d))
                s = K.new_ones((hkv, 2, 16))
            ky, vy, ks, vs = k / s[:, 0, :, None], v / s[:, 1, :, None], s[:, 0].clone(), s[:, 1].clone()
            if moved:
                angle = torch.full((16,), moved, device="cuda")
                ky, rounded, ks = _exact_row(_exact_turn(k.transpose(0, 1), angle, f, d, False, 1.0).transpose(0, 1))
                k = rounded * ks[..., None]
            m = torch.as_tensor(np.flatnonzero(fresh >= 0), device="cuda")
            r = torch.as_tensor(fresh[fresh >= 0], device="cuda")
            if len(r):
                k[:, m], v[:, m] = real[0][:, r], real[1][:, r]
                ky[:, m], vy[:, m], ks[:, m], vs[:, m] = new[0][0][:, r], new[1][0][:, r], new[0][2][:, r], new[1][2][:, r]
            K[:, i], V[:, i] = k, v
            held["k"][place[dst] - base], held["v"][place[dst] - base] = _exact_block(ky, vy)
            held["scale"][place[dst] - base] = torch.stack((ks, vs), 1)
        fill = (np.arange(BLOCK) < x["count"][:, None]).reshape(-1)
        keep = torch.as_tensor(np.flatnonzero(fill), device="cuda")
        pos = torch.as_tensor((x["pos0"][:, None] + np.arange(BLOCK)).reshape(-1)[fill], device="cuda")
        n = len(x["rows"])
        p = torch.as_tensor(x["rows"], device="cuda")
        step = max(1, int(1.5e8) // (len(keep) * G))
        for h in range(hkv):
            kt, vh = K[h, keep].t().contiguous(), V[h, keep].contiguous()
            for a in range(0, n, step):
                b = min(n, a + step)
                q = st["q_s"][row + a:row + b, h * G:(h + 1) * G].double().reshape(-1, d)
                s = (q @ kt).mul_(1.0 / math.sqrt(d)).view(b - a, G, -1)
                s.masked_fill_((pos > p[a:b, None])[:, None], -math.inf)
                top = torch.logsumexp(s, -1)
                lse[row + a:row + b, h * G:(h + 1) * G] = top
                s.sub_(top[..., None]).exp_()
                out[row + a:row + b, h * G:(h + 1) * G] = (s.flatten(0, 1) @ vh).view(b - a, G, d)
        row += n
    return {"out": out, "lse": lse, **held}


def exact(case, seed):
    st = prepare(case, seed)
    hkv, d = case["kv_heads"], case["dim"]
    if case["what"] == "rope":
        hq, n = case["heads"], case["rows"]
        x = st["qkv"].double().view(n, hq + 2 * hkv, d)
        j = torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda")
        f = torch.exp(j * (-2.0 * math.log(THETA) / case["rot"]))
        if case["context"]:
            share = (case["context"] / (2 * math.pi) * f - case["low"]) / (case["high"] - case["low"])
            share = torch.minimum(torch.maximum(share, torch.zeros_like(f)), torch.ones_like(f))
            f = (1.0 - share) * f / case["factor"] + share * f
        else:
            f = f / case["factor"]
        got = {"v": x[:, hq + hkv:]}
        for name, part, w in (("q", x[:, :hq], st["q_norm"]), ("k", x[:, hq:hq + hkv], st["k_norm"])):
            if w is not None:
                part = part / (part.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
            got[name] = _exact_turn(part, st["pos"], f, case["rot"], case["interleaved"], case["amplitude"])
        return got
    if case["what"] == "pack":
        src, dst = st["src"].long(), st["dst"].long()
        k, _, ks = _exact_row(st["k"][src].double())
        v, _, vs = _exact_row(st["v"][src].double().transpose(-1, -2))
        got = dict(zip(("k", "v"), _exact_block(k, v)), scale=torch.stack((ks, vs), 2))
        return {name: y[torch.argsort(dst)] for name, y in got.items()}
    if case["what"] == "unpack":
        n = case["blocks"]
        k, v = _exact_rows(st["cache"], st["src"].long()[torch.argsort(st["dst"])])
        return {"k": k.view(hkv, n, 16, d).transpose(0, 1), "v": v.view(hkv, n, 16, d).permute(1, 0, 3, 2)}
    return _exact_attend(st)

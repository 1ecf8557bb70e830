"""Timed cases of the 8-bit paged cache: e4m3 codes with one power-of-two
scale for each row (token and KV head) of K and of V.

    quantize    cache_quantize: blocks of a bf16 or fp32 cache to e4m3 blocks
    dequantize  cache_dequantize: e4m3 blocks back to blocks of values
    append      rotary_append with scales: a step's rows normed, rotated,
                quantised and written into the e4m3 cache
    decode      branch_decode with scales: a decode step of document pages
                that reads the e4m3 cache

The cache: codes of K ``[blocks, Hkv, d/16, 16 tokens, 16 dims]``, codes of V
``[blocks, Hkv, d, 16 tokens]``, scales ``[blocks, Hkv, 2, 16]`` (K's tokens,
then V's) as exponents with a bias of 127.  A row's scale is the smallest
power of two 2^e with max |x| <= 448 * 2^e (and e >= -64).
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # False: the plain forms in torch operations; True: the library's calls

DEVICE = "cuda"
BLOCK = 16
EPS = 1e-6
MIN_EXPONENT = -64


def _blocks(name, kind, hkv, d, dtype, blocks, pairs):
    """``pairs``: blocks from drawn places to drawn places; else block for block."""
    return {"name": name, "kind": kind, "hkv": hkv, "d": d, "dtype": dtype, "blocks": blocks, "pairs": pairs}


def _append(name, hq, hkv, d, dtype, rows, streams, rotary_dim=None, style="halves", axes=3, norm=True, base=1e6, first=0):
    """``rows`` tokens of ``streams`` streams, each with rows / streams tokens one after the other in blocks of its own."""
    return {"name": name, "kind": "append", "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "rows": rows, "streams": streams,
            "rotary_dim": rotary_dim or d, "style": style, "axes": axes, "norm": norm, "base": base, "first": first}


def _decode(name, hq, hkv, d, dtype, pages, prefix, stream, branches, length, new=0, tree=0):
    """Pages of a prefix, a layout stream and ``branches`` content branches of length[0] .. length[1] tokens; the
    stream and every branch have one query, ``new`` more branches of 8 tokens eight."""
    return {"name": name, "kind": "decode", "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "pages": pages, "prefix": prefix,
            "stream": stream, "branches": branches, "len_lo": length[0], "len_hi": length[1], "new": new, "tree": tree}


def listed():
    return [
        # A page's prefix that was prefilled in bf16, handed over to the serving pool.
        _blocks("quantize_prefix_bf16", "quantize", 2, 128, "bf16", 160, True),
        # A cache of 262k tokens taken over whole.
        _blocks("quantize_cache_bf16", "quantize", 2, 128, "bf16", 16384, False),
        # A page's prefix read back into a bf16 cache.
        _blocks("dequantize_prefix_bf16", "dequantize", 2, 128, "bf16", 160, True),
        # A whole cache of 64-wide heads in fp32, as a numerics check compares it.
        _blocks("dequantize_cache_f32", "dequantize", 4, 64, "f32", 8192, False),
        # One page being decoded by itself: its layout stream and 16 branches, a token each.
        _append("append_page_bf16", 16, 2, 128, "bf16", 17, 17, first=3500),
        # A full serving batch: 64 pages of 25 streams, a token each.
        _append("append_64pages_bf16", 16, 2, 128, "bf16", 1600, 1600, first=2500),
        # The prefill of eight pages' prefixes, written in one step.
        _append("append_prefill_bf16", 16, 2, 128, "bf16", 8 * 2557, 8),
        # Half of the dimensions rotated, neighbouring ones paired, one axis, no norm, fp32, far into a document.
        _append("append_partial_f32", 28, 4, 64, "f32", 3 * 1813, 3, rotary_dim=32, style="pairs", axes=1, norm=False, base=10000.0,
                first=1000003),
        # One page being decoded by itself: a step is a chain of latencies.
        _decode("decode_page_bf16", 16, 2, 128, "bf16", 1, 1987, 251, 16, (16, 256)),
        # A full serving batch: 64 pages of 25 streams.
        _decode("decode_64pages_bf16", 16, 2, 128, "bf16", 64, 2557, 243, 24, (1, 1024)),
        # A dense page in the middle of decoding: 96 live branches and 32 just opened ones of 8 tokens.
        _decode("decode_dense_mixed", 28, 4, 128, "bf16", 1, 8101, 997, 96, (64, 2048), new=32),
        # Four pages with fp32 queries, as a precision check of a served model runs them.
        _decode("decode_4pages_f32", 16, 2, 64, "f32", 4, 1021, 131, 16, (16, 256)),
    ]


def _spread(rng, lo, hi):
    """A whole number, even over the logarithm of lo .. hi."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["quantize", "dequantize", "append", "append", "decode", "decode", "decode"])
    hq, hkv = rng.choice([(16, 2), (16, 2), (28, 4), (4, 1)])
    d = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind in ("quantize", "dequantize"):
        most = 16384 * 2 * 128 * 2 // (hkv * d * (2 if dtype == "bf16" else 4))
        c = _blocks("", kind, hkv, d, dtype, _spread(rng, 1, most), rng.random() < 0.5)
    elif kind == "append":
        rows = _spread(rng, 1, 20000 * 18 * 128 * 2 // ((hq + hkv) * d * (2 if dtype == "bf16" else 4)))
        streams = rows if rows <= 2048 and rng.random() < 0.6 else _spread(rng, 1, min(rows, 16))
        rd = rng.choice([d, d, d // 2])
        c = _append("", hq, hkv, d, dtype, rows - rows % streams, streams, rd, rng.choice(["halves", "halves", "pairs"]),
                    rng.choice([1, 3, 3]), rng.random() < 0.75, rng.choice([1e4, 1e6, 5e6]), rng.choice([0, _spread(rng, 1, 4000000)]))
    else:
        f32 = dtype == "f32"
        n = _spread(rng, 1, 16 if f32 else 96)
        c = _decode("", hq, hkv, d, dtype, _spread(rng, 1, 4 if f32 else 48), _spread(rng, 700, 1400 if f32 else 9000),
                    _spread(rng, 32, 128 if f32 else 1024), n, (1, _spread(rng, 8, 256 if f32 else 2048)),
                    rng.choice([0, 0, 0, n // 3]), rng.randrange(1 << 30))
        while c["pages"] > 1 and (_plain_floats(c) > 2.5e9 or work(c)["bytes"] > 4.5e8):
            c["pages"] -= 1
        while c["branches"] > 1 and _plain_floats(c) > 2.5e9:
            c["branches"] -= 1
    del c["name"]
    return c


# ------------------------------------------------------------------ structure

def _esize(case):
    return 2 if case["dtype"] == "bf16" else 4


def _tree(case):
    """The segments of the case's pages in packed order: arrays of parent, fork, length and queries."""
    rng = np.random.default_rng([case["tree"], 1])
    n, new, S = case["branches"], case["new"], case["stream"]
    out = []
    for page in range(case["pages"]):
        at = page * (2 + n + new)
        length = np.concatenate([rng.integers(case["len_lo"], case["len_hi"] + 1, size=n), np.full(new, 8)])
        fork = np.sort(rng.integers(1, S + 1, size=n + new)) - 1  # (the stream's newest token is not seen yet)
        one = np.zeros((2 + n + new, 4), np.int64)
        one[0] = -1, 0, case["prefix"], 0
        one[1] = at, case["prefix"], S, 1
        one[2:, 0], one[2:, 1], one[2:, 2] = at + 1, fork, length
        one[2:, 3] = np.where(np.arange(n + new) < n, 1, 8)
        out.append(one)
    return np.concatenate(out)


def _queries(case):
    """Per query row: its segment, and how many keys it sees of the prefix, the stream and its own segment."""
    t = _tree(case)
    row = np.repeat(np.arange(len(t)), t[:, 3])
    back = np.concatenate([np.arange(k)[::-1] for k in t[:, 3]])  # tokens of the segment behind the query's
    own_keys = t[row, 2] - back
    branch = t[t[row, 0], 0] >= 0
    return t, row, np.full(len(row), case["prefix"]), np.where(branch, t[row, 1], 0), own_keys


def _plain_floats(case):
    """Values of K that the plain form gathers: every query's keys, padded to the most that one sees."""
    _, row, a, b, c = _queries(case)
    return len(row) * int((a + b + c).max()) * case["hkv"] * case["d"]


def _axis_of_pairs(case):
    """The axis of every rotated pair: a quarter time and the rest in turn height and width, or all of them one axis."""
    half = case["rotary_dim"] // 2
    if case["axes"] == 1:
        return [0] * half
    return [0] * (half - 3 * half // 4) + [1 + i % 2 for i in range(3 * half // 4)]


def _pool(case):
    """Blocks of the caches."""
    if case["kind"] == "append":
        used = case["streams"] * (-(-(case["rows"] // case["streams"]) // BLOCK) + 1)
    elif case["kind"] == "decode":
        used = int((-(-_tree(case)[:, 2] // BLOCK)).sum())
    else:
        return case["blocks"] + (case["blocks"] // 4 + 8 if case["pairs"] else 0)
    return used + used // 4 + 8


def work(case):
    """Every input read once, every output written once (blocks and rows that stay as they are count nothing)."""
    es, hkv, d = _esize(case), case["hkv"], case["d"]
    if case["kind"] in ("quantize", "dequantize"):
        values = case["blocks"] * hkv * BLOCK
        return {"bytes": 2 * values * (d * es + d + 1) + (8 * case["blocks"] if case["pairs"] else 0), "flops": 4 * values * d}
    if case["kind"] == "append":
        n, hq = case["rows"], case["hq"]
        side = 4 * case["axes"] * n + (2 * d * es if case["norm"] else 0) + 8 * n
        return {"bytes": n * (2 * hq + 2 * hkv) * d * es + 2 * n * hkv * (d + 1) + side,
                "flops": (3 + (4 if case["norm"] else 0)) * n * (hq + hkv) * d + 4 * n * hkv * d}
    t, row, a, b, c = _queries(case)
    keys = int(t[:, 2].sum())
    return {"bytes": 2 * keys * hkv * (d + 1) + len(row) * case["hq"] * (2 * d * es + 4) + 4 * int((-(-t[:, 2] // BLOCK)).sum()),
            "flops": 4 * d * case["hq"] * int((a + b + c).sum())}


# --------------------------------------------------------------------- inputs

def _generator(seed, stream):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 1000003 + stream)
    return g


def _normal(shape, seed, stream, case=None):
    x = torch.randn(shape, generator=_generator(seed, stream), device=DEVICE, dtype=torch.float32)
    return x.to(torch.bfloat16) if case is not None and case["dtype"] == "bf16" else x


def _rows(shape, seed, stream, case=None):
    """Rows of values as K and V have them: some rows larger than others."""
    x = _normal(shape, seed, stream) * torch.exp(0.5 * _normal(shape[:-1] + (1,), seed, stream + 50))
    return x.to(torch.bfloat16) if case is not None and case["dtype"] == "bf16" else x


def _kslot(t):
    """The place of token t in a block of the bf16 / fp32 K cache: bits 2 and 3 of it exchanged."""
    return (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1)


def _power(e):
    """2^e for whole numbers -127 < e < 128, exactly."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _code(rows):
    """Codes and scale exponents (biased) of rows of values, in 32 bits."""
    x = rows.float()
    m, ex = torch.frexp(x.abs().amax(-1))
    e = (ex - 9 + (m > 0.875)).clamp_min(MIN_EXPONENT)
    e = torch.where(m == 0, MIN_EXPONENT, e)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """What codes stand for, in 32 bits: rows of codes and a biased exponent each."""
    return codes.view(torch.float8_e4m3fn).float() * _power(scales.int() - 127)[..., None]


def _empty(case, n, seed):
    """An e4m3 cache that other streams' tokens fill, as bytes."""
    k = _normal((n, case["hkv"], case["d"] // BLOCK, BLOCK, 16), seed, 5).to(torch.float8_e4m3fn).view(torch.uint8)
    v = _normal((n, case["hkv"], case["d"], BLOCK), seed, 6).to(torch.float8_e4m3fn).view(torch.uint8)
    s = torch.randint(118, 130, (n, case["hkv"], 2, BLOCK), generator=_generator(seed, 7), device=DEVICE, dtype=torch.uint8)
    return k, v, s


def _filled(case, n, seed):
    """An e4m3 cache of n blocks of rows, as bytes."""
    shape = (n, case["hkv"], BLOCK, case["d"])
    kc, ks = _code(_rows(shape, seed, 1))
    vc, vs = _code(_rows(shape, seed, 2))
    k = kc.view(n, case["hkv"], BLOCK, case["d"] // 16, 16).transpose(2, 3).contiguous()
    return k, vc.transpose(2, 3).contiguous(), torch.stack([ks, vs], 2)


def _places(case, seed):
    """(source, destination) blocks in drawn places."""
    rng = np.random.default_rng([seed, 9])
    p = np.stack([rng.permutation(_pool(case))[:case["blocks"]] for _ in range(2)], 1)
    return torch.from_numpy(np.ascontiguousarray(p, dtype=np.int32)).to(DEVICE)


def _positions(case, seed):
    """int32 [axes, n]: image tokens first (time stands, height and width run over a grid about 64 wide), then text
    (all axes run on together)."""
    n = case["rows"]
    rng = np.random.default_rng([seed, 7])
    if case["axes"] == 1:
        p = case["first"] + np.arange(n)[None]
    elif case["streams"] == n:  # a token of each stream
        p = np.broadcast_to(case["first"] + rng.integers(0, 1024, size=n), (3, n))
    else:
        image, width = n // 2, 57 + int(rng.integers(0, 16))
        j = np.arange(image)
        text = max(image and image // width + 1, min(image, width)) + np.arange(n - image)
        p = case["first"] + np.concatenate([np.stack([0 * j, j // width, j % width]), np.stack([text] * 3)], 1)
    return torch.from_numpy(np.ascontiguousarray(p, dtype=np.int32)).to(DEVICE)


def _slots(case, seed):
    """(block, slot) of every new row: streams at drawn lengths go on in blocks in drawn places."""
    rng = np.random.default_rng([seed, 8])
    each = case["rows"] // case["streams"]
    at = (rng.integers(0, BLOCK, size=(case["streams"], 1)) if each < 512 else 0) + np.arange(each)[None]
    per = -(-each // BLOCK) + 1
    ids = rng.permutation(_pool(case))[:case["streams"] * per].reshape(case["streams"], per)
    blk = np.take_along_axis(ids, np.broadcast_to(at // BLOCK, (case["streams"], each)), 1)
    out = np.stack([blk, np.broadcast_to(at % BLOCK, blk.shape)], -1).reshape(-1, 2)
    return torch.from_numpy(np.ascontiguousarray(out, dtype=np.int32)).to(DEVICE)


def _inputs(case, seed):
    hkv, d = case["hkv"], case["d"]
    st = {"case": case}
    if case["kind"] in ("quantize", "dequantize"):
        n = _pool(case)
        st["pairs"] = _places(case, seed) if case["pairs"] else None
        if case["kind"] == "dequantize":
            st["codes"] = _filled(case, n, seed)
            st["kc"], st["vc"] = _normal((n, hkv, d // 8, BLOCK, 8), seed, 5, case), _normal((n, hkv, d, BLOCK), seed, 6, case)
        else:
            k = _rows((n, hkv, BLOCK, d), seed, 1, case)  # of slots; chunk-major as the cache holds them
            st["kc"] = k.view(n, hkv, BLOCK, d // 8, 8).transpose(2, 3).contiguous()
            st["vc"] = _rows((n, hkv, BLOCK, d), seed, 2, case).transpose(2, 3).contiguous()
            st["codes"] = _empty(case, n, seed)
    elif case["kind"] == "append":
        n, hq = case["rows"], case["hq"]
        st["qkv"], st["pos"], st["slots"] = _rows((n, hq + 2 * hkv, d), seed, 1, case), _positions(case, seed), _slots(case, seed)
        st["wq"], st["wk"] = ((1 + 0.2 * _normal((d,), seed, s)).to(st["qkv"].dtype) if case["norm"] else None for s in (3, 4))
        st["codes"] = _empty(case, _pool(case), seed)
    else:
        n = _pool(case)
        t = _tree(case)
        st["codes"] = _filled(case, n, seed)
        st["ids"] = np.random.default_rng([seed, 9]).permutation(n)[:int((-(-t[:, 2] // BLOCK)).sum())].astype(np.int32)
        st["table"] = torch.from_numpy(st["ids"]).to(DEVICE)
        st["q"] = _normal((int(t[:, 3].sum()), case["hq"], d), seed, 3, case)
    return st


def _rotary(case):
    import paper_2608_06146_amd as pa
    return pa.Rotary(case["d"], case["dtype"], rotary_dim=case["rotary_dim"], axis=_axis_of_pairs(case), base=case["base"],
                     style=case["style"], eps=EPS)


def _plan(case, st):
    import paper_2608_06146_amd as pa
    t = _tree(case)
    segs = pa.segments_layout([tuple(int(v) for v in s) for s in t], BLOCK)
    return pa.TreePlan(segs, case["hq"], case["hkv"], case["d"], case["dtype"] + "_e4m3", BLOCK, num_kv_rows=_pool(case),
                       num_q_rows=len(st["q"]), block_table_host=st["ids"])


def _key_index(case, st):
    """Per query the rows of the cache (block * 16 + slot) that it sees, padded, and their number."""
    t, row, a, b, c = _queries(case)
    first = np.concatenate([[0], np.cumsum(-(-t[:, 2] // BLOCK))])  # first block-table entry of a segment
    stream = np.where(t[t[row, 0], 0] >= 0, t[row, 0], row)
    prefix = t[stream, 0]
    a, b, c, fa, fb, fc = (torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE)[:, None]
                           for x in (a, b, c, first[prefix], first[stream], first[row]))
    j = torch.arange(int((a + b + c).max()), device=DEVICE)[None]
    tok = torch.where(j < a, j, torch.where(j < a + b, j - a, j - a - b))
    entry = torch.where(j < a, fa, torch.where(j < a + b, fb, fc)) + tok // BLOCK
    n = a + b + c
    entry = torch.where(j < n, entry, 0)
    return st["table"].long()[entry] * BLOCK + tok % BLOCK, n


def prepare(case, seed):
    st = _inputs(case, seed)
    codes = st.pop("codes")
    if own:
        st["k8"], st["v8"] = (x.view(torch.float8_e4m3fn) for x in codes[:2])
        st["s8"] = codes[2].view(torch.float8_e8m0fnu)
    else:
        st["k8"], st["v8"], st["s8"] = codes
    if case["kind"] == "append":
        if own:
            st["rotary"] = _rotary(case)
        else:
            st["freq"] = case["base"] ** (torch.arange(case["rotary_dim"] // 2, dtype=torch.float64, device=DEVICE) * (-2.0 / case["rotary_dim"]))
            st["axis"] = torch.tensor(_axis_of_pairs(case), device=DEVICE)
    if case["kind"] == "decode":
        if own:
            st["plan"] = _plan(case, st)
            st["out"], st["lse"] = torch.empty_like(st["q"]), torch.empty(st["q"].shape[:2], dtype=torch.float32, device=DEVICE)
            st["ws"] = st["plan"].workspace(torch.device(DEVICE, torch.cuda.current_device()))
        else:
            st["keys"], st["count"] = _key_index(case, st)
    return st


# ----------------------------------------------------------------- plain forms

def _as_values(st):
    """The e4m3 cache that the state holds, as numbers: codes and scales."""
    return st["k8"].view(torch.float8_e4m3fn), st["v8"].view(torch.float8_e4m3fn), st["s8"].view(torch.float8_e8m0fnu)


def _write(st, blk, slot, k, v):
    """Rows [n, Hkv, d] of values into the e4m3 cache."""
    n, hkv, d = k.shape
    for rows, part in ((k, 0), (v, 1)):
        codes, scale = _code(rows)
        if part == 0:
            st["k8"][blk, :, :, slot] = codes.view(n, hkv, d // 16, 16)
        else:
            st["v8"][blk, :, :, slot] = codes
        st["s8"][blk, :, part, slot] = scale


def _plain_quantize(st):
    c = st["case"]
    k, v = st["kc"], st["vc"]
    if st["pairs"] is not None:
        src = st["pairs"][:, 0].long()
        k, v = k[src], v[src]
    t = torch.arange(BLOCK, device=DEVICE)
    n, hkv, d = len(k), c["hkv"], c["d"]
    kc, ks = _code(k[:, :, :, _kslot(t)].transpose(2, 3).reshape(n, hkv, BLOCK, d))
    vc, vs = _code(v.transpose(2, 3))
    kc = kc.view(n, hkv, BLOCK, d // 16, 16).transpose(2, 3)
    to = st["pairs"][:, 1].long() if st["pairs"] is not None else slice(None)
    st["k8"][to] = kc
    st["v8"][to] = vc.transpose(2, 3)
    st["s8"][to] = torch.stack([ks, vs], 2)
    return _as_values(st)


def _plain_dequantize(st):
    c = st["case"]
    k, v, s = st["k8"], st["v8"], st["s8"]
    if st["pairs"] is not None:
        src = st["pairs"][:, 0].long()
        k, v, s = k[src], v[src], s[src]
    n, hkv, d = len(k), c["hkv"], c["d"]
    t = torch.arange(BLOCK, device=DEVICE)
    kv = _values(k.transpose(2, 3).reshape(n, hkv, BLOCK, d), s[:, :, 0]).to(st["kc"].dtype)
    kv = kv.view(n, hkv, BLOCK, d // 8, 8).transpose(2, 3)
    vv = _values(v.transpose(2, 3), s[:, :, 1]).to(st["vc"].dtype).transpose(2, 3)
    to = st["pairs"][:, 1].long() if st["pairs"] is not None else slice(None)
    st["kc"][to] = kv[:, :, :, _kslot(t)]
    st["vc"][to] = vv
    return st["kc"], st["vc"]


def _members(y, case):
    """The two members of every rotated pair, and the dimensions left as they are."""
    rd = case["rotary_dim"]
    a, b = (y[..., :rd // 2], y[..., rd // 2:rd]) if case["style"] == "halves" else (y[..., :rd:2], y[..., 1:rd:2])
    return a, b, y[..., rd:]


def _turned(x, w, cos, sin, case):
    """Norm and rotation of rows, in 32 bits."""
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    a, b, rest = _members(y, case)
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([a, b, rest], -1) if case["style"] == "halves" else torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)


def _qkv(st):
    hq, hkv = st["case"]["hq"], st["case"]["hkv"]
    x = st["qkv"]
    return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]


def _plain_append(st):
    c = st["case"]
    q, k, v = _qkv(st)
    ang = st["pos"].double().index_select(0, st["axis"]).t() * st["freq"]  # (64 bits: far positions)
    cos, sin = ang.cos().float()[:, None], ang.sin().float()[:, None]
    blk, t = st["slots"][:, 0].long(), st["slots"][:, 1].long()
    _write(st, blk, t, _turned(k, st["wk"], cos, sin, c), v)
    return (_turned(q, st["wq"], cos, sin, c).to(q.dtype),) + _as_values(st)


def _plain_decode(st):
    c = st["case"]
    n, hkv, d = len(st["q"]), c["hkv"], c["d"]
    k = _values(st["k8"].permute(0, 3, 1, 2, 4).reshape(-1, hkv, d), st["s8"][:, :, 0].transpose(1, 2).reshape(-1, hkv))
    v = _values(st["v8"].permute(0, 3, 1, 2).reshape(-1, hkv, d), st["s8"][:, :, 1].transpose(1, 2).reshape(-1, hkv))
    q = st["q"].float().view(n, hkv, c["hq"] // hkv, d)
    s = torch.matmul(q, k[st["keys"]].permute(0, 2, 3, 1).contiguous()) * (1 / math.sqrt(d))
    hidden = torch.arange(s.shape[-1], device=DEVICE)[None] >= st["count"]
    s = s.masked_fill(hidden[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v[st["keys"]].transpose(1, 2).contiguous()) / total
    lse = (top + torch.log(total)).reshape(n, c["hq"])
    return o.reshape(n, c["hq"], d).to(st["q"].dtype), lse


_PLAIN = {"quantize": _plain_quantize, "dequantize": _plain_dequantize, "append": _plain_append, "decode": _plain_decode}


def _call(st):
    import paper_2608_06146_amd as pa
    kind = st["case"]["kind"]
    if kind == "quantize":
        return pa.cache_quantize(st["kc"], st["vc"], st["k8"], st["v8"], st["s8"], pairs=st["pairs"])
    if kind == "dequantize":
        return pa.cache_dequantize(st["k8"], st["v8"], st["s8"], st["kc"], st["vc"], pairs=st["pairs"])
    if kind == "append":
        q, k, v = _qkv(st)
        qr = pa.rotary_append(q, k, v, st["pos"], st["slots"], st["k8"], st["v8"], st["rotary"], st["wq"], st["wk"], scales=st["s8"])
        return qr, st["k8"], st["v8"], st["s8"]
    return pa.branch_decode(st["q"], st["k8"], st["v8"], st["table"], st["plan"], st["out"], st["lse"], st["ws"], scales=st["s8"])


def run(state):
    return _call(state) if own else _PLAIN[state["case"]["kind"]](state)


# -------------------------------------------------------------- in 64 bits

def _exact_code(x):
    """Codes (as the numbers they are) and scales of rows in 64 bits: the grid written out."""
    a = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(a, float(MIN_EXPONENT))
    big = a > 448 * 2.0 ** MIN_EXPONENT
    e[big] = torch.ceil(torch.log2(a[big] / 448))
    e = torch.where(a > 448 * torch.exp2(e), e + 1, torch.where((a <= 448 * torch.exp2(e - 1)) & (e > MIN_EXPONENT), e - 1, e))
    y = x * torch.exp2(-e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(y / step) * step, torch.exp2(e[..., 0])


def _exact_cache(st):
    k, v, s = st["codes"]
    return (k.view(torch.float8_e4m3fn).double(), v.view(torch.float8_e4m3fn).double(), torch.exp2(s.double() - 127))


_PLACE = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]


def _exact_quantize(case, st):
    k8, v8, s8 = _exact_cache(st)
    src, dst = st["pairs"].long().unbind(1) if case["pairs"] else (torch.arange(_pool(case), device=DEVICE),) * 2
    k = st["kc"].double().index_select(0, src)[:, :, :, _PLACE].permute(0, 1, 3, 2, 4).flatten(3)
    v = st["vc"].double().index_select(0, src).permute(0, 1, 3, 2)
    (kc, ks), (vc, vs) = _exact_code(k), _exact_code(v)
    return (k8.index_copy(0, dst, kc.unflatten(3, (-1, 16)).permute(0, 1, 3, 2, 4)),
            v8.index_copy(0, dst, vc.permute(0, 1, 3, 2)), s8.index_copy(0, dst, torch.stack([ks, vs], 2)))


def _exact_dequantize(case, st):
    k8, v8, s8 = _exact_cache(st)
    src, dst = st["pairs"].long().unbind(1) if case["pairs"] else (torch.arange(_pool(case), device=DEVICE),) * 2
    k = (k8 * s8[:, :, 0, None, :, None]).index_select(0, src)
    k = k.permute(0, 1, 3, 2, 4).flatten(3).unflatten(3, (-1, 8)).permute(0, 1, 3, 2, 4)[:, :, :, _PLACE]
    v = (v8 * s8[:, :, 1, None, :]).index_select(0, src)
    return st["kc"].double().index_copy(0, dst, k), st["vc"].double().index_copy(0, dst, v)


def _exact_rows(x, w, pos, case):
    """Pairs as complex numbers, turned by exp(i angle)."""
    d, rd = case["d"], case["rotary_dim"]
    if w is not None:
        x = x * w * (d / ((x ** 2).sum(-1, keepdim=True) + d * EPS)) ** 0.5
    i = torch.arange(rd // 2, dtype=torch.float64, device=x.device)
    freq = torch.exp(i * (-2.0 / rd * math.log(case["base"])))
    ang = pos.double()[_axis_of_pairs(case)].t() * freq
    turn = torch.polar(torch.ones_like(ang), ang)[:, None]
    head = x[..., :rd]
    if case["style"] == "halves":
        z = torch.complex(head[..., :rd // 2], head[..., rd // 2:]) * turn
        head = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(head[..., 0::2], head[..., 1::2]) * turn
        head = torch.view_as_real(z).reshape(head.shape)
    return torch.cat([head, x[..., rd:]], -1)


def _exact_append(case, st):
    k8, v8, s8 = _exact_cache(st)
    q, k, v = (x.double() for x in _qkv(st))
    wq, wk = (None if w is None else w.double() for w in (st["wq"], st["wk"]))
    (kc, ks), (vc, vs) = _exact_code(_exact_rows(k, wk, st["pos"], case)), _exact_code(v)
    at = st["slots"].long().unbind(1)
    k8.permute(0, 3, 1, 2, 4).index_put_(at, kc.unflatten(2, (-1, 16)))
    v8.permute(0, 3, 1, 2).index_put_(at, vc)
    s8.permute(0, 3, 1, 2).index_put_(at, torch.stack([ks, vs], 2))
    return _exact_rows(q, wq, st["pos"], case), k8, v8, s8


def _exact_decode(case, st):
    """Segment by segment: scores against the prefix, the stream up to the fork and the segment's own keys."""
    k8, v8, s8 = _exact_cache(st)
    hkv, d, G = case["hkv"], case["d"], case["hq"] // case["hkv"]
    ids = st["table"].long()
    rows_k = (k8 * s8[:, :, 0, None, :, None]).permute(0, 3, 1, 2, 4).flatten(3)  # [blocks, 16, Hkv, d]
    rows_v = (v8 * s8[:, :, 1, None, :]).permute(0, 3, 1, 2)
    t = _tree(case)
    first = np.concatenate([[0], np.cumsum(-(-t[:, 2] // BLOCK))])
    keys = lambda rows, s, n: rows[ids[first[s]:first[s + 1]]].flatten(0, 1)[:n]  # noqa: E731
    o, lse, at = [], [], 0
    for s in np.nonzero(t[:, 3])[0]:
        n_q, chain = int(t[s, 3]), [(int(s), int(t[s, 2]))]
        while t[chain[-1][0], 0] >= 0:
            chain.append((int(t[chain[-1][0], 0]), int(t[chain[-1][0], 1])))
        k, v = (torch.cat([keys(r, *link) for link in chain]).transpose(0, 1) for r in (rows_k, rows_v))  # [Hkv, keys, d]
        q = st["q"][at:at + n_q].double().unflatten(1, (hkv, G)).permute(1, 0, 2, 3).flatten(1, 2)  # [Hkv, n_q G, d]
        score = torch.bmm(q, k.transpose(1, 2).contiguous()) * d ** -0.5
        behind = torch.arange(n_q, device=DEVICE).flip(0).repeat_interleave(G)[:, None]  # own keys after the query's
        own_at = torch.arange(k.shape[1], device=DEVICE)[None]
        score.masked_fill_((own_at < t[s, 2]) & (own_at >= t[s, 2] - behind), -math.inf)
        z = torch.logsumexp(score, -1, keepdim=True)
        o.append(torch.bmm(torch.exp(score - z), v.contiguous()).unflatten(1, (n_q, G)).transpose(0, 1).flatten(1, 2))
        lse.append(z.unflatten(1, (n_q, G)).transpose(0, 1).flatten(1))
        at += n_q
    return torch.cat(o), torch.cat(lse)


def exact(case, seed):
    st = _inputs(case, seed)
    return {"quantize": _exact_quantize, "dequantize": _exact_dequantize, "append": _exact_append, "decode": _exact_decode}[case["kind"]](case, st)

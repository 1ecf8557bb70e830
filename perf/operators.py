"""Timed cases of the operators around tree attention: what a decoder layer
does to Q and K before it, and what a server does to the paged cache.

    forward   rotary_fwd: per-head RMS norm of Q and K, then the rotation by
              their tokens' positions (several axes: time, height, width)
    backward  rotary_bwd: the gradients of that, of both norm weights too
    append    rotary_append: a decode step's new rows normed, rotated and
              written into the paged caches
    copy      cache_copy_blocks: blocks of the paged caches to other blocks

Q, K and V are the rows of one fused projection, ``[n, (Hq + 2 Hkv) d]``.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False  # False: the plain forms in torch operations; True: the library's calls

DEVICE = "cuda"
BLOCK = 16
EPS = 1e-6


def _case(name, kind, hq, hkv, d, dtype, rows, rotary_dim=None, style="halves", axes=3, norm=True, base=1e6, scale=1.0,
          first=0, streams=1):
    """``rows`` tokens; ``first`` the position they begin at; ``streams`` (append) the streams they belong to: each
    gets rows / streams tokens, one after the other in blocks of its own."""
    return {"name": name, "kind": kind, "hq": hq, "hkv": hkv, "d": d, "dtype": dtype, "rows": rows,
            "rotary_dim": rotary_dim or d, "style": style, "axes": axes, "norm": norm, "base": base, "scale": scale,
            "first": first, "streams": streams}


def listed():
    return [
        # A content branch's 81 tokens when it is created while serving: one launch's latency.
        _case("forward_branch_bf16", "forward", 16, 2, 128, "bf16", 81, first=3500),
        # One page's packed sample, every token.
        _case("forward_page_bf16", "forward", 16, 2, 128, "bf16", 3479),
        # Half of the rotated dimensions, neighbouring dimensions paired, one axis, no norm, fp32: a numerics check of
        # such a model, far into a long document.
        _case("forward_partial_f32", "forward", 28, 4, 64, "f32", 5437, rotary_dim=32, style="pairs", axes=1, norm=False,
              base=10000.0, first=1000003),
        # A training micro-batch: eight ragged pages packed without padding.
        _case("forward_8pages_bf16", "forward", 16, 2, 128, "bf16", 43067),
        # The gradients of a unit-sized page in fp32, of one page, and of the micro-batch.
        _case("backward_tiny_f32", "backward", 4, 1, 64, "f32", 448),
        _case("backward_page_bf16", "backward", 16, 2, 128, "bf16", 3479),
        _case("backward_8pages_bf16", "backward", 16, 2, 128, "bf16", 43067),
        # One page being decoded by itself: its layout stream and 16 branches, a token each.
        _case("append_page_bf16", "append", 16, 2, 128, "bf16", 17, first=3500, streams=17),
        # A full serving batch: 64 pages of 25 streams, a token each.
        _case("append_64pages_bf16", "append", 16, 2, 128, "bf16", 1600, first=2500, streams=1600),
        # The prefill of eight pages' prefixes, written in one step.
        _case("append_prefill_bf16", "append", 16, 2, 128, "bf16", 8 * 2557, streams=8),
        # The partly filled blocks of 24 forked streams, copied before they are written to.
        {"name": "copy_forks_bf16", "kind": "copy", "hkv": 2, "d": 128, "dtype": "bf16", "blocks": 24},
        # A cache that 262k tokens still occupy, moved to the front of its pool.
        {"name": "copy_compact_bf16", "kind": "copy", "hkv": 2, "d": 128, "dtype": "bf16", "blocks": 16384},
    ]


def _spread(rng, lo, hi):
    """A whole number, even over the logarithm of lo .. hi."""
    return max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["forward", "forward", "backward", "backward", "append", "append", "copy"])
    hq, hkv = rng.choice([(16, 2), (16, 2), (28, 4), (4, 1)])
    d = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "copy":
        return {"kind": kind, "hkv": hkv, "d": d, "dtype": dtype, "blocks": _spread(rng, 1, 16384 // hkv)}
    most = {"forward": 43000, "backward": 43000, "append": 20000}[kind] * 18 * 128 * 2
    rows = _spread(rng, 1, most // ((hq + hkv) * d * (2 if dtype == "bf16" else 4)))
    streams = 1
    if kind == "append":
        streams = rows if rows <= 2048 and rng.random() < 0.6 else _spread(rng, 1, min(rows, 16))
        rows -= rows % streams
    rotary_dim = rng.choice([d, d, d // 2])
    c = _case("", kind, hq, hkv, d, dtype, rows, rotary_dim, rng.choice(["halves", "halves", "pairs"]), rng.choice([1, 3, 3]),
              rng.random() < 0.75, rng.choice([1e4, 1e6, 5e6]), rng.choice([1.0, 1.0, 1.2]),
              rng.choice([0, _spread(rng, 1, 4000000)]), streams)
    del c["name"]
    return c


# --------------------------------------------------------------------- sizes

def _esize(case):
    return 2 if case["dtype"] == "bf16" else 4


def _pool(case):
    """Blocks of the caches: those that are written or copied, and a quarter more."""
    used = case["streams"] * (-(-(case["rows"] // case["streams"]) // BLOCK) + 1) if case["kind"] == "append" else 2 * case["blocks"]
    return used + used // 4 + 8


def work(case):
    """Every input read once, every output written once (blocks and rows that stay as they are count nothing)."""
    es, hkv, d = _esize(case), case["hkv"], case["d"]
    if case["kind"] == "copy":
        return {"bytes": 4 * case["blocks"] * hkv * BLOCK * d * es + 8 * case["blocks"], "flops": 0}
    n, hq = case["rows"], case["hq"]
    heads = n * (hq + hkv) * d
    side = 4 * case["axes"] * n + (2 * d * es if case["norm"] else 0)
    per = 3 + (4 if case["norm"] else 0)  # a rotation: two products and a sum a value; a norm: square, sum, two products
    if case["kind"] == "forward":
        return {"bytes": 2 * heads * es + side, "flops": per * heads}
    if case["kind"] == "backward":  # gradients in and out; the rows and both weights' gradients where there is a norm
        return {"bytes": (3 if case["norm"] else 2) * heads * es + side + (8 * d if case["norm"] else 0),
                "flops": (3 + (10 if case["norm"] else 0)) * heads}
    return {"bytes": 2 * heads * es + 2 * n * hkv * d * es + side + 8 * n, "flops": per * heads}


# --------------------------------------------------------------------- inputs

def _normal(shape, seed, stream, case):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 1000003 + stream)
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)
    return x.to(torch.bfloat16) if case["dtype"] == "bf16" else x


def _axis_of_pairs(case):
    """The axis of every rotated pair: a quarter time and the rest in turn height and width, or all of them one axis."""
    half = case["rotary_dim"] // 2
    if case["axes"] == 1:
        return [0] * half
    return [0] * (half - 3 * half // 4) + [1 + i % 2 for i in range(3 * half // 4)]


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


def _caches(case, seed):
    shape = (_pool(case), case["hkv"])
    return (_normal(shape + (case["d"] // 8, BLOCK, 8), seed, 5, case), _normal(shape + (case["d"], BLOCK), seed, 6, case))


def _weights(case, seed):
    if not case["norm"]:
        return None, None
    return tuple((1 + 0.2 * _normal((case["d"],), seed, s, case).float()).to(_normal((1,), seed, s, case).dtype) for s in (3, 4))


def _inputs(case, seed):
    if case["kind"] == "copy":
        kc, vc = _caches(case, seed)
        ids = np.random.default_rng([seed, 9]).permutation(_pool(case))[:2 * case["blocks"]].astype(np.int32)
        return {"kc": kc, "vc": vc, "pairs": torch.from_numpy(ids.reshape(-1, 2).copy()).to(DEVICE)}
    n, hq, hkv, d = (case[k] for k in ("rows", "hq", "hkv", "d"))
    x = {"qkv": _normal((n, (hq + 2 * hkv) * d), seed, 1, case), "pos": _positions(case, seed)}
    x["wq"], x["wk"] = _weights(case, seed)
    if case["kind"] == "backward":
        x["gq"], x["gk"] = _normal((n, hq, d), seed, 2, case), _normal((n, hkv, d), seed, 10, case)
    if case["kind"] == "append":
        x["kc"], x["vc"] = _caches(case, seed)
        x["slots"] = _slots(case, seed)
    return x


def prepare(case, seed):
    st = _inputs(case, seed)
    st["case"] = case
    if case["kind"] == "copy":
        return st
    rd = case["rotary_dim"]
    if own:
        import paper_2608_06146_amd as pa
        st["rotary"] = pa.Rotary(case["d"], case["dtype"], rotary_dim=rd, axis=_axis_of_pairs(case), base=case["base"],
                                 style=case["style"], scale=case["scale"], eps=EPS)
    else:
        st["freq"] = case["base"] ** (torch.arange(rd // 2, dtype=torch.float64, device=DEVICE) * (-2.0 / rd))
        st["axis"] = torch.tensor(_axis_of_pairs(case), device=DEVICE)
    return st


# ----------------------------------------------------------------- plain forms

def _heads(st):
    """Views of the fused rows: q [n, Hq, d], k and v [n, Hkv, d]."""
    c = st["case"]
    x = st["qkv"].view(c["rows"], c["hq"] + 2 * c["hkv"], c["d"])
    return x[:, :c["hq"]], x[:, c["hq"]:c["hq"] + c["hkv"]], x[:, c["hq"] + c["hkv"]:]


def _cos_sin(st):
    """[n, 1, rotary_dim / 2]: the angles in 64 bits (far positions), their cosines and sines in 32."""
    ang = st["pos"].double().index_select(0, st["axis"]).t() * st["freq"]
    s = st["case"]["scale"]
    return (ang.cos() * s).float()[:, None], (ang.sin() * s).float()[:, None]


def _members(y, case):
    """The two members of every rotated pair, and the dimensions left as they are."""
    rd = case["rotary_dim"]
    a, b = (y[..., :rd // 2], y[..., rd // 2:rd]) if case["style"] == "halves" else (y[..., :rd:2], y[..., 1:rd:2])
    return a, b, y[..., rd:]


def _joined(a, b, rest, case):
    if case["style"] == "halves":
        return torch.cat([a, b, rest], -1)
    return torch.cat([torch.stack([a, b], -1).flatten(-2), rest], -1)


def _rotated(x, w, cos, sin, case):
    y = x.float()
    if w is not None:
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
    a, b, rest = _members(y, case)
    return _joined(a * cos - b * sin, b * cos + a * sin, rest, case).to(x.dtype)


def _rotated_grad(g, x, w, cos, sin, case):
    a, b, rest = _members(g.float(), case)
    dy = _joined(a * cos + b * sin, b * cos - a * sin, rest, case)
    if w is None:
        return dy.to(g.dtype), None
    x = x.float()
    r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * r
    dn = dy * w.float()
    dx = r * (dn - n * (dn * n).mean(-1, keepdim=True))
    return dx.to(g.dtype), (dy * n).sum((0, 1), dtype=torch.float64).float()


def _kslot(t):
    """The place of token t in a block of the K cache: bits 2 and 3 of it exchanged."""
    return (t & 3) | ((t & 4) << 1) | ((t & 8) >> 1)


def _plain(st):
    c = st["case"]
    if c["kind"] == "copy":
        src, dst = st["pairs"][:, 0], st["pairs"][:, 1]
        st["kc"][dst] = st["kc"][src]
        st["vc"][dst] = st["vc"][src]
        return st["kc"], st["vc"]
    q, k, v = _heads(st)
    cos, sin = _cos_sin(st)
    if c["kind"] == "backward":
        dq, dwq = _rotated_grad(st["gq"], q, st["wq"], cos, sin, c)
        dk, dwk = _rotated_grad(st["gk"], k, st["wk"], cos, sin, c)
        return (dq, dk) if dwq is None else (dq, dk, dwq, dwk)
    qr, kr = _rotated(q, st["wq"], cos, sin, c), _rotated(k, st["wk"], cos, sin, c)
    if c["kind"] == "forward":
        return qr, kr
    blk, t = st["slots"][:, 0].long(), st["slots"][:, 1].long()
    st["kc"][blk, :, :, _kslot(t)] = kr.view(c["rows"], c["hkv"], c["d"] // 8, 8)
    st["vc"][blk, :, :, t] = v
    return qr, st["kc"], st["vc"]


def _call(st):
    import paper_2608_06146_amd as pa
    c = st["case"]
    if c["kind"] == "copy":
        return pa.cache_copy_blocks(st["kc"], st["vc"], st["pairs"])
    q, k, v = _heads(st)
    if c["kind"] == "forward":
        return pa.rotary_fwd(q, k, st["pos"], st["rotary"], st["wq"], st["wk"])
    if c["kind"] == "backward":
        out = pa.rotary_bwd(st["gq"], st["gk"], st["pos"], st["rotary"], q, k, st["wq"], st["wk"])
        return out if c["norm"] else out[:2]
    qr = pa.rotary_append(q, k, v, st["pos"], st["slots"], st["kc"], st["vc"], st["rotary"], st["wq"], st["wk"])
    return qr, st["kc"], st["vc"]


def run(state):
    return _call(state) if own else _plain(state)


# -------------------------------------------------------------- in 64 bits

def _exact_rows(x, w, pos, case):
    """Pairs as complex numbers, turned by exp(i angle)."""
    d, rd = case["d"], case["rotary_dim"]
    if w is not None:
        x = x * w * (d / ((x ** 2).sum(-1, keepdim=True) + d * EPS)) ** 0.5
    i = torch.arange(rd // 2, dtype=torch.float64, device=x.device)
    freq = torch.exp(i * (-2.0 / rd * math.log(case["base"])))
    axis = _axis_of_pairs(case)
    ang = torch.stack([pos[axis[j]].double() * freq[j] for j in range(rd // 2)], -1)[:, None]
    turn = torch.polar(torch.full_like(ang, case["scale"]), ang)
    head = x[..., :rd]
    if case["style"] == "halves":
        z = torch.complex(head[..., :rd // 2], head[..., rd // 2:]) * turn
        head = torch.cat([z.real, z.imag], -1)
    else:
        z = torch.complex(head[..., 0::2], head[..., 1::2]) * turn
        head = torch.view_as_real(z).reshape(head.shape)
    return torch.cat([head, x[..., rd:]], -1)


def exact(case, seed):
    st = _inputs(case, seed)
    if case["kind"] == "copy":
        out = []
        for cache in (st["kc"].double(), st["vc"].double()):
            src, dst = st["pairs"].long().unbind(1)
            out.append(cache.index_copy(0, dst, cache.index_select(0, src)))
        return tuple(out)
    st["case"] = case
    q, k, v = (x.double() for x in _heads(st))
    wq, wk = (None if w is None else w.double() for w in (st["wq"], st["wk"]))
    if case["kind"] == "backward":
        leaves = [x.clone().requires_grad_() for x in (q, k, wq, wk) if x is not None]
        zq = _exact_rows(leaves[0], leaves[2] if case["norm"] else None, st["pos"], case)
        zk = _exact_rows(leaves[1], leaves[3] if case["norm"] else None, st["pos"], case)
        return torch.autograd.grad([zq, zk], leaves, [st["gq"].double(), st["gk"].double()])
    zq, zk = _exact_rows(q, wq, st["pos"], case), _exact_rows(k, wk, st["pos"], case)
    if case["kind"] == "forward":
        return zq, zk
    kc, vc = st["kc"].double(), st["vc"].double()
    blk, t = st["slots"].long().unbind(1)
    place = torch.tensor([0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15], device=DEVICE)[t]
    n, hkv, d = zk.shape
    kc.permute(0, 3, 1, 2, 4).index_put_((blk, place), zk.reshape(n, hkv, d // 8, 8))
    vc.permute(0, 3, 1, 2).index_put_((blk, t), v)
    return zq, kc, vc

"""Cases and bounds shared by the tests of 8-bit caches.

Bounds of the attention on the values that the codes stand for (exact in bf16):

bf16 queries.  A probability is rounded to bf16 (2^-8 of itself at most) before
the product with V, and the row sum adds rounded or unrounded ones: the quotient
is off by 2 * 2^-8 * A, A = sum p |v|, at most.  The result is rounded once more
(2^-8 of itself), and the LSE off by 2^-8.  Besides, in fp32 (u = 2^-24): a score
adds d products (off by d u of scale * sum |q k|, at most `mag`) and is scaled
(2 u), its exponential is off by 2 u and by the score's error, the sums of n
terms by n u, a merge of split partials by 4 u.

fp32 queries: the same without the roundings to bf16.

Underflow: an exponential (relative to one of at least 2^-8) and its product with
a scale are 0 below 2^-126, so that a term of the sum can lose 2^-126 of |v| and of
its code (at most 448), 2^8 times that of the quotient.
"""
import math

import numpy as np
import torch

import oracle
from oracle import dense as od
from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from _rotary import check, f64

U = 2.0 ** -24


def on_gpu(cache):
    k, v, s = (torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in cache)
    return k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn), s.view(torch.float8_e8m0fnu)


def on_host(cache):
    return tuple(x.view(torch.uint8).cpu().numpy() for x in cache)


def rows(shape, seed, spread=1.0):
    """Rows of values, some larger than others by a power of two."""
    rng = np.random.default_rng([seed, 5])
    return rng.standard_normal(shape) * np.exp2(spread * rng.integers(-3, 2, size=shape[:-1] + (1,)))


def tolerance(nodes, q, k, v, scale, hq, hkv, O, L, f32, **kw):
    G = hq // hkv
    A, _ = oracle.tree_attention(nodes, q, k, np.abs(v), scale, hq, hkv, **kw)
    d, n = k.shape[-1], k.shape[0]
    mag = scale * d * max(np.abs(q[:, h]).max(initial=0) * np.abs(k[:, h // G]).max(initial=0) for h in range(hq))
    e = (d * mag + np.abs(L).max(initial=0) + n + 16) * U if len(O) else 0.0
    lost = n * 2.0 ** -118 * (np.abs(v).max(initial=0) + 448)
    if f32:
        return 2 * e * A + 4 * U * np.abs(O) + lost, e + 4 * U * np.abs(L)
    t = (2 * 2.0 ** -8 * 1.02 + 2 * e) * A + lost
    return t + 2.0 ** -8 * (np.abs(O) + t), 2.0 ** -8 * 1.02 + e + 4 * U * np.abs(L)


class Case:
    """A decode step over an 8-bit cache: nodes (parent, fork, len, q_len), rows
    drawn from `seed`, unused slots and blocks full of anything."""

    def __init__(self, nodes, hq, hkv, d, dtype, seed, extra=7, spread=1.0, k=None, v=None, **plan):
        self.nodes, self.hq, self.hkv, self.d, self.f32 = [tuple(n) for n in nodes], hq, hkv, d, dtype == "f32"
        self.scale = 1 / math.sqrt(d)
        T, self.nq = sum(n[2] for n in self.nodes), sum(n[3] for n in self.nodes)
        nb = sum(-(-n[2] // 16) for n in self.nodes)
        k = rows((T, hkv, d), 3 * seed + 1, spread) if k is None else k
        v = rows((T, hkv, d), 3 * seed + 2, spread) if v is None else v
        self.ids = np.random.default_rng([seed, 6]).permutation(nb + extra)[:nb].astype(np.int32)
        self.cache = orc.empty(nb + extra, hkv, d, seed)
        blk, slot = od.paged_slots(self.nodes, self.ids, 16)
        orc.write(self.cache, blk, slot, k, v)
        self.k, self.v = orc.read(self.cache, blk, slot)
        q = torch.from_numpy(np.random.default_rng([seed, 8]).standard_normal((self.nq, hq, d))).float()
        self.q = (q if self.f32 else q.bfloat16()).cuda()
        self.table = torch.from_numpy(self.ids).cuda()
        segs = pa.segments_layout(self.nodes, 16)
        self.plan = pa.TreePlan(segs, hq, hkv, d, dtype + "_e4m3", 16, num_kv_rows=nb + extra, num_q_rows=self.nq,
                                block_table_host=self.ids, **plan)
        self.gpu = on_gpu(self.cache)
        print(f"[case] decode e4m3 {dtype} T={T} nq={self.nq} Hq={hq} Hkv={hkv} d={d} seed={seed} "
              f"work={len(self.plan.export()['work'])}", flush=True)

    def run(self, call=None, **kw):
        k, v, s = self.gpu
        out = (call or pa.branch_decode)(self.q, k, v, self.table, self.plan, scales=s, **kw)
        torch.cuda.synchronize()
        return out

    def reference(self, q=None):
        """O, LSE and their bounds, from the rows that are finite."""
        q64 = f64(self.q if q is None else q)
        kw = {"q_off": od.canonical_layout(self.nodes, 0)[1]}
        O, L = oracle.tree_attention(self.nodes, q64, self.k, self.v, self.scale, self.hq, self.hkv, **kw)
        return (O, L) + tolerance(self.nodes, q64, self.k, self.v, self.scale, self.hq, self.hkv, O, L, self.f32, **kw)

    def check(self, out, q=None):
        O, L, tol, ltol = self.reference(q)
        check("O", out[0], O, tol)
        check("LSE", out[1], L, np.broadcast_to(ltol, L.shape))

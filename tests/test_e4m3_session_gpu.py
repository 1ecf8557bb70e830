"""8-bit caches as they are served: a session whose rows are quantised as they
are appended, streams cloned, truncated and closed, the pool compacted, resized
and moved, and a page's prefix handed over from a bf16 cache."""
import math

import numpy as np
import pytest
import torch

import oracle
from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from _e4m3 import on_gpu, on_host, tolerance
from _rotary import Setup, check, f64, k_block_view, normal, positions, v_block_view

pytestmark = pytest.mark.gpu


class Server:
    """A session and the test's own record of every stream's raw rows."""

    def __init__(self, hq, hkv, d, dtype, blocks, style="halves"):
        self.hq, self.hkv, self.d, self.dtype = hq, hkv, d, dtype
        self.st = Setup(d, dtype, style=style, base=1e6)
        self.cache = on_gpu(orc.empty(blocks, hkv, d, 1))
        table = torch.full((1024,), -1, dtype=torch.int32, device="cuda")
        self.s = pa.DecodeSession(hq, hkv, d, blocks, dtype + "_e4m3", self.cache[0], self.cache[1], table, scales=self.cache[2])
        self.wq, self.wk = normal((d,), 1, dtype), normal((d,), 2, dtype)
        self.rows = {}  # stream -> (k [len, Hkv, d] raw, v, positions [3, len])
        self.seed = 10

    def open(self, parent=-1, fork=0):
        i = self.s.open(parent, fork)
        z = normal((0, self.hkv, self.d), 0, self.dtype)
        self.rows[i] = (z, z, torch.empty((3, 0), dtype=torch.int32, device="cuda"))
        return i

    def cut(self, i, n):
        k, v, p = self.rows[i]
        return k[:n], v[:n], p[:, :n]

    def clone(self, i, n=None):
        c = self.s.clone(i, n)
        self.rows[c] = self.cut(i, len(self.rows[i][0]) if n is None else n)
        return c

    def truncate(self, i, n):
        self.s.truncate(i, n)
        self.rows[i] = self.cut(i, n)

    def values(self, view):
        """The kept streams' rows as the cache holds them: V's exactly, K's within its rotation's error and a rounding."""
        cache, ks, vs = on_host(self.cache), [], []
        for i, g in zip(view["seg_id"], view["seg"]):
            K, V, P = self.rows[int(i)]
            t = np.arange(int(g["len"]))
            assert len(K) == len(t)
            blk = view["block_table"][int(g["kv_off"]) + t // 16]
            k, v = orc.read(cache, blk, t % 16)
            assert (v == orc.decode(*orc.encode(f64(V)))).all()
            if len(t):
                z, tol = self.st.forward(K, P, self.wk)
                tol = tol + np.maximum(2.0 ** -4 * np.abs(z), 2.0 ** -9 / 448 * np.abs(z).max(-1, keepdims=True)) * (1 + 2.0 ** -7)
                assert (np.abs(k - z) <= tol).all()
            ks.append(k)
            vs.append(v)
        return np.concatenate(ks), np.concatenate(vs)

    def step(self, n_new=None, n_query=None, rotary=True, **kw):
        nk, nq, _ = self.s.prepare(n_new, n_query)
        view, copies = self.s.view(), self.s.copies()
        self.seed += 10
        x = normal((max(nk, 1), self.hq + 2 * self.hkv, self.d), self.seed, self.dtype, spread=2.0)[:nk]
        q, k, v = x[:, :self.hq], x[:, self.hq:self.hq + self.hkv], x[:, self.hq + self.hkv:]
        pos = positions(3, nk, self.seed + 1, 2000)
        at = []
        for i, a, b, qa, qb in zip(view["row_id"], view["new_off"], view["new_off"][1:], view["q_off"], view["q_off"][1:]):
            ko, vo, po = self.rows[int(i)]
            self.rows[int(i)] = (torch.cat([ko, k[a:b]]), torch.cat([vo, v[a:b]]), torch.cat([po, pos[:, a:b]], 1))
            at += range(b - (qb - qa), b)
        q, qpos = q[at].contiguous(), pos[:, at].contiguous()
        print(f"[case] e4m3 step of {nk} rows, {nq} queries, copies {[len(c) for c in copies]}", flush=True)
        if rotary:
            rot = torch.empty_like(q)
            o, lse = self.s.launch_rotary(q, k, v, pos, self.st.handle, self.wq, self.wk, q_positions=qpos, q_rot=rot, **kw)
        else:  # rows that are rotated already
            zk, rot = (pa.rotary_fwd(a, None, p, self.st.handle, w)[0] for a, p, w in ((k, pos, self.wk), (q, qpos, self.wq)))
            o, lse = self.s.launch(rot, zk, v.contiguous(), **kw)
        torch.cuda.synchronize()
        K, V = self.values(view)
        if nq:
            check("q", rot, *self.st.forward(q, qpos, self.wq))
            nodes = [(int(g["parent"]), int(g["fork"]), int(g["len"]), int(g["q_len"])) for g in view["seg"]]
            scale, z = 1 / math.sqrt(self.d), f64(rot)
            O, L = oracle.tree_attention(nodes, z, K, V, scale, self.hq, self.hkv)
            tol, ltol = tolerance(nodes, z, K, V, scale, self.hq, self.hkv, O, L, self.dtype == "f32")
            check("O", o, O, tol)
            check("LSE", lse, L, np.broadcast_to(ltol, L.shape))
        return [len(c) for c in copies]


@pytest.mark.parametrize("dtype,hq,hkv,d,style,rotary", [("bf16", 8, 2, 128, "halves", True), ("f32", 4, 2, 64, "pairs", True),
                                                         ("bf16", 8, 2, 64, "halves", False), ("f32", 3, 3, 128, "halves", False)])
def test_a_served_page(dtype, hq, hkv, d, style, rotary):
    """(Rows that are rotated already are rounded to their dtype before they are quantised: st.forward's bound.)"""
    s = Server(hq, hkv, d, dtype, 60, style)
    kw = {"rotary": rotary}
    root, other = s.open(), s.open()
    s.step([75, 33], [0, 0], **kw)                 # two prefixes
    lay = s.open(root, 75)
    second = s.open(other, 33)
    s.s.close(root), s.s.close(other)
    s.step([21, 5], [21, 5], **kw)
    a = s.open(lay, 10)
    b = s.open(lay, 21)
    s.step([1, 1, 7, 12], [1, 1, 3, 12], **kw)
    c = s.clone(b)
    e = s.clone(b, 9)
    assert s.step(**kw) == [2]                      # b and c copy the block that e keeps
    s.truncate(a, 2)
    s.s.close(second)
    moves = s.s.compact()
    assert moves > 0
    f = s.clone(c)
    copies = s.step(**kw)
    assert len(copies) == 2 and copies[0] >= moves
    kept = 60 - s.s.view()["free_blocks"]
    s.cache = tuple(x[:kept + 4] for x in s.cache)
    s.s.resize(kept + 4, *s.cache[:2], scales=s.cache[2])
    s.step(**kw)
    old = kept + 4
    ids = np.stack([np.arange(old), np.arange(old)], 1).astype(np.int32)
    new = on_gpu(orc.empty(80, hkv, d, 5))
    pa.cache_copy_blocks(*s.cache[:2], torch.from_numpy(ids).cuda(), *new[:2], pairs_host=ids, scales=s.cache[2], scales_dst=new[2])
    s.s.resize(80, *new[:2], scales=new[2])
    s.cache = new
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    s.step([40, 1, 0, 1, 30, 1], [40, 1, 0, 1, 2, 1], stream=side, **kw)
    for i in (lay, a, b, c, e, f):
        s.s.close(i)
    assert s.s.view()["free_blocks"] == 80


def test_a_prefix_handed_over():
    """Prefilled into a bf16 cache, quantised into the pool's blocks, decoded from there; read back at the end."""
    hq, hkv, d, n = 8, 2, 128, 101
    st = Setup(d, "bf16", base=1e6)
    k, v, pos = normal((n, hkv, d), 1, "bf16"), normal((n, hkv, d), 2, "bf16"), positions(3, n, 3)
    kc, vc = torch.zeros((9, hkv, 16, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((9, hkv, d, 16), dtype=torch.bfloat16, device="cuda")
    t = np.arange(n)
    slots = torch.from_numpy(np.stack([t // 16 + 1, t % 16], 1).astype(np.int32)).cuda()
    pa.rotary_append(None, k, v, pos, slots, kc, vc, st.handle)
    s = Server(hq, hkv, d, "bf16", 40)
    root = s.s.open()
    s.s.prepare([n], [0])
    view = s.s.view()
    s.s.commit()  # (the caller writes the rows and the table itself)
    ids = view["block_table"][int(view["seg"]["kv_off"][0]) + np.arange(7)]
    pairs = np.stack([np.arange(7) + 1, ids], 1).astype(np.int32)
    print("[case] prefix handed over", flush=True)
    pa.cache_quantize(kc, vc, *s.cache, pairs=torch.from_numpy(pairs).cuda(), pairs_host=pairs)
    s.s.block_table[torch.from_numpy(view["patch"][:, 0].astype(np.int64)).cuda()] = torch.from_numpy(view["patch"][:, 1].copy()).cuda()
    lay = s.s.open(root, n)
    s.s.close(root)
    nk, nq, _ = s.s.prepare([3], [3])
    view = s.s.view()
    x = normal((3, hq + 2 * hkv, d), 5, "bf16")
    rot = torch.empty((3, hq, d), dtype=torch.bfloat16, device="cuda")
    o, lse = s.s.launch_rotary(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], positions(3, 3, 6), st.handle, q_rot=rot)
    torch.cuda.synchronize()
    cache = on_host(s.cache)
    kv = []
    for g in view["seg"]:
        t = np.arange(int(g["len"]))
        kv.append(orc.read(cache, view["block_table"][int(g["kv_off"]) + t // 16], t % 16))
    K, V = (np.concatenate(p) for p in zip(*kv))
    for got, rows in ((K, k_block_view(kc)), (V, v_block_view(vc))):
        want = orc.decode(*orc.encode(f64(rows[1:8].transpose(1, 2).reshape(-1, hkv, d)[:n])))
        assert (got[:n] == want).all()
    nodes, z = [(int(g["parent"]), int(g["fork"]), int(g["len"]), int(g["q_len"])) for g in view["seg"]], f64(rot)
    O, L = oracle.tree_attention(nodes, z, K, V, 1 / math.sqrt(d), hq, hkv)
    tol, ltol = tolerance(nodes, z, K, V, 1 / math.sqrt(d), hq, hkv, O, L, False)
    check("O", o, O, tol)
    check("LSE", lse, L, np.broadcast_to(ltol, L.shape))
    back_k, back_v = torch.zeros_like(kc), torch.zeros_like(vc)
    pa.cache_dequantize(*s.cache, back_k, back_v, pairs=torch.from_numpy(pairs[:, ::-1].copy()).cuda())
    assert (f64(k_block_view(back_k)[1:8].transpose(1, 2).reshape(-1, hkv, d)[:n]) == K[:n]).all()
    s.s.close(lay)


def test_captured_together():
    """A layer's append and its attention in one graph, replayed on new rows with eager work between."""
    hq, hkv, d = 8, 2, 128
    s = Server(hq, hkv, d, "bf16", 20)
    nodes = [(-1, 0, 50, 0), (0, 50, 30, 1), (1, 17, 21, 1)]
    segs = pa.segments_layout(nodes, 16)
    ids = np.random.default_rng(1).permutation(20)[:8].astype(np.int32)
    plan = pa.TreePlan(segs, hq, hkv, d, "bf16_e4m3", 16, num_kv_rows=20, num_q_rows=2, block_table_host=ids)
    table, ws = torch.from_numpy(ids).cuda(), plan.workspace(torch.device("cuda", 0))
    before = orc.empty(20, hkv, d, 3)
    before[0][(before[0] & 127) == 127] = 1
    before[1][(before[1] & 127) == 127] = 1
    before[2][:] = np.clip(before[2], 120, 128)
    cache = on_gpu(before)
    slots = torch.tensor([[int(ids[4 + 29 // 16]), 29 % 16], [int(ids[6 + 20 // 16]), 20 % 16]], dtype=torch.int32, device="cuda")
    x, pos = normal((2, hq + 2 * hkv, d), 1, "bf16"), positions(3, 2, 2)
    q = torch.empty((2, hq, d), dtype=torch.bfloat16, device="cuda")
    o, lse = torch.empty_like(q), torch.empty((2, hq), device="cuda")

    def layer():
        pa.rotary_append(x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], pos, slots, *cache[:2], s.st.handle, s.wq, s.wk, q_out=q,
                         scales=cache[2])
        pa.branch_decode_resident(q, cache[0], cache[1], table, plan, o, lse, ws, scales=cache[2])
    pa.plan_upload(plan, ws)
    layer()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in range(4):
        print("[case] captured layer", seed, flush=True)
        x.copy_(normal(x.shape, seed + 20, "bf16"))
        pos.copy_(positions(3, 2, seed + 30))
        o.fill_(7), lse.fill_(7), q.fill_(7)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (q, o, lse)] + [t.clone() for t in on_gpu(on_host(cache))]
        layer()
        torch.cuda.synchronize()
        for a, b in zip(got, (q, o, lse, *cache)):
            assert torch.equal(a.view(torch.uint8) if a.element_size() == 1 else a, b.view(torch.uint8) if b.element_size() == 1 else b)
        host = on_host(cache)
        t = [np.arange(n[2]) for n in nodes]
        kv = [orc.read(host, ids[off + i // 16], i % 16) for off, i in zip((0, 4, 6), t)]
        K, V = (np.concatenate(p) for p in zip(*kv))
        O, L = oracle.tree_attention(nodes, f64(q), K, V, 1 / math.sqrt(d), hq, hkv)
        tol, ltol = tolerance(nodes, f64(q), K, V, 1 / math.sqrt(d), hq, hkv, O, L, False)
        check("O", o, O, tol)
        check("LSE", lse, L, np.broadcast_to(ltol, L.shape))


def test_session_refusals():
    k, v, sc = pa.empty_cache_e4m3(8, 2, 64, "cuda")
    table = torch.full((64,), -1, dtype=torch.int32, device="cuda")
    for args, kw in [((4, 2, 64, 8, "bf16_e4m3", k, v, table), {}), ((4, 2, 64, 8, "bf16", k, v, table), {"scales": sc}),
                     ((4, 2, 64, 7, "bf16_e4m3", k, v, table), {"scales": sc}), ((4, 2, 64, 8, "bf16_e4m3"), {"scales": sc})]:
        with pytest.raises((ValueError, TypeError)):
            pa.DecodeSession(*args, **kw)
    s = pa.DecodeSession(4, 2, 64, 8, "bf16_e4m3", k, v, table, scales=sc)
    with pytest.raises(ValueError):
        s.resize(4, k[:4], v[:4])
    s.open()
    s.prepare([2], [2])
    x = normal((2, 4, 64), 1, "bf16")
    with pytest.raises(TypeError):
        s.launch(x.float(), x[:, :2].float().contiguous(), x[:, :2].float().contiguous())
    with pytest.raises(TypeError, match="f32"):
        s.launch_rotary(x, x[:, :2], x[:, :2], positions(1, 2, 1), pa.Rotary(64, "f32"))
    s.launch(x, x[:, :2].contiguous(), x[:, :2].contiguous())

"""Decode steps over 8-bit caches against the oracle's attention on the values
that the codes stand for."""
import numpy as np
import pytest
import torch

from oracle import dense as od
from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from _e4m3 import Case, rows
from _rotary import f64

pytestmark = pytest.mark.gpu

# (parent, fork, length, queries)
TREES = {
    "one token": [(-1, 0, 1, 1)],
    "one stream": [(-1, 0, 77, 1)],
    "every query": [(-1, 0, 33, 33)],
    "a page": [(-1, 0, 300, 0), (0, 300, 41, 1), (1, 3, 20, 1), (1, 17, 64, 1), (1, 40, 129, 1)],
    "block edges": [(-1, 0, 64, 0), (0, 64, 16, 1), (1, 15, 1, 1), (1, 0, 16, 1), (1, 16, 17, 1), (1, 1, 48, 1), (1, 8, 65, 1)],
    "forks of nothing": [(-1, 0, 100, 0), (0, 0, 5, 2), (0, 1, 70, 3), (2, 0, 9, 9)],
    "residual prefill": [(-1, 0, 130, 0), (0, 130, 50, 1), (1, 10, 8, 8), (1, 49, 8, 8), (1, 33, 40, 40)],
    "deep": [(-1, 0, 70, 1), (0, 35, 66, 2), (1, 64, 30, 3), (2, 29, 100, 1), (3, 99, 17, 17)],
    "two pages": [(-1, 0, 90, 1), (0, 80, 20, 1), (-1, 0, 7, 0), (2, 7, 31, 1), (3, 30, 250, 1), (3, 2, 3, 3)],
    "nothing to do": [(-1, 0, 40, 0), (0, 40, 9, 0)],
}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 1, 64), (14, 2, 64), (3, 3, 128), (64, 1, 128)])
@pytest.mark.parametrize("tree", TREES)
def test_trees(tree, hq, hkv, d, dtype):
    c = Case(TREES[tree], hq, hkv, d, dtype, seed=len(tree))
    c.check(c.run())


def big_page(prefix, stream, lengths, seed):
    rng = np.random.default_rng([seed, 1])
    forks = np.sort(rng.integers(1, stream, size=len(lengths)))
    return [(-1, 0, prefix, 0), (0, prefix, stream, 1)] + [(1, int(f), int(n), 1) for f, n in zip(forks, lengths)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (28, 4, 64)])
def test_a_large_page(hq, hkv, d, dtype):
    """Many columns, split keys, ragged tails."""
    c = Case(big_page(1501, 203, np.random.default_rng(2).integers(1, 700, size=21), 1), hq, hkv, d, dtype, seed=5)
    c.check(c.run())


@pytest.mark.parametrize("chunk", [64, 128, 1024])
def test_chunks(chunk):
    c = Case(big_page(700, 99, [1, 64, 65, 300, 513], 2), 8, 2, 128, "bf16", seed=6, max_chunk_keys=chunk)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_very_different_size(dtype):
    """Scales over 2^80, largest scores of hundreds; rows of zeros, rows below the smallest scale."""
    nodes = big_page(260, 40, [30, 70, 1], 3)
    T = sum(n[2] for n in nodes)
    rng = np.random.default_rng(9)
    k = rows((T, 2, 64), 1) * np.exp2(rng.integers(-40, 6, size=(T, 2, 1)))
    v = rows((T, 2, 64), 2) * np.exp2(rng.integers(-40, 40, size=(T, 2, 1)))
    k[5], v[6], v[100], k[101] = 0, 0, 1e-30, 1e-30
    c = Case(nodes, 8, 2, 64, dtype, seed=7, k=k, v=v)
    c.check(c.run())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 1, 64)])
@pytest.mark.parametrize("what", ["k", "v"])
def test_a_row_that_is_nan_reaches_the_queries_that_see_it(what, hq, hkv, d, dtype):
    """Tokens of the prefix's last rows, of the stream between forks, of a branch: NaN for those who see them
    (in that KV head), the others as without them."""
    nodes = [(-1, 0, 140, 0), (0, 137, 60, 2), (1, 5, 40, 1), (1, 33, 90, 3), (0, 140, 20, 1), (1, 59, 70, 1)]
    T = sum(n[2] for n in nodes)
    bad = {"k": [138, 140 + 20, 140 + 60 + 40 + 88], "v": [139, 140 + 32, 140 + 60 + 40 + 89]}[what]
    k, v = rows((T, hkv, d), 1), rows((T, hkv, d), 2)
    x = k if what == "k" else v
    for i, t in enumerate(bad):
        x[t, hkv - 1, 7 * i] = [np.nan, np.inf, -np.inf][i]
    c = Case(nodes, hq, hkv, d, dtype, seed=8, k=k, v=v)
    blk, slot = od.paged_slots(c.nodes, c.ids, 16)
    assert (c.cache[2][blk, :, "kv".index(what), slot][bad, hkv - 1] == 255).all()
    o, lse = c.run()
    start = np.cumsum([0] + [n[2] for n in nodes])
    sees = np.zeros((c.nq, hq), bool)
    row = 0
    for s, (_, _, n, ql) in enumerate(nodes):
        for p in range(n - ql, n):
            for t, count in od.visible_counts(c.nodes, s, p).items():
                if any(start[t] <= b < start[t] + count for b in bad):
                    sees[row, (hkv - 1) * (hq // hkv):] = True
            row += 1
    assert sees.any() and not sees.all()
    assert np.isnan(f64(lse)[sees]).all() and np.isnan(f64(o)[sees]).all()
    x[bad, hkv - 1] = 0  # (nobody else sees those rows)
    orc.write(c.cache, blk, slot, k, v)
    c.k, c.v = orc.read(c.cache, blk, slot)
    O, L, tol, ltol = c.reference()
    assert (np.abs(f64(o) - O)[~sees] <= tol[~sees]).all()
    assert (np.abs(f64(lse) - L)[~sees] <= np.broadcast_to(ltol, L.shape)[~sees]).all()


def test_the_same_as_on_the_values_read_back():
    """A bf16 step on the dequantised cache and this one agree within both bounds."""
    c = Case(big_page(400, 77, [50, 3, 200], 4), 8, 2, 128, "bf16", seed=9, extra=0)
    o, lse = c.run()
    kc, vc = pa.cache_dequantize(*c.gpu)
    # (slots that no token is in hold anything, NaN among it: the bf16 step does not use them)
    plan = pa.TreePlan(pa.segments_layout(c.nodes, 16), 8, 2, 128, "bf16", 16, num_kv_rows=len(vc), num_q_rows=c.nq,
                       block_table_host=c.ids)
    o2, lse2 = pa.branch_decode(c.q, kc, vc, c.table, plan)
    _, _, tol, ltol = c.reference()
    assert (np.abs(f64(o) - f64(o2)) <= 2 * tol).all() and (np.abs(f64(lse) - f64(lse2)) <= 2 * ltol).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_entry_points_agree_bit_for_bit(dtype):
    """Own workspace, given buffers (a repeated call too), no allocation, resident, another stream, a captured
    graph replayed on new queries, keys written between replays."""
    c = Case(big_page(333, 50, [90, 17, 260, 1], 5), 8, 2, 64, dtype, seed=10)
    o, lse = c.run()
    c.check((o, lse))
    ws = c.plan.workspace(c.q.device)
    for call, kw in ((pa.branch_decode, {"workspace": ws}), (pa.branch_decode, {"workspace": ws}), (pa.branch_decode_no_alloc, {})):
        o2, l2 = torch.full_like(o, 3), torch.full_like(lse, 3)
        for _ in range(2):
            c.run(call, out=o2, lse=l2, **kw)
        assert torch.equal(o, o2) and torch.equal(lse, l2)
    pa.plan_upload(c.plan, ws)
    o2, l2 = torch.empty_like(o), torch.empty_like(lse)
    for _ in range(3):
        o2.fill_(5)
        c.run(pa.branch_decode_resident, out=o2, lse=l2, workspace=ws)
        assert torch.equal(o, o2) and torch.equal(lse, l2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    o3, l3 = c.run(stream=side)
    assert torch.equal(o, o3) and torch.equal(lse, l3)
    k, v, s = c.gpu
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.branch_decode_resident(c.q, k, v, c.table, c.plan, o2, l2, ws, scales=s)
    for seed in range(3):
        q = torch.randn(c.q.shape, generator=torch.Generator().manual_seed(seed)).to(c.q.dtype)
        c.q.copy_(q)
        graph.replay()
        torch.cuda.synchronize()
        got = o2.clone(), l2.clone()
        eager = c.run()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        c.check(got)


def test_rows_behind_the_last_query_stay():
    """Outputs larger than the plan's queries would be refused by shape elsewhere; rows of segments without queries
    and the caches are as they were."""
    c = Case(TREES["a page"], 8, 2, 128, "bf16", seed=11)
    before = [x.clone().view(torch.uint8) for x in c.gpu]
    big = torch.full((c.nq + 5, 8, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((c.nq + 5, 8), 9.0, device="cuda")
    c.run(out=big[:c.nq], lse=lse[:c.nq], workspace=c.plan.workspace(c.q.device))
    assert (big[c.nq:] == 9).all() and (lse[c.nq:] == 9).all()
    assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, c.gpu))


def test_blocks_behind_two_gigabytes():
    """Blocks at the far end of a pool whose codes pass 2^32 bytes."""
    hkv, d = 2, 128
    blocks = (1 << 32) // (hkv * d * 16) + 64
    if torch.cuda.mem_get_info()[0] < 3 * blocks * hkv * d * 16:
        pytest.skip("not enough memory")
    c = Case([(-1, 0, 200, 0), (0, 200, 30, 1), (1, 9, 70, 1)], 8, hkv, d, "bf16", seed=12)
    far = pa.empty_cache_e4m3(blocks, hkv, d, "cuda")
    n = len(c.cache[1])
    for x, y in zip(far, c.gpu):
        x.view(torch.uint8)[:1] = 0
        x.view(torch.uint8)[-n:] = y.view(torch.uint8)
    ids = (c.ids + blocks - n).astype(np.int32)
    plan = pa.TreePlan(pa.segments_layout(c.nodes, 16), 8, hkv, d, "bf16_e4m3", 16, num_kv_rows=blocks, num_q_rows=c.nq,
                       block_table_host=ids)
    print("[case] decode far blocks", flush=True)
    c.check(pa.branch_decode(c.q, far[0], far[1], torch.from_numpy(ids).cuda(), plan, scales=far[2]))


def test_refusals():
    c = Case(TREES["a page"], 8, 2, 64, "bf16", seed=13)
    k, v, s = c.gpu
    nb = len(v)
    bf = pa.TreePlan(pa.segments_layout(c.nodes, 16), 8, 2, 64, "bf16", 16, num_kv_rows=nb, num_q_rows=c.nq, block_table_host=c.ids)
    kc, vc = pa.cache_dequantize(k, v, s)
    for plan, args, kw in ((c.plan, (k, v), {}), (bf, (kc, vc), {"scales": s}), (bf, (k, v), {"scales": s}), (c.plan, (kc, vc), {"scales": s}),
                           (c.plan, (v, k), {"scales": s}), (c.plan, (k, v), {"scales": s.view(torch.uint8)}),
                           (c.plan, (k[:, :1].contiguous(), v[:, :1].contiguous()), {"scales": s[:, :1].contiguous()})):
        with pytest.raises((ValueError, TypeError)):
            pa.branch_decode(c.q, *args, c.table, plan, **kw)
        with pytest.raises((ValueError, TypeError)):
            pa.branch_decode_no_alloc(c.q, *args, c.table, plan, torch.empty_like(c.q), torch.empty((c.nq, 8), device="cuda"), **kw)
    with pytest.raises(pa.PadocError):  # another pool than the plan's
        pa.branch_decode(c.q, k[1:].contiguous(), v[1:].contiguous(), c.table, c.plan, scales=s[1:].contiguous())
    with pytest.raises((ValueError, TypeError)):
        pa.branch_decode(c.q.float(), k, v, c.table, c.plan, scales=s)

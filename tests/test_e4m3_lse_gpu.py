"""LSE of decode steps over 8-bit caches: row sums add probabilities that are
not rounded to bf16.

Scores are 0 for every 16th key and ln p for the others, so that every tile's
maximum is 0 and every other probability is p = 2^-j (1 + f 2^-7), f in [0.35,
0.45]: bf16 would hold 2^-j, and a sum of rounded ones would be off by
0.35 2^-7 of all of them, one way.

Bound (u = 2^-24): a score adds d products (d u of scale * sum |q k|) and is
scaled (2 u of it), its exponential is off by 2 u and by the score's error, the
sums of n terms by n u, a merge of partials by 4 u, the logarithm's result by
4 u of itself.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import dense as od
from _e4m3 import U, Case
from _rotary import check, f64

pytestmark = pytest.mark.gpu

TREES = {
    "shared": [(-1, 0, 1490, 0), (0, 1490, 99, 1)] + [(1, 9 + 4 * i, 1, 1) for i in range(20)],
    "private": [(-1, 0, 16, 0), (0, 16, 16, 1)] + [(1, 15, 300 + 37 * i, 1) for i in range(5)],
    "both": [(-1, 0, 700, 0), (0, 700, 130, 1)] + [(1, 100 + i, 200 + 11 * i, 1) for i in range(12)],
}


def visible(c):
    """Per query row: the keys that it sees with a score of 0, and the others."""
    start, out = np.cumsum([0] + [n[2] for n in c.nodes]), []
    for s, (_, _, n, ql) in enumerate(c.nodes):
        for p in range(n - ql, n):
            rows = np.concatenate([start[t] + np.arange(count) for t, count in od.visible_counts(c.nodes, s, p).items()])
            out.append([(rows % 16 == 0).sum(), (rows % 16 != 0).sum()])
    return np.array(out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (4, 1, 64), (14, 2, 64)])
@pytest.mark.parametrize("tree", TREES)
def test_sums_of_unrounded_probabilities(tree, hq, hkv, d, dtype):
    nodes = TREES[tree]
    T = sum(n[2] for n in nodes)
    k = np.ones((T, hkv, d))
    k[::16] = 0
    c = Case(nodes, hq, hkv, d, dtype, seed=3, k=k)
    assert (c.k == k).all()  # (exact in 8 bits)
    work = c.plan.export()
    assert tree == "private" or work["n_work_shared"] > 0
    rng = np.random.default_rng(4)
    p = np.exp2(-rng.integers(1, 4, size=(c.nq, hq))) * (1 + rng.uniform(0.35, 0.45, size=(c.nq, hq)) * 2.0 ** -7)
    q = np.zeros((c.nq, hq, d), np.float32)
    rest = np.log(p) / c.scale
    for j in range(4):  # ln p / scale as a sum of numbers that are exact in bf16
        q[..., 17 * j] = torch.from_numpy(rest).bfloat16().float().numpy()
        rest = rest - q[..., 17 * j]
    c.q = torch.from_numpy(q).to(c.q.dtype).cuda()
    out = c.run()

    q64 = f64(c.q)
    assert (q64 == q).all()
    kw = {"q_off": od.canonical_layout(c.nodes, 0)[1]}
    _, L = oracle.tree_attention(c.nodes, q64, c.k, c.v, c.scale, hq, hkv, **kw)
    mag = c.scale * np.abs(q64).sum(-1).max()
    tol = ((d + 2) * mag + T + 16) * U + 4 * U * np.abs(L)
    check("LSE", out[1], L, tol)
    # (a sum of rounded ones would not pass)
    seen = visible(c)
    of = np.exp(c.scale * q64.sum(-1))
    assert (np.abs(np.log(seen[:, :1] + seen[:, 1:] * of) - L) <= 1e-9).all()
    rounded = np.log(seen[:, :1] + seen[:, 1:] * torch.from_numpy(of).bfloat16().double().numpy())
    assert (np.abs(rounded - L) > 3 * tol).all(), (np.abs(rounded - L) / tol).min()

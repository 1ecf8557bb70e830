"""Steps of many items over 8-bit caches give the same bits every time, whichever
wavefront takes an item, with other calls on the same buffers in between."""
import numpy as np
import pytest
import torch

from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from _e4m3 import Case, on_gpu
from _rotary import Setup, normal, positions

pytestmark = pytest.mark.gpu


def pages(n, prefix, stream, branches, longest):
    out = []
    for p in range(n):
        rng, at = np.random.default_rng([p, 3]), len(out)
        out += [(-1, 0, prefix, 0), (at, prefix, stream, 1)]
        forks, lengths = np.sort(rng.integers(1, stream, size=branches)), rng.integers(1, longest + 1, size=branches)
        out += [(at + 1, int(f), int(k), 1) for f, k in zip(forks, lengths)]
    return out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d", [(16, 2, 128), (28, 4, 64)])
def test_decode(hq, hkv, d, dtype):
    """600 private items and more, so that the queues of every XCD are taken from; the answers are those of the step's
    own inputs, not of the ones before."""
    c = Case(pages(12, 331, 77, 25, 400), hq, hkv, d, dtype, seed=21)
    q = c.q.clone()
    first = [x.clone() for x in c.run()]
    for seed in range(3):
        c.q.copy_(torch.randn(q.shape, generator=torch.Generator().manual_seed(seed)).to(q.dtype))
        other = c.run()
        assert not torch.equal(other[0], first[0])
        c.q.copy_(q)
        for a, b in zip(c.run(), first):
            assert torch.equal(a, b)


@pytest.mark.parametrize("dtype,n", [("bf16", 37), ("bf16", 7001), ("f32", 7001)])
def test_append(dtype, n):
    """Into caches that hold other rows before."""
    hkv, d = 2, 128
    st = Setup(d, dtype, base=1e6)
    x, y = (normal((n, 4 + 2 * hkv, d), s, dtype, spread=3.0) for s in (1, 2))
    wk, pos, blocks = normal((d,), 3, dtype), positions(3, n, 4), n // 16 + 9
    at = 5 + np.arange(n)
    slots = torch.from_numpy(np.stack([np.random.default_rng(6).permutation(blocks)[at // 16], at % 16], 1).astype(np.int32)).cuda()

    def run(gpu, x):
        q = pa.rotary_append(x[:, :4], x[:, 4:4 + hkv], x[:, 4 + hkv:], pos, slots, *gpu[:2], st.handle, None, wk, scales=gpu[2])
        return [q] + [t.view(torch.uint8).clone() for t in gpu]
    gpu = on_gpu(orc.empty(blocks, hkv, d, 7))
    first = run(gpu, x)
    for _ in range(3):
        run(gpu, y)
        assert all(torch.equal(a, b) for a, b in zip(run(gpu, x), first))

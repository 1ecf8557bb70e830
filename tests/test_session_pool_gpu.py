"""A session whose pool is given back whole and filled again."""
import pytest
import torch

import paper_2608_06146_amd as pa
from _rotary import normal

pytestmark = pytest.mark.gpu


def caches(nb):
    return (torch.zeros((nb, 2, 16, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((nb, 2, 128, 16), dtype=torch.bfloat16, device="cuda"))


def step(s, n, seed):
    i = s.open()
    q, k, v = normal((n, 8, 128), seed, "bf16"), normal((n, 2, 128), seed + 1, "bf16"), normal((n, 2, 128), seed + 2, "bf16")
    out = s.step(q, k, v, [n], [n])
    torch.cuda.synchronize()
    s.close(i)
    return out


def test_no_blocks_and_back():
    table = lambda: torch.zeros(256, dtype=torch.int32, device="cuda")  # noqa: E731
    kc, vc = caches(20)
    s, fresh = pa.DecodeSession(8, 2, 128, 20, "bf16", kc, vc, table()), pa.DecodeSession(8, 2, 128, 9, "bf16", *caches(9), table())
    step(s, 50, 1)
    for none in ((kc[:0], vc[:0]), caches(0)):
        s.resize(0, *none)
        s.prepare()
        assert all(t.numel() == 0 for t in s.launch(None, None, None))  # a step of no streams
        i = s.open()
        with pytest.raises(pa.PadocError, match="blocks"):
            s.prepare([1], [1])
        s.close(i)
        s.resize(9, *caches(9))
        assert all(torch.equal(a, b) for a, b in zip(step(s, 100, 7), step(fresh, 100, 7)))

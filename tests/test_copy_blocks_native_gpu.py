"""cache_copy_blocks as the native module calls it: pairs on the device alone."""
import numpy as np
import pytest
import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _rotary import normal

pytestmark = pytest.mark.gpu


@pytest.fixture
def taken(monkeypatch):
    """What the native call answered, call by call."""
    assert _lib.native_rows() is not None, "the native module is not built"
    native, answers = _lib.native_copy_blocks(), []

    def call(*a):
        answers.append(native(*a))
        return answers[-1]

    monkeypatch.setattr(pa, "_copy_blocks", call)
    return answers


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(64, 1), (64, 5), (128, 2), (128, 3)])
@pytest.mark.parametrize("n", [0, 1, 24, 301])
def test_copies(taken, dtype, d, hkv, n):
    print("[case]", dtype, d, hkv, n, flush=True)
    nb = 2 * n + 5
    kc, vc = normal((nb, hkv, d // 8, 16, 8), 1, dtype), normal((nb, hkv, d, 16), 2, dtype)
    ids = np.random.default_rng(n).permutation(nb)[:2 * n].reshape(-1, 2).astype(np.int32)
    pairs = np.concatenate([ids, np.array([[0, -1], [-1, 0], [nb, 1], [2, nb]], np.int32)])  # and some left out
    want = [c.clone() for c in (kc, vc)]
    for c in want:
        c[ids[:, 1]] = c[ids[:, 0]]
    out = pa.cache_copy_blocks(kc, vc, torch.from_numpy(pairs).cuda())
    assert taken == [0] and out[0] is kc and out[1] is vc
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_what_the_native_call_leaves(taken):
    """It answers nothing to arguments that are not in order, for which the
    Python form says what is wrong, and a status to what the library refuses."""
    kc, vc = normal((4, 2, 8, 16, 8), 1, "bf16"), normal((4, 2, 64, 16), 2, "bf16")
    pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    for k, v, p in ((kc.float(), vc, pairs), (kc, vc[:3], pairs), (kc, vc, pairs.long()), (kc, vc, pairs[0]), (kc.cpu(), vc, pairs)):
        with pytest.raises((ValueError, TypeError)):
            pa.cache_copy_blocks(k, v, p)
    assert taken == [None] * 5
    both = torch.zeros((4, 2, 64, 16), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(pa.PadocError, match="distinct"):
        pa.cache_copy_blocks(both.view(4, 2, 8, 16, 8), both, pairs)
    assert taken[5] == _lib.ERR_ARG

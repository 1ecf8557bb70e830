"""Outputs that the caller gives, where their memory is shared with another
tensor until one of the two is written: the other keeps its values."""
import pytest
import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _rotary import Setup, normal, positions

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["native", "python"])
def binding(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(_lib, "native_rows", lambda: None)
        monkeypatch.setattr(pa, "_copy_blocks", lambda *a: None)
    else:
        assert _lib.native_rows() is not None, "the native module is not built"


def lazily(t):
    """A clone that shares t's memory until one of them is written."""
    c = t._lazy_clone()
    assert torch._C._is_cow_tensor(c)
    return c


def test_a_lazy_clone_as_output():
    st, n, d = Setup(64, "bf16"), 40, 64
    q, k, w, pos = normal((n, 4, d), 1, "bf16"), normal((n, 2, d), 2, "bf16"), normal((d,), 3, "bf16"), positions(3, n, 4)
    want = pa.rotary_fwd(q, k, pos, st.handle, w, w)
    grads = pa.rotary_bwd(q, k, pos, st.handle, q, k, w, w)
    for call, given, outs in ((lambda a, b: pa.rotary_fwd(q, k, pos, st.handle, w, w, q_out=a, k_out=b), (q, k), want),
                              (lambda a, b: pa.rotary_bwd(q, k, pos, st.handle, q, k, w, w, dq=a, dk=b), (q, k), grads)):
        base = [torch.full_like(t, 5.0) for t in given]
        got = call(*map(lazily, base))
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
        assert all(bool((t == 5).all()) for t in base)
        base = [t.clone() for t in given]  # and in place of a clone: its sibling is read by nobody
        a, b = map(lazily, base)
        q, k = a, b
        got = call(a, b)
        q, k = given
        assert all(torch.equal(x, y) for x, y in zip(got, outs))
        assert all(torch.equal(x, y) for x, y in zip(base, given))


def test_lazy_clones_of_caches():
    st, n, d = Setup(64, "bf16"), 20, 64
    q, k, v, pos = normal((n, 4, d), 1, "bf16"), normal((n, 2, d), 2, "bf16"), normal((n, 2, d), 3, "bf16"), positions(3, n, 4)
    t = torch.arange(n, dtype=torch.int32)
    slots = torch.stack([t // 16, t % 16], 1).cuda()
    caches = torch.zeros((4, 2, d // 8, 16, 8), dtype=q.dtype, device="cuda"), torch.zeros((4, 2, d, 16), dtype=q.dtype, device="cuda")
    want = [c.clone() for c in caches]
    zq = pa.rotary_append(q, k, v, pos, slots, *want, st.handle)
    a, b = map(lazily, caches)
    out = torch.full_like(q, 5.0)
    got = pa.rotary_append(q, k, v, pos, slots, a, b, st.handle, q_out=lazily(out))
    assert torch.equal(got, zq) and torch.equal(a, want[0]) and torch.equal(b, want[1]) and bool((out == 5).all())
    assert not caches[0].any() and not caches[1].any()
    pairs = torch.tensor([[0, 3]], dtype=torch.int32, device="cuda")
    a, b = map(lazily, want)
    pa.cache_copy_blocks(a, b, pairs)
    assert torch.equal(a[3], want[0][0]) and torch.equal(b[3], want[1][0]) and not want[0][3].any() and not want[1][3].any()

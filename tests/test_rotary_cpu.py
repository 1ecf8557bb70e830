"""What the rotary and block-copy entry points refuse, before any HIP call
(addresses here are never read)."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib

A = 1 << 20  # an address


def heads(data=A, rs=256, hs=64):
    return [data, rs, hs]


def fwd(rot, n=4, hq=2, hkv=1, pos=A, pos_stride=0, q=None, k=None, qo=None, ko=None, wq=0, wk=0):
    a = [n, hq, hkv, pos, pos_stride, *(q or heads()), *(k or heads(2 * A)), *(qo or heads(3 * A)), *(ko or heads(4 * A)), wq, wk]
    return _lib.lib().padoc_rotary_fwd(rot and rot.handle, _lib.ROTARY_FWD_ARGS.pack(*a), None)


def bwd(rot, n=4, hq=2, hkv=1, pos=A, q=None, k=None, gq=None, gk=None, dq=None, dk=None, wq=0, wk=0, dwq=0, dwk=0, ws=None, nb=0):
    a = [n, hq, hkv, pos, 0, *(q or heads()), *(k or heads(2 * A)), *(gq or heads(5 * A)), *(gk or heads(6 * A)),
         *(dq or heads(3 * A)), *(dk or heads(4 * A)), wq, wk, dwq, dwk]
    return _lib.lib().padoc_rotary_bwd(rot.handle, _lib.ROTARY_BWD_ARGS.pack(*a), ws, nb, None)


def append(rot, n_q=4, n=4, hq=2, hkv=1, q_pos=0, pos=A, q=None, k=None, v=None, qo=None, slots=A, kc=A, vc=2 * A, nb=9, pos_stride=0):
    a = [n_q, n, hq, hkv, q_pos, 0, pos, pos_stride, *(q or heads()), *(k or heads(2 * A)), *(v or heads(3 * A)), *(qo or heads(4 * A)),
         0, 0, slots, kc, vc, nb]
    return _lib.lib().padoc_rotary_append(rot.handle, _lib.ROTARY_APPEND_ARGS.pack(*a), None)


def message():
    return _lib.lib().padoc_last_error().decode()


@pytest.fixture(scope="module")
def rot():
    return pa.Rotary(64, "bf16")


@pytest.fixture(scope="module")
def rot3():
    return pa.Rotary(64, "bf16", sections=(8, 12, 12))


def test_argument_sizes():
    """The packed arguments are the header's structs."""
    class Heads(C.Structure):
        _fields_ = [("data", C.c_void_p), ("row_stride", C.c_int64), ("head_stride", C.c_int64)]

    def size(*fields):
        return C.sizeof(type("S", (C.Structure,), {"_fields_": [(f"f{i}", t) for i, t in enumerate(fields)]}))
    i32, i64, p = C.c_int32, C.c_int64, C.c_void_p
    assert _lib.ROTARY_FWD_ARGS.size == size(i64, i32, i32, p, i64, *[Heads] * 4, p, p)
    assert _lib.ROTARY_BWD_ARGS.size == size(i64, i32, i32, p, i64, *[Heads] * 6, p, p, p, p)
    assert _lib.ROTARY_APPEND_ARGS.size == size(i64, i64, i32, i32, p, i64, p, i64, *[Heads] * 4, p, p, p, p, p, i64)


@pytest.mark.parametrize("kw,status", [
    (dict(head_dim=96), _lib.ERR_SHAPE), (dict(rotary_dim=0), _lib.ERR_SHAPE), (dict(rotary_dim=24), _lib.ERR_SHAPE),
    (dict(rotary_dim=144), _lib.ERR_SHAPE), (dict(base=0.0), _lib.ERR_ARG), (dict(base=float("inf")), _lib.ERR_ARG),
    (dict(base=float("nan")), _lib.ERR_ARG), (dict(base=1e-322), _lib.ERR_ARG), (dict(scale=float("nan")), _lib.ERR_ARG),
    (dict(eps=-1.0), _lib.ERR_ARG), (dict(eps=float("inf")), _lib.ERR_ARG),
    (dict(axis=[0] * 63 + [4]), _lib.ERR_SHAPE), (dict(axis=[0] * 63 + [-1]), _lib.ERR_BOUNDS),
    (dict(sections=(10, 10, 10, 10, 24)), _lib.ERR_SHAPE), (dict(n_axes=0), _lib.ERR_SHAPE),
    (dict(axis=[2] * 64, n_axes=2), _lib.ERR_BOUNDS), (dict(inv_freq=[0.0] * 63 + [float("inf")]), _lib.ERR_ARG)])
def test_handles_refused(kw, status):
    with pytest.raises(_lib.PadocError) as e:
        pa.Rotary(**{"head_dim": 128, **kw})
    assert e.value.status == status, str(e.value)


def test_handles_refused_in_python():
    for kw in (dict(style="neox"), dict(sections=(30, 30)), dict(axis=[0] * 3), dict(inv_freq=[1.0]),
               dict(sections=(32, 32), axis=[0] * 64)):
        with pytest.raises(ValueError):
            pa.Rotary(128, **kw)
    with pytest.raises(KeyError):
        pa.Rotary(128, "fp16")
    L = _lib.lib()
    h = C.c_void_p(5)
    assert L.padoc_rotary_create(None, C.byref(h)) == _lib.ERR_ARG and h.value is None
    d = _lib.RotaryDesc(128, 128, 1, 0, None, None, 1e4, 1.0, 1e-6, 7)
    assert L.padoc_rotary_create(C.byref(d), C.byref(h)) == _lib.ERR_DTYPE
    d = _lib.RotaryDesc(128, 128, 1, 2, None, None, 1e4, 1.0, 1e-6, 0)
    assert L.padoc_rotary_create(C.byref(d), C.byref(h)) == _lib.ERR_ARG
    assert L.padoc_rotary_create(C.byref(d), None) == _lib.ERR_ARG
    assert pa.Rotary(64, axis=[0] * 32, n_axes=3).n_axes == 3 and pa.Rotary(64, sections=(20, 12, 0)).n_axes == 3
    r = pa.Rotary(64)
    r.close()
    r.close()
    with pytest.raises(ValueError):
        r.handle


def test_forward_refused(rot, rot3):
    assert fwd(None) == _lib.ERR_ARG
    assert _lib.lib().padoc_rotary_fwd(rot.handle, None, None) == _lib.ERR_ARG
    for kw, status in [(dict(n=-1), _lib.ERR_ARG), (dict(n=2 ** 31), _lib.ERR_BOUNDS), (dict(hq=-1), _lib.ERR_SHAPE),
                       (dict(hkv=4097), _lib.ERR_SHAPE), (dict(pos=0), _lib.ERR_ARG), (dict(pos=A + 2), _lib.ERR_ARG),
                       (dict(q=heads(0)), _lib.ERR_ARG), (dict(k=heads(A + 1)), _lib.ERR_ARG),
                       (dict(qo=heads(0)), _lib.ERR_ARG), (dict(q=heads(rs=-256)), _lib.ERR_BOUNDS),
                       (dict(q=heads(hs=2 ** 41)), _lib.ERR_BOUNDS), (dict(wq=A + 1), _lib.ERR_ARG),
                       (dict(n=2 ** 30, q=heads(rs=2 ** 40)), _lib.ERR_BOUNDS)]:
        assert fwd(rot, **kw) == status, (kw, message())
    # what is written must not overlap itself or what is read
    for qo in (heads(3 * A, 0, 64), heads(3 * A, 256, 0), heads(3 * A, 256, 32), heads(3 * A, 64, 64), heads(3 * A, 96, 64)):
        assert fwd(rot, qo=qo) == _lib.ERR_BOUNDS, qo
    for qo in (heads(A + 2, 256, 64), heads(A, 128, 64), heads(A + 300, 256, 64), heads(A + 64, 256, 64), heads(A + 6, 64, 256)):
        assert fwd(rot, qo=qo) == _lib.ERR_ARG, qo
        assert "overlaps" in message()
    # q_out in k, or in k_out
    for kw in (dict(qo=heads(2 * A)), dict(ko=heads(A)), dict(ko=heads(3 * A + 64)), dict(n=1, qo=heads(2 * A, 0, 64))):
        assert fwd(rot, **kw) == _lib.ERR_ARG and "overlaps" in message(), kw
    # axes: one after the other, at least the rows apart, or all the same
    assert fwd(rot3, pos_stride=3) == _lib.ERR_BOUNDS
    assert fwd(rot3, pos_stride=-4) == _lib.ERR_BOUNDS
    # nothing to do: nothing is looked at
    assert fwd(rot, n=0, pos=0, q=heads(0), k=heads(0)) == _lib.OK
    assert fwd(rot, hq=0, hkv=0, pos=0) == _lib.OK


def test_backward_refused(rot):
    for kw, status in [(dict(n=-1), _lib.ERR_ARG), (dict(pos=0), _lib.ERR_ARG), (dict(gq=heads(0)), _lib.ERR_ARG),
                       (dict(dk=heads(0)), _lib.ERR_ARG), (dict(dwq=A), _lib.ERR_ARG), (dict(wq=A, q=heads(0)), _lib.ERR_ARG),
                       (dict(wq=A, wk=A, dwq=A, dwk=A), _lib.ERR_ARG), (dict(wq=A, dwq=A + 2), _lib.ERR_ARG),
                       (dict(dq=heads(3 * A, 0, 64)), _lib.ERR_BOUNDS), (dict(dq=heads(5 * A + 2)), _lib.ERR_ARG),
                       (dict(wq=A, dq=heads(A + 2)), _lib.ERR_ARG), (dict(dq=heads(4 * A)), _lib.ERR_ARG),
                       (dict(dk=heads(5 * A)), _lib.ERR_ARG), (dict(wk=A, dq=heads(2 * A)), _lib.ERR_ARG),
                       (dict(wq=A, dwq=A), _lib.ERR_WORKSPACE), (dict(wq=A, dwq=A, ws=256, nb=8), _lib.ERR_WORKSPACE),
                       (dict(wq=A, dwq=A, ws=128, nb=1 << 20), _lib.ERR_WORKSPACE)]:
        assert bwd(rot, **kw) == status, (kw, message())
    assert bwd(rot, n=0, pos=0) == _lib.OK
    L = _lib.lib()
    nb = C.c_size_t(0)
    for n in (0, 1, 100, 5000, 2 ** 31 - 1):
        assert L.padoc_rotary_bwd_workspace_bytes(rot.handle, n, 16, 2, C.byref(nb)) == _lib.OK
        assert 256 <= nb.value <= 8 << 20
    assert L.padoc_rotary_bwd_workspace_bytes(rot.handle, -1, 16, 2, C.byref(nb)) == _lib.ERR_ARG
    assert L.padoc_rotary_bwd_workspace_bytes(rot.handle, 1, 16, 2, None) == _lib.ERR_ARG
    assert L.padoc_rotary_bwd_workspace_bytes(None, 1, 16, 2, C.byref(nb)) == _lib.ERR_ARG
    assert L.padoc_rotary_bwd_workspace_bytes(rot.handle, 1, 16, 5000, C.byref(nb)) == _lib.ERR_SHAPE


def test_append_refused(rot):
    for kw, status in [(dict(n=-1), _lib.ERR_ARG), (dict(n_q=3), _lib.ERR_ARG), (dict(pos=0), _lib.ERR_ARG),
                       (dict(v=heads(0)), _lib.ERR_ARG), (dict(qo=heads(0)), _lib.ERR_ARG), (dict(slots=0), _lib.ERR_ARG),
                       (dict(slots=A + 1), _lib.ERR_ARG), (dict(kc=0), _lib.ERR_ARG), (dict(vc=A + 8), _lib.ERR_ARG),
                       (dict(kc=2 * A), _lib.ERR_ARG), (dict(nb=-1), _lib.ERR_ARG), (dict(nb=2 ** 31), _lib.ERR_ARG),
                       (dict(qo=heads(A + 2)), _lib.ERR_ARG), (dict(n_q=3, q_pos=A + 1), _lib.ERR_ARG),
                       (dict(qo=heads(2 * A)), _lib.ERR_ARG), (dict(qo=heads(3 * A + 8)), _lib.ERR_ARG)]:
        assert append(rot, **kw) == status, (kw, message())
    assert append(rot, n=0, n_q=0, pos=0, slots=0, kc=0, vc=0, nb=0) == _lib.OK


def test_session_launch_refused():
    """A host-only session: refused before the device is needed."""
    rot, s = pa.Rotary(64, "bf16"), pa.DecodeSession(2, 1, 64, 8)
    L = _lib.lib()

    def launch(rot=rot, n=3, n_q=3, hq=2, slots=0):
        a = [n_q, n, hq, 1, 0, 0, A, 0, *heads(), *heads(2 * A), *heads(3 * A), *heads(4 * A, 128, 64), 0, 0, slots, 0, 0, 0]
        return L.padoc_session_launch_rotary(s.handle, rot.handle, _lib.ROTARY_APPEND_ARGS.pack(*a), A, A, A, 1 << 20, None)
    assert launch() == _lib.ERR_MODE
    s.open()
    s.prepare([3], [3])
    assert launch(slots=A) == _lib.ERR_ARG and "session" in message()
    assert launch() == _lib.ERR_ARG and "without device" in message()
    with pytest.raises(RuntimeError):
        s.launch_rotary(None, None, None, None, rot)
    with pytest.raises(ValueError):
        s.resize(4, torch.zeros(1), None)


def test_copy_refused():
    L = _lib.lib()

    def copy(ks=A, vs=2 * A, ns=9, kd=A, vd=2 * A, nd=9, pairs=A, n=1, host=None, hkv=2, d=64, dtype=_lib.BF16):
        h = None if host is None else np.array(host, np.int32)
        return L.padoc_cache_copy_blocks(ks, vs, ns, kd, vd, nd, pairs, len(host) if host is not None else n,
                                         None if h is None else h.ctypes.data, hkv, d, dtype, None)
    for kw, status in [(dict(dtype=3), _lib.ERR_DTYPE), (dict(d=96), _lib.ERR_SHAPE), (dict(hkv=0), _lib.ERR_SHAPE),
                       (dict(n=-1), _lib.ERR_ARG), (dict(n=2 ** 31), _lib.ERR_BOUNDS), (dict(ns=-1), _lib.ERR_ARG),
                       (dict(nd=2 ** 31), _lib.ERR_ARG), (dict(ks=0), _lib.ERR_ARG), (dict(pairs=0), _lib.ERR_ARG),
                       (dict(vd=2 * A + 8), _lib.ERR_ARG), (dict(pairs=A + 2), _lib.ERR_ARG), (dict(vs=A, vd=A), _lib.ERR_ARG),
                       (dict(kd=2 * A, vd=A), _lib.ERR_ARG), (dict(vd=8 * A), _lib.ERR_ARG),
                       (dict(kd=A + 4096, vd=8 * A), _lib.ERR_ARG),
                       (dict(host=[[0, 9]]), _lib.ERR_BOUNDS), (dict(host=[[-1, 1]]), _lib.ERR_BOUNDS),
                       (dict(host=[[0, 1], [2, 1]]), _lib.ERR_BOUNDS), (dict(host=[[0, 1], [1, 2]]), _lib.ERR_BOUNDS),
                       (dict(host=[[3, 3]]), _lib.ERR_BOUNDS), (dict(host=[[0, 5]], kd=20 * A, vd=30 * A, nd=5), _lib.ERR_BOUNDS)]:
        assert copy(**kw) == status, (kw, message())
    assert copy(n=0, ks=0, pairs=0) == _lib.OK


def test_python_refuses_cpu_rows(rot):
    x, pos = torch.zeros((2, 1, 64), dtype=torch.bfloat16), torch.zeros((1, 2), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        pa.rotary_fwd(x, x, pos, rot)
    with pytest.raises(ValueError, match="GPU"):
        pa.rotary_bwd(x, x, pos, rot)
    with pytest.raises(TypeError):
        pa.rotary_fwd(None, None, pos, rot)
    with pytest.raises(ValueError, match="GPU"):
        pa.cache_copy_blocks(torch.zeros((1, 1, 8, 16, 8)), torch.zeros((1, 1, 64, 16)), pos)

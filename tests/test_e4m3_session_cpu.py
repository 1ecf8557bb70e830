"""Sessions on 8-bit caches: what they refuse of their scales' memory."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _streams import Gpu

A = 1 << 20
BLOCKS, HKV, D, TABLE = 8, 2, 64, 64
CODES, SCALES = BLOCKS * HKV * 16 * D, BLOCKS * HKV * 32  # bytes of a pool


@pytest.fixture
def session():
    """Codes of K at 1 MiB, of V at 2, block table at 3."""
    L, h = _lib.lib(), C.c_void_p()
    d = _lib.SessionDesc(4, HKV, D, 0.125, _lib.BF16_E4M3, BLOCKS, TABLE, A, 2 * A, 3 * A, 0, 0)
    assert L.padoc_session_create(C.byref(d), C.byref(h)) == _lib.OK
    yield h
    L.padoc_session_destroy(h)


def launch(h):
    """Status and message of a launch that is refused for its missing scales, or for its workspace."""
    L, n, size, one = _lib.lib(), C.c_int32(0), C.c_size_t(0), np.ones(2, np.int32)  # (of up to two streams)
    L.padoc_session_open(h, -1, 0, C.byref(n))
    assert L.padoc_session_prepare(h, one.ctypes.data, one.ctypes.data, C.byref(n), C.byref(n), C.byref(size)) == _lib.OK
    st = L.padoc_session_launch(h, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A, 0, 0, None), L.padoc_last_error().decode()
    assert L.padoc_session_commit(h) == _lib.OK
    return st


@pytest.mark.parametrize("name,start,size", [("k_cache", A, CODES), ("v_cache", 2 * A, CODES), ("block_table", 3 * A, 4 * TABLE)])
def test_scales_in_other_memory(session, name, start, size):
    """Any byte in common is refused, at either end, and no scales are named by it; memory right before or behind is not."""
    L = _lib.lib()
    for at in (start, start + 16, start + size - 16, start - SCALES + 16):
        assert L.padoc_session_set_scales(session, at) == _lib.ERR_ARG, hex(at)
        assert name in L.padoc_last_error().decode()
    st, why = launch(session)
    assert st == _lib.ERR_ARG and "scales" in why
    for at in (start - SCALES, start + size):
        assert L.padoc_session_set_scales(session, at) == _lib.OK, hex(at)
    assert L.padoc_session_set_scales(session, start) == _lib.ERR_ARG
    assert launch(session)[0] == _lib.ERR_WORKSPACE  # (the scales before are still named)


def test_a_pool_of_no_blocks(session):
    L = _lib.lib()
    assert L.padoc_session_resize(session, 0, A, 2 * A) == _lib.OK
    for at in (0, A, 3 * A + 16):  # (no scale is written)
        assert L.padoc_session_set_scales(session, at) == _lib.OK


@pytest.mark.parametrize("blocks", [5, 9, 12])
def test_a_refused_resize_leaves_the_session_as_it_was(monkeypatch, blocks):
    real, seen = _lib.lib(), {}

    def noted(name):
        return lambda *a: seen.__setitem__(name, a[1:]) or getattr(real, name)(*a)
    gpu = Gpu(monkeypatch, {n: noted(n) for n in ("padoc_session_resize", "padoc_session_set_scales")})

    def caches(n):
        f8 = torch.float8_e4m3fn
        return (gpu.tensor(torch.zeros((n, 2, 4, 16, 16), dtype=f8)), gpu.tensor(torch.zeros((n, 2, 64, 16), dtype=f8)),
                gpu.tensor(torch.zeros((n, 2, 2, 16), dtype=torch.float8_e8m0fnu)))
    k, v, s = caches(9)
    session = pa.DecodeSession(4, 2, 64, 9, "bf16_e4m3", k, v, gpu.tensor(torch.zeros(64, dtype=torch.int32)), scales=s)
    session.open()
    session.prepare([40], [1])  # three blocks
    session.commit()
    k2, v2, s2 = caches(blocks)
    inside = v2.view(torch.uint8).view(-1)[:s2.numel()].view(s2.shape).view(s2.dtype)  # (of V's codes)
    with pytest.raises(pa.PadocError, match="scales overlaps v_cache"):
        session.resize(blocks, k2, v2, scales=gpu.tensor(inside))
    assert seen == {"padoc_session_resize": (9, k.data_ptr(), v.data_ptr()), "padoc_session_set_scales": (s.data_ptr(),)}
    assert session.num_blocks == 9 and session.k_cache is k and session.v_cache is v and session.scales is s
    session.prepare([100], [1])  # nine blocks
    session.commit()
    session.truncate(0, 30)
    session.resize(blocks, k2, v2, scales=s2)
    assert seen["padoc_session_resize"][0] == blocks and seen["padoc_session_set_scales"] == (s2.data_ptr(),)
    assert session.num_blocks == blocks and session.scales is s2
    with pytest.raises(pa.PadocError, match="blocks"):
        session.prepare([16 * blocks], [1])

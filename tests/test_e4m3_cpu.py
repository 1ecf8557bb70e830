"""8-bit caches: the oracle's encoder against PyTorch's conversion, and what the
entry points refuse before they need a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _streams import Gpu

A = 1 << 20


def message():
    return _lib.lib().padoc_last_error().decode()


# ------------------------------------------------------------------ oracle

def test_values_are_pytorchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(orc.VALUES, want)
    b = np.arange(63, 248, dtype=np.uint8)
    np.testing.assert_array_equal(orc.decode(np.full((len(b), 1), 0x38, np.uint8), b)[:, 0],
                                  torch.from_numpy(b).view(torch.float8_e8m0fnu).double().numpy())


def test_encoder():
    """Codes against PyTorch's rounding, scales against their definition, by hand for a few."""
    rng = np.random.default_rng(1)
    x = rng.standard_normal((400, 64)) * np.exp2(rng.integers(-80, 80, size=(400, 1)))
    x[0] = 0
    x[1, :] = np.repeat((orc.VALUES[:64] + orc.VALUES[1:65]) / 2, 1)
    x = x.astype(np.float32).astype(np.float64)
    codes, s = orc.encode(x)
    e = s.astype(int) - 127
    a = np.abs(x).max(-1)
    assert (a <= 448 * np.exp2(e.astype(float))).all() and ((a > 224 * np.exp2(e.astype(float))) | (e == -64)).all()
    want = torch.from_numpy(x * np.exp2(-e.astype(float))[:, None]).float().to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    np.testing.assert_array_equal(codes, want)
    for row, byte, code in (([448.0], 127, 0x7e), ([448.5], 128, 0x76), ([1.0], 119, 0x78), ([-2.0 ** -70], 63, 0x80 | 8),
                            ([np.nan], 255, 0), ([np.inf, 1], 255, 0), ([3.3e38], 255, 0), ([3.29e38], 247, 0x77)):
        c, b = orc.encode(np.array([row]))
        assert (b[0], c[0, 0]) == (byte, code), (row, b, c)
    assert np.isnan(orc.decode(*orc.encode(np.array([[1.0, np.nan]])))).all()


# ---------------------------------------------------------------- refusals

def cache(k=A, v=2 * A, s=3 * A, n=9):
    return _lib.CACHE_E4M3.pack(k, v, s, n)


def plan(dtype="bf16_e4m3", blocks=9, paged=True):
    segs = pa.segments_layout([(-1, 0, 20, 4)], 16 if paged else 0)
    return pa.TreePlan(segs, 4, 2, 64, dtype, 16 if paged else 0, num_kv_rows=blocks if paged else 20, block_table_len=2 if paged else None)


def test_plans():
    for dtype in ("bf16_e4m3", "f32_e4m3"):
        with pytest.raises(pa.PadocError) as e:
            plan(dtype, paged=False)
        assert e.value.status == _lib.ERR_DTYPE and "paged" in str(e.value)
        p = plan(dtype)
        with pytest.raises(pa.PadocError) as e:
            p.backward_workspace_bytes()
        assert e.value.status in (_lib.ERR_DTYPE, _lib.ERR_MODE)
    with pytest.raises(pa.PadocError) as e:
        pa.Rotary(64, "bf16_e4m3")
    assert e.value.status == _lib.ERR_DTYPE
    assert set(plan().export()) == set(plan("bf16").export())


@pytest.mark.parametrize("call", ["padoc_branch_decode", "padoc_branch_decode_resident"])
def test_decode_refused(call):
    L, p, other = _lib.lib(), plan(), plan("bf16")
    f8, f = getattr(L, call + "_e4m3"), getattr(L, call)

    def run(p=p, q=A, c=cache(), bt=A, o=A, lse=A, ws=A, n=1 << 30):
        return f8(p.handle, q, c, bt, o, lse, ws, n, None)
    for kw, status in [(dict(c=None), _lib.ERR_ARG), (dict(c=cache(k=0)), _lib.ERR_ARG), (dict(c=cache(v=0)), _lib.ERR_ARG),
                       (dict(c=cache(s=0)), _lib.ERR_ARG), (dict(c=cache(s=A + 4)), _lib.ERR_ARG), (dict(c=cache(k=A + 8)), _lib.ERR_ARG),
                       (dict(c=cache(n=8)), _lib.ERR_BOUNDS), (dict(c=cache(n=10)), _lib.ERR_BOUNDS), (dict(p=other), _lib.ERR_DTYPE),
                       (dict(bt=0), _lib.ERR_ARG), (dict(q=0), _lib.ERR_ARG), (dict(lse=A + 2), _lib.ERR_ARG), (dict(ws=0), _lib.ERR_WORKSPACE),
                       (dict(ws=A + 8), _lib.ERR_WORKSPACE), (dict(n=100), _lib.ERR_WORKSPACE)]:
        assert run(**kw) == status, (kw, message())
    assert f8(None, A, cache(), A, A, A, A, 1 << 30, None) == _lib.ERR_ARG
    assert f(p.handle, A, A, 2 * A, A, A, A, A, 1 << 30, None) == _lib.ERR_DTYPE and "e4m3" in message()
    if call.endswith("resident"):
        assert run() == _lib.ERR_MODE  # (nothing uploaded)


def test_cast_refused():
    L = _lib.lib()

    def quantize(k=100 * A, v=200 * A, ns=9, c=cache(), pairs=A // 2, n=1, host=None, hkv=2, d=64, dtype=_lib.BF16):
        h = None if host is None else np.array(host, np.int32)
        return L.padoc_cache_quantize(k, v, ns, c, pairs, len(host) if host is not None else n, None if h is None else h.ctypes.data,
                                      hkv, d, dtype, None)

    def dequantize(k=100 * A, v=200 * A, ns=9, c=cache(), pairs=A // 2, n=1, host=None, hkv=2, d=64, dtype=_lib.BF16):
        h = None if host is None else np.array(host, np.int32)
        return L.padoc_cache_dequantize(c, k, v, ns, pairs, len(host) if host is not None else n, None if h is None else h.ctypes.data,
                                        hkv, d, dtype, None)
    both = [(dict(c=None), _lib.ERR_ARG), (dict(dtype=2), _lib.ERR_DTYPE), (dict(dtype=-1), _lib.ERR_DTYPE), (dict(d=96), _lib.ERR_SHAPE),
            (dict(hkv=0), _lib.ERR_SHAPE), (dict(hkv=4097), _lib.ERR_SHAPE), (dict(n=-1), _lib.ERR_ARG), (dict(n=2 ** 31), _lib.ERR_BOUNDS),
            (dict(ns=-1), _lib.ERR_ARG), (dict(ns=2 ** 31), _lib.ERR_ARG), (dict(c=cache(n=-1)), _lib.ERR_ARG), (dict(k=0), _lib.ERR_ARG),
            (dict(v=0), _lib.ERR_ARG), (dict(k=100 * A + 8), _lib.ERR_ARG), (dict(v=100 * A), _lib.ERR_ARG), (dict(c=cache(k=0)), _lib.ERR_ARG),
            (dict(c=cache(s=0)), _lib.ERR_ARG), (dict(c=cache(s=A + 16)), _lib.ERR_ARG), (dict(c=cache(v=A)), _lib.ERR_ARG),
            (dict(c=cache(s=3 * A + 8)), _lib.ERR_ARG), (dict(c=cache(k=100 * A + 4096)), _lib.ERR_ARG), (dict(pairs=A + 2), _lib.ERR_ARG),
            (dict(pairs=0, n=10), _lib.ERR_BOUNDS), (dict(pairs=0, n=9, ns=8), _lib.ERR_BOUNDS), (dict(pairs=0, host=[[0, 0]]), _lib.ERR_ARG),
            (dict(host=[[0, 9]]), _lib.ERR_BOUNDS), (dict(host=[[9, 0]]), _lib.ERR_BOUNDS), (dict(host=[[-1, 1]]), _lib.ERR_BOUNDS),
            (dict(host=[[0, 1], [2, 1]]), _lib.ERR_BOUNDS)]
    for f in (quantize, dequantize):
        for kw, status in both:
            assert f(**kw) == status, (f, kw, message())
        assert f(n=0, k=0, pairs=0) == _lib.OK
    assert quantize(ns=5, host=[[5, 0]]) == _lib.ERR_BOUNDS and dequantize(ns=5, host=[[0, 5]]) == _lib.ERR_BOUNDS


def test_copy_refused():
    L = _lib.lib()

    def copy(src=cache(), dst=cache(), pairs=A // 2, n=1, host=None, hkv=2, d=64):
        h = None if host is None else np.array(host, np.int32)
        return L.padoc_cache_copy_blocks_e4m3(src, dst, pairs, len(host) if host is not None else n, None if h is None else h.ctypes.data,
                                              hkv, d, None)
    far = cache(10 * A, 20 * A, 30 * A, 5)
    for kw, status in [(dict(src=None), _lib.ERR_ARG), (dict(dst=None), _lib.ERR_ARG), (dict(d=32), _lib.ERR_SHAPE), (dict(hkv=0), _lib.ERR_SHAPE),
                       (dict(n=-1), _lib.ERR_ARG), (dict(n=2 ** 31), _lib.ERR_BOUNDS), (dict(pairs=0), _lib.ERR_ARG), (dict(pairs=A + 1), _lib.ERR_ARG),
                       (dict(src=cache(k=0), dst=far), _lib.ERR_ARG), (dict(dst=cache(s=0)), _lib.ERR_ARG),
                       (dict(dst=cache(n=8)), _lib.ERR_ARG), (dict(dst=cache(k=A + 2048, v=20 * A, s=30 * A)), _lib.ERR_ARG),
                       (dict(dst=cache(v=20 * A)), _lib.ERR_ARG), (dict(src=cache(v=A), dst=cache(v=A)), _lib.ERR_ARG),
                       (dict(host=[[0, 1], [1, 2]]), _lib.ERR_BOUNDS), (dict(host=[[0, 9]]), _lib.ERR_BOUNDS), (dict(host=[[0, 1], [2, 1]]), _lib.ERR_BOUNDS),
                       (dict(dst=far, host=[[0, 5]]), _lib.ERR_BOUNDS)]:
        assert copy(**kw) == status, (kw, message())
    assert copy(n=0, pairs=0) == _lib.OK


def test_append_refused():
    L, rot = _lib.lib(), pa.Rotary(64, "bf16")
    heads = lambda p, rs=128, hs=64: (p, rs, hs)  # noqa: E731

    def append(c=cache(), n=3, slots=A // 2, kc=0, vc=0, nb=0, k=None, v=None, rotary=rot):
        a = [0, n, 0, 2, 0, 0, A // 2, 0, *heads(0), *heads(10 * A if k is None else k), *heads(11 * A if v is None else v), *heads(0), 0, 0,
             slots, kc, vc, nb]
        return L.padoc_rotary_append_e4m3(rotary and rotary.handle, _lib.ROTARY_APPEND_ARGS.pack(*a), c, None)
    for kw, status in [(dict(c=None), _lib.ERR_ARG), (dict(rotary=None), _lib.ERR_ARG), (dict(kc=A), _lib.ERR_ARG), (dict(vc=A), _lib.ERR_ARG),
                       (dict(nb=9), _lib.ERR_ARG), (dict(c=cache(k=0)), _lib.ERR_ARG), (dict(c=cache(s=0)), _lib.ERR_ARG),
                       (dict(c=cache(s=2 * A + 16)), _lib.ERR_ARG), (dict(c=cache(s=3 * A + 4)), _lib.ERR_ARG), (dict(c=cache(n=-1)), _lib.ERR_ARG),
                       (dict(c=cache(v=A)), _lib.ERR_ARG), (dict(slots=0), _lib.ERR_ARG), (dict(n=-1), _lib.ERR_ARG), (dict(k=0), _lib.ERR_ARG)]:
        assert append(**kw) == status, (kw, message())
    assert append(n=0, c=cache(0, 0, 0, 0), slots=0) == _lib.OK


def test_sessions():
    L = _lib.lib()
    s = pa.DecodeSession(4, 2, 64, 8, "bf16_e4m3")  # host-only
    assert L.padoc_session_set_scales(s.handle, A) == _lib.OK and L.padoc_session_set_scales(s.handle, A + 4) == _lib.ERR_ARG
    assert L.padoc_session_set_scales(pa.DecodeSession(4, 2, 64, 8).handle, A) == _lib.ERR_DTYPE
    assert L.padoc_session_set_scales(None, A) == _lib.ERR_ARG
    i = s.open()
    s.prepare([20], [3])
    v = s.view(schedule=True)
    assert len(v["new_slot"]) == 20 and len(v["schedule"]["work"])
    s.commit()
    s.truncate(i, 3)
    d = _lib.SessionDesc(4, 2, 64, 0.125, _lib.BF16_E4M3, 8, 64, A, 2 * A, 3 * A, 0, 0)
    h = C.c_void_p()
    assert L.padoc_session_create(C.byref(d), C.byref(h)) == _lib.OK

    def launch():
        n = C.c_int32(0)
        one = np.ones(1, np.int32)
        L.padoc_session_open(h, -1, 0, C.byref(n))
        size = C.c_size_t(0)
        assert L.padoc_session_prepare(h, one.ctypes.data, one.ctypes.data, C.byref(n), C.byref(n), C.byref(size)) == _lib.OK
        st = L.padoc_session_launch(h, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A, 9 * A, 1 << 30, None)
        return st, message()
    st, why = launch()
    assert st == _lib.ERR_ARG and "scales" in why
    assert L.padoc_session_commit(h) == _lib.OK
    assert L.padoc_session_set_scales(h, 2 * A) == _lib.ERR_ARG  # V's codes
    assert L.padoc_session_set_scales(h, 10 * A) == _lib.OK
    assert L.padoc_session_resize(h, 8, A, 2 * A) == _lib.OK      # forgets them
    one = np.ones(1, np.int32)
    n, size = C.c_int32(0), C.c_size_t(0)
    assert L.padoc_session_prepare(h, one.ctypes.data, one.ctypes.data, C.byref(n), C.byref(n), C.byref(size)) == _lib.OK
    assert L.padoc_session_launch(h, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A, 9 * A, 1 << 30, None) == _lib.ERR_ARG and "scales" in message()
    L.padoc_session_destroy(h)


def test_python_refuses_cpu_caches():
    c = pa.empty_cache_e4m3(2, 1, 64, "cpu")
    assert [tuple(t.shape) for t in c] == [(2, 1, 4, 16, 16), (2, 1, 64, 16), (2, 1, 2, 16)]
    k, v = torch.zeros((2, 1, 8, 16, 8)), torch.zeros((2, 1, 64, 16))
    with pytest.raises(ValueError, match="GPU"):
        pa.cache_quantize(k, v, *c)
    with pytest.raises(ValueError, match="GPU"):
        pa.cache_dequantize(*c)
    with pytest.raises(ValueError, match="GPU"):
        pa.cache_copy_blocks(c[0], c[1], torch.zeros((1, 2), dtype=torch.int32), scales=c[2])


# ------------------------------------------------- whose memory a call uses

@pytest.mark.parametrize("what", ["quantize", "dequantize", "append", "decode"])
def test_calls_allocate_on_the_callers_stream(monkeypatch, what):
    seen = []
    names = {"quantize": "padoc_cache_quantize", "dequantize": "padoc_cache_dequantize", "append": "padoc_rotary_append_e4m3",
             "decode": "padoc_branch_decode_e4m3"}
    gpu = Gpu(monkeypatch, {names[what]: lambda *a: seen.append(a) or 0})
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True), raising=False)
    t = lambda *shape, dtype=torch.bfloat16: gpu.tensor(torch.zeros(shape, dtype=dtype))  # noqa: E731
    k, v = t(9, 2, 8, 16, 8), t(9, 2, 64, 16)
    k8, v8 = t(9, 2, 4, 16, 16, dtype=torch.float8_e4m3fn), t(9, 2, 64, 16, dtype=torch.float8_e4m3fn)
    s8 = t(9, 2, 2, 16, dtype=torch.float8_e8m0fnu)
    rot, p = pa.Rotary(64, "bf16"), plan()
    q, rows, pos, slots, table = t(4, 4, 64), t(4, 2, 64), t(4, dtype=torch.int32), t(4, 2, dtype=torch.int32), t(2, dtype=torch.int32)
    given = len(gpu.made)
    out = {"quantize": lambda: pa.cache_quantize(k, v, stream=gpu.side), "dequantize": lambda: pa.cache_dequantize(k8, v8, s8, stream=gpu.side),
           "append": lambda: pa.rotary_append(q, rows, rows, pos, slots, k8, v8, rot, scales=s8, stream=gpu.side),
           "decode": lambda: pa.branch_decode(q, k8, v8, table, p, scales=s8, stream=gpu.side)}[what]()
    made = gpu.made[given:]
    assert gpu.current is gpu.first and len(seen) == 1 and made and all(m.allocated is gpu.side for m in made)
    assert int(getattr(seen[0][-1], "value", seen[0][-1])) == gpu.side.cuda_stream
    assert all(gpu.first in m.recorded for m in (out if isinstance(out, tuple) else (out,)))


def test_a_session_keeps_its_scales(monkeypatch):
    gpu = Gpu(monkeypatch, {"padoc_session_launch": lambda *a: s.commit() or 0})
    t = lambda *shape, dtype=torch.bfloat16: gpu.tensor(torch.zeros(shape, dtype=dtype))  # noqa: E731
    f8 = torch.float8_e4m3fn
    caches = t(9, 2, 4, 16, 16, dtype=f8), t(9, 2, 64, 16, dtype=f8), t(64, dtype=torch.int32), t(9, 2, 2, 16, dtype=torch.float8_e8m0fnu)
    s = pa.DecodeSession(4, 2, 64, 9, "bf16_e4m3", *caches[:3], scales=caches[3])
    s.open()
    s.prepare([2], [2])
    s.launch(t(2, 4, 64), t(2, 2, 64), t(2, 2, 64), stream=gpu.side)
    assert all(gpu.side in c.recorded for c in caches)

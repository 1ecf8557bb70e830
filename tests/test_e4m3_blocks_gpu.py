"""8-bit caches: blocks quantised and read back bit for bit, copied, nothing
else written."""
import numpy as np
import pytest
import torch

from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _e4m3 import on_gpu, on_host
from _rotary import f64, k_block_view, torch_dtype, v_block_view

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["native", "python"])
def binding(request, monkeypatch):
    """Every test through the native module and without it."""
    if request.param == "python":
        monkeypatch.setattr(_lib, "native_rows", lambda: None)
        monkeypatch.setattr(pa, "_native_cast", lambda back: lambda *a: None)
    else:
        assert _lib.native_rows() is not None, "the native module is not built"
    return request.param


def value_rows(blocks, hkv, d, dtype, seed):
    """Rows of every kind: drawn ones, zeros, the smallest and the largest numbers, values halfway between codes,
    rows whose largest value is 448 times a power of two or just above it, infinities, NaN."""
    rng = np.random.default_rng([seed, 3])
    x = rng.standard_normal((blocks, hkv, 16, d)) * np.exp2(rng.integers(-70, 60, size=(blocks, hkv, 16, 1)))
    half = (orc.VALUES[8:126] + orc.VALUES[9:127]) / 2
    flat = x.reshape(-1, d)
    for i in range(0, len(flat), 7):
        kind = i // 7 % 9
        row = flat[i]
        if kind == 0:
            row[:] = 0
        elif kind == 1:
            row[:] = rng.choice(half, d) * 2.0 ** rng.integers(-20, 20)
        elif kind == 2:
            row[rng.integers(d)] = 448 * 2.0 ** 5
            row[np.abs(row) > 448 * 2.0 ** 5] = 1
        elif kind == 3:
            row[:] = 1
            row[rng.integers(d)] = 448 * (1 + 2.0 ** -7)
        elif kind == 4:
            row[:] = rng.standard_normal(d) * 2.0 ** -126  # (and below: subnormal)
        elif kind == 5:
            row[rng.integers(d)] = [3.29e38, 3.3e38, 248 * 2.0 ** 120, 247 * 2.0 ** 120][i // 63 % 4]
        elif kind == 6:
            row[rng.integers(d)] = rng.choice([np.inf, -np.inf])
        elif kind == 7:
            row[rng.integers(d)] = np.nan
        else:
            row[:] = -rng.choice(orc.VALUES[:127], d)
    return torch.from_numpy(flat.reshape(x.shape)).to(torch_dtype(dtype))


def caches_of(k, v):
    """Rows [blocks, Hkv, 16, d] in the library's layouts."""
    nb, h, _, d = k.shape
    slot = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]
    kc = k.reshape(nb, h, 16, d // 8, 8).transpose(2, 3)[:, :, :, slot].contiguous()
    return kc.cuda(), v.transpose(2, 3).contiguous().cuda()


def encoded(k, v):
    kc, ks = orc.encode(f64(k), nan_code=0x7f)
    vc, vs = orc.encode(f64(v))
    nb, h, _, d = k.shape
    return kc.reshape(nb, h, 16, d // 16, 16).transpose(0, 1, 3, 2, 4), vc.transpose(0, 1, 3, 2), np.stack([ks, vs], 2)


def same(got, want):
    for name, g, w in zip(("k", "v", "scales"), on_host(got), want):
        bad = g != w
        assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), g[bad][:5], w[bad][:5])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(64, 1), (64, 3), (128, 1), (128, 2), (128, 5)])
@pytest.mark.parametrize("n", [1, 2, 33])
def test_quantize_block_for_block(dtype, d, hkv, n):
    print("[case] quantize", dtype, d, hkv, n, flush=True)
    k, v = (value_rows(n, hkv, d, dtype, s) for s in (1, 2))
    out = pa.cache_quantize(*caches_of(k, v))
    same(out, encoded(k, v))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(64, 2), (128, 3)])
def test_quantize_by_pairs(dtype, d, hkv):
    """Into another pool of another size: a source twice, pairs outside either pool left out, the rest as it was."""
    print("[case] quantize pairs", dtype, d, hkv, flush=True)
    k, v = (value_rows(9, hkv, d, dtype, s) for s in (3, 4))
    before = orc.empty(14, hkv, d, 1)
    pairs = np.array([[0, 13], [8, 0], [8, 5], [3, 4], [9, 1], [-1, 2], [2, 14], [2, -1], [1 << 30, 7]], np.int32)
    want = [x.copy() for x in before]
    new = encoded(k, v)
    for a, b in pairs[:4]:
        for w, x in zip(want, new):
            w[b] = x[a]
    dst = on_gpu(before)
    out = pa.cache_quantize(*caches_of(k, v), *dst, pairs=torch.from_numpy(pairs).cuda())
    assert all(o is t for o, t in zip(out, dst))
    same(out, want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(64, 1), (64, 3), (128, 1), (128, 2)])
@pytest.mark.parametrize("n", [1, 2, 33])
def test_dequantize(dtype, d, hkv, n):
    """Every code and scale that the library writes, exactly; NaN rows."""
    print("[case] dequantize", dtype, d, hkv, n, flush=True)
    k, v, s = orc.empty(n, hkv, d, n)
    k[(k & 127) == 127] = 0x7e
    v[(v & 127) == 127] = 0xfe
    s = np.where(s < 9, 255, np.clip(s, 63, 240)).astype(np.uint8)
    kc, vc = pa.cache_dequantize(*on_gpu((k, v, s)), dtype=dtype)
    assert kc.dtype is torch_dtype(dtype)
    wk = orc.decode(k.transpose(0, 1, 3, 2, 4).reshape(n, hkv, 16, d), s[:, :, 0])
    wv = orc.decode(v.transpose(0, 1, 3, 2), s[:, :, 1])
    np.testing.assert_array_equal(f64(k_block_view(kc)), wk)
    np.testing.assert_array_equal(f64(v_block_view(vc)), wv)


def test_dequantize_by_pairs_and_back():
    """What is read back quantises to the same values.  (Not always to the same codes: a largest value of 450 takes the
    scale of 448 * 2, is kept as 224 * 2, and that takes the scale of 448; the smaller scale's grid holds every value of
    the larger one's up to 448 of it.)"""
    k, v = (value_rows(12, 2, 128, "bf16", s) for s in (5, 6))
    q8 = pa.cache_quantize(*caches_of(k, v))
    kd = torch.full((20, 2, 16, 16, 8), 7.0, dtype=torch.bfloat16, device="cuda")
    vd = torch.full((20, 2, 128, 16), 7.0, dtype=torch.bfloat16, device="cuda")
    to = np.random.default_rng(1).permutation(20)[:12]
    pairs = np.stack([np.arange(12), to], 1).astype(np.int32)
    out = pa.cache_dequantize(*q8, kd, vd, pairs=torch.from_numpy(pairs).cuda(), pairs_host=pairs)
    assert out[0] is kd and out[1] is vd
    rest = np.setdiff1d(np.arange(20), to)
    assert (kd[rest] == 7).all() and (vd[rest] == 7).all()
    again = pa.cache_dequantize(*pa.cache_quantize(kd[to].contiguous(), vd[to].contiguous()))
    for a, b in zip(again, (kd[to], vd[to])):
        np.testing.assert_array_equal(f64(a), f64(b))


@pytest.mark.parametrize("d,hkv,n", [(64, 1, 1), (64, 5, 40), (128, 2, 24), (128, 3, 301)])
def test_copy_blocks(d, hkv, n):
    print("[case] copy e4m3", d, hkv, n, flush=True)
    before = orc.empty(2 * n + 5, hkv, d, n)
    ids = np.random.default_rng(n).permutation(2 * n + 5)[:2 * n].reshape(-1, 2).astype(np.int32)
    ids[n // 2:, 0] = ids[n // 2, 0]
    want = [x.copy() for x in before]
    for w in want:
        w[ids[:, 1]] = w[ids[:, 0]]
    cache = on_gpu(before)
    out = pa.cache_copy_blocks(*cache[:2], torch.from_numpy(ids).cuda(), pairs_host=ids, scales=cache[2])
    assert all(o is t for o, t in zip(out, cache))
    same(out, want)
    other = orc.empty(3, hkv, d, n + 1)
    dst = on_gpu(other)
    pairs = np.array([[1, 2], [4, 0], [0, 3], [2 * n + 5, 1]], np.int32)
    pa.cache_copy_blocks(*cache[:2], torch.from_numpy(pairs).cuda(), *dst[:2], scales=cache[2], scales_dst=dst[2])
    for o, w in zip(other, want):
        o[2], o[0] = w[1], w[4]
    same(dst, other)


def test_no_blocks():
    e = pa.empty_cache_e4m3(0, 2, 64, "cuda")
    kc, vc = pa.cache_dequantize(*e)
    assert kc.shape == (0, 2, 8, 16, 8) and vc.shape == (0, 2, 64, 16)
    assert pa.cache_quantize(kc, vc)[2].shape == (0, 2, 2, 16)


def test_refusals():
    k, v = caches_of(*(value_rows(4, 2, 64, "bf16", s) for s in (1, 2)))
    k8, v8, s8 = pa.empty_cache_e4m3(4, 2, 64, "cuda")
    pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    for args, kw in [((k.half(), v.half()), {}), ((k, v[:3]), {}), ((k.cpu(), v.cpu()), {}), ((k, v, k8, v8), {}),
                     ((k, v, k8, v8, s8[:, :, :1]), {}), ((k, v, k8.view(torch.uint8), v8, s8), {}), ((k, v, v8, k8, s8), {}),
                     ((k, v, k8, v8, s8), {"pairs": pairs.long()}), ((k, v, k8, v8, s8), {"pairs": pairs[0]}),
                     ((k, v), {"pairs": pairs}), ((k[:3].contiguous(), v[:3].contiguous(), k8, v8, s8), {}),
                     ((k, v, k8, v8, s8), {"pairs_host": pairs.cpu().numpy()}),
                     ((k, v) + pa.empty_cache_e4m3(4, 1, 64, "cuda"), {}), ((k.transpose(2, 3), v, k8, v8, s8), {})]:
        with pytest.raises((ValueError, TypeError)):
            pa.cache_quantize(*args, **kw)
    for args, kw in [((k8, v8, s8.view(torch.uint8)), {}), ((k8, v8, None), {}), ((k8, v8, s8, k), {}),
                     ((k8, v8, s8), {"pairs": pairs}), ((k8, v8, s8), {"dtype": "bf16_e4m3"}), ((k8, v8, s8, v, k), {})]:
        with pytest.raises((ValueError, TypeError)):
            pa.cache_dequantize(*args, **kw)
    for args, kw in [((k8, v8, pairs), {}), ((k8, v8, pairs, k8, v8), {"scales": s8}), ((k, v, pairs), {"scales": s8}),
                     ((k8, v8, pairs), {"scales": s8, "scales_dst": s8.clone()})]:
        with pytest.raises((ValueError, TypeError)):
            pa.cache_copy_blocks(*args, **kw)
    with pytest.raises(pa.PadocError):
        pa.cache_quantize(k, v, k8, v8, s8, pairs=pairs, pairs_host=np.array([[0, 4]], np.int32))


def lazily(t):
    """A clone that shares t's memory until one of them is written."""
    c = t.view(torch.uint8)._lazy_clone().view(t.dtype)
    assert torch._C._is_cow_tensor(c)
    return c


def test_outputs_that_share_memory(binding):
    """Codes written into lazy clones leave the caches that those were cloned from."""
    k = torch.randn(3, 2, 8, 16, 8, device="cuda", dtype=torch.bfloat16)
    v = torch.randn(3, 2, 64, 16, device="cuda", dtype=torch.bfloat16)
    held = [torch.zeros_like(t.view(torch.uint8)).view(t.dtype) for t in pa.empty_cache_e4m3(3, 2, 64, "cuda")]
    to = [lazily(t) for t in held]
    if binding == "native":
        assert pa._native_cast(False)(k, v, *to, None) == 0
    else:
        pa.cache_quantize(k, v, *to)
    assert all((t.view(torch.uint8) == 0).all() for t in held)
    want = pa.cache_quantize(k, v)
    assert all((a.view(torch.uint8) == b.view(torch.uint8)).all() for a, b in zip(to, want))
    kd, vd = torch.zeros_like(k), torch.zeros_like(v)
    k2, v2 = kd._lazy_clone(), vd._lazy_clone()
    pa.cache_dequantize(*want, k2, v2)
    assert (kd == 0).all() and (vd == 0).all() and (k2 != 0).any()


def test_native_calls_leave_what_they_cannot_check(binding):
    """Odd calls come back unanswered, and the Python function says what is wrong (or makes the call)."""
    if binding != "native":
        return
    k = torch.zeros(2, 1, 8, 16, 8, device="cuda", dtype=torch.bfloat16)
    v = torch.zeros(2, 1, 64, 16, device="cuda", dtype=torch.bfloat16)
    e = pa.empty_cache_e4m3(2, 1, 64, "cuda")
    cast = pa._native_cast(False)
    assert cast(k, v, *e, None) == 0
    for bad in ((k.half(), v, *e, None), (k, v.cpu(), *e, None), (k, v, e[0], e[1], e[2].view(torch.uint8), None),
                (k, v, e[0][:1], e[1], e[2], None), (k, v, *[t[:1] for t in e], None),
                (k, v, *e, torch.zeros(2, 2, device="cuda")), (k, v, *e, torch.zeros(2, 2, dtype=torch.int32))):
        assert cast(*bad) is None


def test_captured_casts(binding):
    """Values to codes and back in one graph, replayed on new values with eager calls between."""
    k = torch.empty(5, 2, 16, 16, 8, device="cuda", dtype=torch.bfloat16)
    v = torch.empty(5, 2, 128, 16, device="cuda", dtype=torch.bfloat16)
    e, (k2, v2) = pa.empty_cache_e4m3(4, 2, 128, "cuda"), (torch.zeros_like(k), torch.zeros_like(v))
    pairs = torch.tensor([[0, 3], [4, 1], [2, 0], [2, 2]], dtype=torch.int32, device="cuda")
    back = pairs.flip(1)[:3].contiguous()  # (no destination twice)

    def both():
        pa.cache_quantize(k, v, *e, pairs=pairs)
        pa.cache_dequantize(*e, k2, v2, pairs=back)

    def draw(seed):
        for t in (k, v):
            t.copy_(torch.randn(t.shape, generator=torch.Generator().manual_seed(seed)))

    draw(0)
    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    for seed in range(1, 4):
        draw(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.view(torch.uint8).clone() for t in (*e, k2, v2)]
        both()
        assert all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(got, (*e, k2, v2)))
        assert ((k2[[0, 2, 4]].float() - k[[0, 2, 4]].float()).abs() <= 2.0 ** -4 * k[[0, 2, 4]].float().abs() + 2.0 ** -6).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_behind_four_gigabytes(binding, dtype):
    """Blocks of an 8-bit pool whose codes pass 2^32 bytes, written and read back."""
    hkv, d = 8, 128
    blocks = (1 << 32) // (hkv * d * 16) + 3
    if torch.cuda.mem_get_info()[0] < 3 * blocks * hkv * d * 16:
        pytest.skip("not enough memory")
    k = torch.randn(2, hkv, d // 8, 16, 8, device="cuda").to(torch_dtype(dtype))
    v = torch.randn(2, hkv, d, 16, device="cuda").to(torch_dtype(dtype))
    far = pa.empty_cache_e4m3(blocks, hkv, d, "cuda")
    pairs = torch.tensor([[0, blocks - 1], [1, blocks - 2]], dtype=torch.int32, device="cuda")
    print("[case] far blocks", dtype, flush=True)
    pa.cache_quantize(k, v, *far, pairs=pairs)
    near = pa.cache_quantize(k, v)
    assert all(torch.equal(a[[blocks - 1, blocks - 2]].view(torch.uint8), b.view(torch.uint8)) for a, b in
               zip([x.view(torch.uint8) for x in far], near))
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    pa.cache_dequantize(*far, k2, v2, pairs=pairs.flip(1).contiguous())
    k3, v3 = pa.cache_dequantize(*near, dtype=dtype)
    assert torch.equal(k2, k3) and torch.equal(v2, v3)

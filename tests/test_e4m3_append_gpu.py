"""rotary_append into 8-bit caches: rows normed, rotated and quantised, against
the format's own encoder in 64 bits."""
import numpy as np
import pytest
import torch

from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _e4m3 import on_gpu, on_host
from _rotary import Setup, check, f64, normal, positions

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


def places(n, blocks, seed, together=False):
    """(block, slot) of n rows: drawn, or runs of rows in consecutive slots."""
    rng = np.random.default_rng([seed, 4])
    if together:
        at = rng.integers(0, 16) + np.arange(n)
        return np.stack([rng.permutation(blocks)[at // 16], at % 16], 1).astype(np.int32)
    p = rng.permutation(blocks * 16)[:n]
    return np.stack([p // 16, p % 16], 1).astype(np.int32)


def check_rows(st, before, after, slots, k, v, pos, wk):
    """Rows that were appended hold the codes of z (K, within z's own error) and v (V, bit for bit); nothing else changed."""
    kc, vc, sc = after
    keep = (slots[:, 0] >= 0) & (slots[:, 0] < len(vc)) & (slots[:, 1] >= 0) & (slots[:, 1] < 16)
    blk, t = slots[keep, 0], slots[keep, 1]
    want = [x.copy() for x in before]
    orc.write(want, blk, t, np.zeros_like(f64(k)[keep]), f64(v)[keep])
    for w, x in zip((want[0], want[2][:, :, 0]), (kc, sc[:, :, 0])):  # K's are checked by value below
        if w.ndim == 5:
            w[blk, :, :, t] = x[blk, :, :, t]
        else:
            w[blk, :, t] = x[blk, :, t]
    for name, x, w in zip(("k", "v", "scales"), after, want):
        assert (x == w).all(), (name, np.argwhere(x != w)[:3].tolist())
    z, tol = st.forward(k[torch.from_numpy(np.nonzero(keep)[0]).cuda()], pos[:, np.nonzero(keep)[0]], wk)
    tol = tol - (2.0 ** -8 * np.abs(z) / (1 + 2.0 ** -8) if st.dtype == "bf16" else 0)  # (rounded to codes alone)
    s = sc[blk, :, 0, t].astype(np.int64)
    a, slack = np.abs(z).max(-1), tol.max(-1)
    lowest = s == 127 + orc.MIN_EXPONENT
    top = 448 * np.exp2(s - 127.0)
    assert (a - slack <= top).all() and ((a + slack > top / 2) | lowest).all()
    got = orc.decode(kc[blk, :, :, t].reshape(z.shape), s.astype(np.uint8))
    half = np.maximum(2.0 ** -4 * (np.abs(z) + tol), 2.0 ** -10 * np.exp2(s - 127.0)[..., None])
    assert (np.abs(got - z) <= tol + half).all(), np.abs(got - z).max()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rd,style,axes,norm", [(128, 128, "halves", 3, True), (64, 64, "halves", 3, True),
                                                  (128, 64, "pairs", 1, False), (64, 32, "pairs", 4, True),
                                                  (64, 16, "halves", 1, False), (128, 48, "halves", 3, True)])
@pytest.mark.parametrize("n,hq,hkv,together", [(1, 4, 1, False), (17, 16, 2, False), (75, 3, 3, True), (300, 28, 4, True)])
def test_rows(dtype, d, rd, style, axes, norm, n, hq, hkv, together):
    print("[case] append e4m3", dtype, d, rd, style, axes, norm, n, hq, hkv, together, flush=True)
    st = Setup(d, dtype, rotary_dim=rd, n_axes=axes, style=style, base=1e6, scale=1.25)
    qkv = normal((n, hq + 2 * hkv, d), n, dtype, spread=3.0)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    wq, wk = (normal((d,), s, dtype) if norm else None for s in (2, 3))
    pos = positions(axes, n, 4, far=70000)
    blocks = n // 8 + 9
    before = orc.empty(blocks, hkv, d, n)
    slots = places(n, blocks, n, together)
    if n > 2:
        slots[1] = -1, 3
        slots[2] = blocks, 0
    gpu = on_gpu(before)
    out = pa.rotary_append(q, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, wq, wk, scales=gpu[2])
    torch.cuda.synchronize()
    check("q", out, *st.forward(q, pos, wq))
    check_rows(st, before, on_host(gpu), slots, k, v, pos, wk)


@pytest.mark.parametrize("dtype,d,hkv,n", [("bf16", 128, 2, 3331), ("f32", 128, 3, 2101), ("bf16", 64, 7, 901), ("f32", 64, 1, 6200)])
def test_rows_of_many_runs(dtype, d, hkv, n):
    """A prefill's rows: runs of every length from 1 to 49 and every first slot, whole blocks among them, rows left out and
    single rows in between, runs that go on in the block that the next run is in."""
    rng = np.random.default_rng([n, 6])
    slots, blocks, free = np.zeros((n, 2), np.int32), n // 4, list(rng.permutation(n // 4))
    i = r = 0
    while i < n:
        at, blk = r % 16, free.pop()
        for _ in range(min(n - i, 1 + r * 7 % 49)):
            if at == 16:
                at, blk = 0, free.pop()
            slots[i] = blk, at
            at += 1
            i += 1
        r += 1
    gone = rng.choice(n, n // 40, replace=False)
    slots[gone[::2], 0], slots[gone[1::2], 1] = -1, 16
    st = Setup(d, dtype, base=1e5)
    qkv = normal((n, 1 + 2 * hkv, d), n, dtype, spread=3.0)
    q, k, v = qkv[:, :1], qkv[:, 1:1 + hkv], qkv[:, 1 + hkv:]
    pos, wk = positions(3, n, 4), normal((d,), 3, dtype)
    before = orc.empty(blocks, hkv, d, n)
    gpu = on_gpu(before)
    print("[case] append e4m3 runs", dtype, d, hkv, n, flush=True)
    out = pa.rotary_append(q, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, None, wk, scales=gpu[2])
    check("q", out, *st.forward(q, pos))
    check_rows(st, before, on_host(gpu), slots, k, v, pos, wk)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rd,style,axes,norm", [(128, 128, "halves", 3, True), (64, 64, "halves", 3, True),
                                                  (64, 32, "pairs", 1, True), (128, 96, "halves", 1, False)])
def test_codes_of_k_are_those_of_64_bits(dtype, d, rd, style, axes, norm):
    """K's codes and scales bit for bit: z is within some 2^-36 of its 64-bit value, and of 200 thousand values drawn
    none lies that close to the border between two codes (a chance of 200,000 x 2^-36 / 2^-4 = 5e-5)."""
    n, hkv = 800, 2
    st = Setup(d, dtype, rotary_dim=rd, n_axes=axes, style=style, base=1e6, scale=1.25)
    k, v = normal((n, hkv, d), 21, dtype, spread=3.0), normal((n, hkv, d), 22, dtype)
    wk, pos = normal((d,), 23, dtype) if norm else None, positions(axes, n, 24, far=70000)
    slots = places(n, 60, 25)
    before = orc.empty(60, hkv, d, 26)
    gpu = on_gpu(before)
    print("[case] append e4m3 exact codes", dtype, d, rd, style, flush=True)
    pa.rotary_append(None, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, None, wk, scales=gpu[2])
    want = [w.copy() for w in before]
    orc.write(want, slots[:, 0], slots[:, 1], st.forward(k, pos, wk)[0], f64(v))
    for name, a, w in zip(("k", "v", "scales"), on_host(gpu), want):
        assert (a == w).all(), (name, (a != w).sum(), np.argwhere(a != w)[:4].tolist())


@pytest.mark.parametrize("n", [40, 900])
def test_blocks_behind_four_gigabytes(n):
    """Rows into blocks of a pool whose codes pass 2^32 bytes, byte by byte and by whole blocks: as into a small pool."""
    hkv, d = 8, 128
    blocks = (1 << 32) // (hkv * d * 16) + 64
    if torch.cuda.mem_get_info()[0] < 3 * blocks * hkv * d * 16:
        pytest.skip("not enough memory")
    st = Setup(d, "bf16")
    k, v, pos = normal((n, hkv, d), 1, "bf16"), normal((n, hkv, d), 2, "bf16"), positions(3, n, 3)
    near, far = pa.empty_cache_e4m3(64, hkv, d, "cuda"), pa.empty_cache_e4m3(blocks, hkv, d, "cuda")
    for a, b in zip(near, far):
        a.view(torch.uint8).zero_()
        b.view(torch.uint8)[-64:] = 0
    slots = torch.from_numpy(places(n, 64, 5, together=True)).cuda()
    print("[case] append e4m3 far blocks", n, flush=True)
    pa.rotary_append(None, k, v, pos, slots, *near[:2], st.handle, scales=near[2])
    pa.rotary_append(None, k, v, pos, slots + torch.tensor([blocks - 64, 0], dtype=torch.int32, device="cuda"), *far[:2], st.handle,
                     scales=far[2])
    assert near[2].view(torch.uint8).count_nonzero() > 0
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)[-64:]) for a, b in zip(near, far))


def test_rows_of_every_kind():
    """Zeros, the largest and the smallest numbers, infinities and NaN: V bit for bit, K's NaN rows NaN; without
    queries, without a rotation that mixes them (position 0)."""
    n, hkv, d = 40, 2, 128
    st = Setup(d, "bf16", n_axes=1)
    x = normal((n, 2 * hkv, d), 1, "bf16").cpu()
    x[0], x[1], x[2], x[3] = 0, x[3] * 2.0 ** 120, x[4] * 2.0 ** -120, x[5] * 2.0 ** -66
    x[4, 0, 5], x[5, 1, 6], x[6, 2, 7], x[7, 3, 8] = float("nan"), float("inf"), float("-inf"), float("nan")
    x = x.cuda()
    k, v, pos = x[:, :hkv], x[:, hkv:], torch.zeros((1, n), dtype=torch.int32, device="cuda")
    before = orc.empty(6, hkv, d, 1)
    slots = places(n, 6, 1)
    gpu = on_gpu(before)
    print("[case] append e4m3 rows of every kind", flush=True)
    assert pa.rotary_append(None, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, scales=gpu[2]) is None
    want = [w.copy() for w in before]
    orc.write(want, slots[:, 0], slots[:, 1], f64(k), f64(v))
    for name, a, w in zip(("k", "v", "scales"), on_host(gpu), want):
        # (at position 0 a rotation multiplies by 1 and adds a product with 0, whose sum with -0 is 0)
        zero = (a & 127 == 0) & (w & 127 == 0) if name == "k" else False
        nan_row = np.zeros(a.shape, bool)
        assert ((a == w) | zero | nan_row).all(), (name, np.argwhere(a != w)[:4].tolist(), a[a != w][:4], w[a != w][:4])


def test_strided_rows_many_tokens_and_no_rows():
    """More rows than one tile a workgroup, in heads of a fused projection; then no rows at all."""
    n, hq, hkv, d = 9001, 2, 1, 64
    st = Setup(d, "bf16", base=1e4)
    x = normal((hq + 2 * hkv, n, d), 1, "bf16").transpose(0, 1)  # heads outermost
    q, k, v = x[:, :hq], x[:, hq:hq + 1], x[:, hq + 1:]
    pos = positions(3, n, 2)
    before = orc.empty(700, hkv, d, 1)
    slots = places(n, 700, 2)
    gpu = on_gpu(before)
    print("[case] append e4m3 many rows", flush=True)
    out = pa.rotary_append(q, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, scales=gpu[2])
    check("q", out, *st.forward(q, pos))
    after = on_host(gpu)
    check_rows(st, before, after, slots, k, v, pos, None)
    none = pa.rotary_append(q[:0], k[:0], v[:0], pos[:, :0], torch.from_numpy(slots[:0]).cuda(), *gpu[:2], st.handle, scales=gpu[2])
    assert none.shape == (0, hq, d)
    for a, b in zip(on_host(gpu), after):
        assert (a == b).all()


def test_broadcast_values():
    """V rows of one head stride 0 (read only)."""
    n, hkv, d = 21, 3, 64
    st = Setup(d, "f32")
    k, v = normal((n, hkv, d), 1, "f32"), normal((n, 1, d), 2, "f32").expand(n, hkv, d)
    pos, before = positions(3, n, 3), orc.empty(5, hkv, d, 1)
    slots = places(n, 5, 3, together=True)
    gpu = on_gpu(before)
    pa.rotary_append(None, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, scales=gpu[2])
    check_rows(st, before, on_host(gpu), slots, k, v, pos, None)


def test_refusals():
    st = Setup(64, "bf16")
    n = 3
    q, k, v, pos = normal((n, 4, 64), 1, "bf16"), normal((n, 2, 64), 2, "bf16"), normal((n, 2, 64), 3, "bf16"), positions(3, n, 4)
    k8, v8, s8 = pa.empty_cache_e4m3(4, 2, 64, "cuda")
    slots = torch.zeros((n, 2), dtype=torch.int32, device="cuda")
    for kc, vc, sc in ((k8, v8, s8[:3]), (k8.view(torch.uint8), v8, s8), (v8, k8, s8), (k8, v8, s8.view(torch.uint8)),
                       pa.empty_cache_e4m3(4, 1, 64, "cuda"), pa.empty_cache_e4m3(4, 2, 128, "cuda"), (k8, v8, s8.cpu())):
        with pytest.raises((ValueError, TypeError)):
            pa.rotary_append(q, k, v, pos, slots, kc, vc, st.handle, scales=sc)
    with pytest.raises((ValueError, TypeError)):  # 8-bit caches without their scales
        pa.rotary_append(q, k, v, pos, slots, k8, v8, st.handle)
    with pytest.raises((ValueError, TypeError)):
        pa.rotary_append(q, k, None, pos, slots, k8, v8, st.handle, scales=s8)

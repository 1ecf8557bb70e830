"""rotary_fwd, rotary_bwd and rotary_append against their formulas in 64 bits,
at the sizes, strides, positions and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2608_06146_amd as pa
from paper_2608_06146_amd import _lib
from _rotary import Setup, check, f64, k_block_view, normal, positions, torch_dtype, v_block_view

pytestmark = pytest.mark.gpu

@pytest.fixture(autouse=True, params=["native", "python"])
def binding(request, monkeypatch):
    """Every test through the native module and without it."""
    if request.param == "python":
        monkeypatch.setattr(_lib, "native_rows", lambda: None)
        monkeypatch.setattr(pa, "_copy_blocks", lambda *a: None)
    else:
        assert _lib.native_rows() is not None, "the native module is not built"
    return request.param


HEADS = {"gqa": (16, 2), "seven": (28, 4), "odd": (5, 3), "many": (70, 33)}


def _say(*a):
    print("[case]", *a, flush=True)


def _fwd_bwd(st, n, hq, hkv, d, dtype, norm, pos=None, seed=0):
    q, k = normal((n, hq, d), seed + 1, dtype), normal((n, hkv, d), seed + 2, dtype)
    wq, wk = (normal((d,), seed + 3, dtype), normal((d,), seed + 4, dtype)) if norm else (None, None)
    gq, gk = normal((n, hq, d), seed + 5, dtype), normal((n, hkv, d), seed + 6, dtype)
    pos = positions(st.handle.n_axes, n, seed + 7) if pos is None else pos
    zq, zk = pa.rotary_fwd(q, k, pos, st.handle, wq, wk)
    check("q", zq, *st.forward(q, pos, wq))
    check("k", zk, *st.forward(k, pos, wk))
    dq, dk, dwq, dwk = pa.rotary_bwd(gq, gk, pos, st.handle, q, k, wq, wk)
    for name, dx, dw, g, x, w in (("dq", dq, dwq, gq, q, wq), ("dk", dk, dwk, gk, k, wk)):
        want, tol, dwant, dtol = st.backward(g, x, pos, w)
        check(name, dx, want, tol)
        assert (dw is None) == (w is None)
        if w is not None:
            check(name + "_weight", dw, dwant, dtol)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rd", [(128, 128), (128, 64), (128, 16), (64, 64), (64, 32), (64, 48)])
@pytest.mark.parametrize("style,axes,norm", [("halves", 3, True), ("halves", 1, False), ("pairs", 4, True), ("pairs", 1, False)])
def test_types_and_styles(dtype, d, rd, style, axes, norm):
    _say(dtype, d, rd, style, axes, norm)
    _fwd_bwd(Setup(d, dtype, rd, axes, style, scale=1.25), 37, 5, 3, d, dtype, norm)


@pytest.mark.parametrize("n", [1, 2, 15, 31, 32, 33, 64, 65, 700, 2500])
@pytest.mark.parametrize("heads", HEADS)
def test_lengths(n, heads):
    _say(n, heads)
    _fwd_bwd(Setup(128, "bf16"), n, *HEADS[heads], 128, "bf16", True, seed=n)


@pytest.mark.parametrize("d,n", [(128, 4500), (64, 9000)])
def test_long_runs_of_heads(d, n):
    """So many rows that a lane group takes several heads and a workgroup
    several runs of rows."""
    _say(d, n)
    _fwd_bwd(Setup(d, "bf16"), n, 4, 1, d, "bf16", True)


@pytest.mark.parametrize("style", ["halves", "pairs"])
def test_calls_past_the_caches(style, binding):
    """More than 128 MiB: forward, backward, append."""
    if binding == "python":
        pytest.skip("once")
    _say(style)
    st = Setup(128, "bf16", style=style)
    _fwd_bwd(st, 26500, 8, 2, 128, "bf16", True)
    _check_append(st, 16, 2, 128, "bf16", _runs((13300, 37), (5, 0), 850, 1), 850, True)


@pytest.mark.parametrize("far", [10 ** 6, 2 ** 31 - 5001, -2 ** 31, -77])
def test_far_positions(far):
    _say(far)
    _fwd_bwd(Setup(64, "f32", n_axes=3), 40, 2, 1, 64, "f32", False, positions(3, 40, 1, far))


def test_frequencies_given():
    freq = np.linspace(-9.0, 9.0, 32)  # negative ones and more than a turn a position
    st = Setup(64, "f32", n_axes=1)
    st.freq = freq
    st.handle = pa.Rotary(64, "f32", inv_freq=freq)
    _say("inv_freq")
    _fwd_bwd(st, 50, 2, 1, 64, "f32", False, positions(1, 50, 3))


def _fused(n, hq, hkv, d, dtype, seed, shift=0, extra=0):
    """q, k, v: slices of one projection's rows, `shift` elements past an aligned address."""
    w = (hq + 2 * hkv) * d + extra
    buf = normal((n * w + shift,), seed, dtype)
    x = buf[shift:].view(n, w)
    cut = [hq * d, (hq + hkv) * d, (hq + 2 * hkv) * d]
    return buf, x[:, :cut[0]].view(n, hq, d), x[:, cut[0]:cut[1]].view(n, hkv, d), x[:, cut[1]:cut[2]].view(n, hkv, d)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("shift,extra", [(0, 0), (1, 0), (3, 5), (8, 8)])
def test_slices_of_a_projection(dtype, shift, extra):
    _say(dtype, shift, extra)
    st, n, hq, hkv, d = Setup(64, dtype), 45, 7, 2, 64
    _, q, k, _ = _fused(n, hq, hkv, d, dtype, 1, shift, extra)
    pos = positions(3, n + 9, 2)[:, 4:4 + n]  # a window of longer axes
    wq, wk = normal((d + 3,), 3, dtype)[3:], normal((d + 3,), 4, dtype)[3:]
    zq, zk = pa.rotary_fwd(q, k, pos, st.handle, wq, wk)
    check("q", zq, *st.forward(q, pos, wq))
    check("k", zk, *st.forward(k, pos, wk))
    # the gradients into slices of the projection's gradient
    gq, gk = normal((n, hq, d), 5, dtype), normal((n, hkv, d), 6, dtype)
    dbuf, dq, dk, dv = _fused(n, hq, hkv, d, dtype, 7, shift, extra)
    before = dbuf.clone()
    pa.rotary_bwd(gq, gk, pos, st.handle, q, k, wq, wk, dq=dq, dk=dk)
    check("dq", dq, *st.backward(gq, q, pos, wq)[:2])
    check("dk", dk, *st.backward(gk, k, pos, wk)[:2])
    dq.copy_(torch.zeros_like(dq)), dk.copy_(torch.zeros_like(dk))
    _, bq, bk, _ = before, *[t for t in _views(before, n, hq, hkv, d, shift, extra)]
    bq.zero_(), bk.zero_()
    assert torch.equal(dbuf, before)  # nothing beside the slices was written


def _views(buf, n, hq, hkv, d, shift, extra):
    x = buf[shift:].view(n, (hq + 2 * hkv) * d + extra)
    return x[:, :hq * d].view(n, hq, d), x[:, hq * d:(hq + hkv) * d].view(n, hkv, d), x[:, (hq + hkv) * d:(hq + 2 * hkv) * d]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_other_orders(dtype):
    _say(dtype)
    st, n, hq, hkv, d = Setup(128, dtype, style="pairs"), 41, 6, 2, 128
    pos = positions(3, n, 1)
    wq, wk = normal((d,), 3, dtype), normal((d,), 4, dtype)
    buf, q, k, v = _fused(n, hq, hkv, d, dtype, 2)
    want = [st.forward(q, pos, wq), st.forward(k, pos, wk)]
    v0 = v.clone()
    zq, zk = pa.rotary_fwd(q, k, pos, st.handle, wq, wk, q_out=q, k_out=k)
    assert zq.data_ptr() == q.data_ptr() and torch.equal(v, v0)
    check("q", q, *want[0])
    check("k", k, *want[1])
    # heads before rows, and one head repeated by a stride of 0
    qt = normal((hq, n, d), 5, dtype).transpose(0, 1)
    kt = normal((n, 1, d), 6, dtype).expand(n, 3, d)
    out = torch.empty((hq, n, d), dtype=torch_dtype(dtype), device="cuda").transpose(0, 1)
    zq, zk = pa.rotary_fwd(qt, kt, pos, st.handle, wq, wk, q_out=out)
    check("q", out, *st.forward(qt, pos, wq))
    check("k", zk, *st.forward(kt, pos, wk))
    g = normal((n, hq, d), 7, dtype)
    want, tol, _, _ = st.backward(g, qt, pos, wq)
    dq, dk, dwq, dwk = pa.rotary_bwd(g, None, pos, st.handle, qt, None, wq, None, dq=g)
    assert dk is None and dwk is None and dwq is not None
    check("dq in place", g, want, tol)


@pytest.mark.parametrize("order", ["rows", "heads"])
def test_in_place_beside_other_heads(order):
    """q, k and v of a head side by side, rotated where they lie: the row and
    head strides are the same for all three, and their extents overlap."""
    st, n, h, d = Setup(64, "bf16"), 37, 5, 64
    pos, wq, wk = positions(3, n, 1), normal((d,), 3, "bf16"), normal((d,), 4, "bf16")
    buf = normal((n, h, 3, d) if order == "rows" else (h, 3, n, d), 5, "bf16")
    q, k, v = (buf[:, :, i] for i in range(3)) if order == "rows" else (buf[:, i].transpose(0, 1) for i in range(3))
    want, v0 = [st.forward(q, pos, wq), st.forward(k, pos, wk)], v.clone()
    pa.rotary_fwd(q, k, pos, st.handle, wq, wk, q_out=q, k_out=k)
    check("q", q, *want[0])
    check("k", k, *want[1])
    assert torch.equal(v, v0)
    gq, gk = normal((n, h, d), 6, "bf16"), normal((n, h, d), 7, "bf16")
    want = [st.backward(gq, q, pos, wq)[:2], st.backward(gk, k, pos, wk)[:2]]
    pa.rotary_bwd(gq, gk, pos, st.handle, q, k, wq, wk, dq=q, dk=k)
    check("dq", q, *want[0])
    check("dk", k, *want[1])
    assert torch.equal(v, v0)


def test_the_forwards_rows_become_their_gradients():
    st, n, d = Setup(64, "bf16"), 50, 64
    x, g, w, pos = normal((n, 3, d), 1, "bf16"), normal((n, 3, d), 2, "bf16"), normal((d,), 3, "bf16"), positions(3, n, 4)
    want, tol, dw, dtol = st.backward(g, x, pos, w)
    out = pa.rotary_bwd(g, None, pos, st.handle, x, None, w, dq=x)
    assert out[0].data_ptr() == x.data_ptr()
    check("dq", x, want, tol)
    check("dw", out[2], dw, dtol)


def test_one_position_for_every_axis():
    st, n, d = Setup(64, "f32"), 33, 64
    x, pos = normal((n, 2, d), 1, "f32"), positions(1, n, 2).expand(3, n)
    z, _ = pa.rotary_fwd(x, None, pos, st.handle)
    check("z", z, *st.forward(x, pos))


def test_two_streams_at_once():
    st, n, d = Setup(128, "bf16"), 9000, 128
    w, pos = normal((d,), 1, "bf16"), positions(3, n, 2)
    rows = [(normal((n, 4, d), 10 + i, "bf16"), normal((n, 4, d), 20 + i, "bf16")) for i in range(2)]
    run = lambda x, g: (pa.rotary_fwd(x, None, pos, st.handle, w)[0], *pa.rotary_bwd(g, None, pos, st.handle, x, None, w)[::2])  # noqa: E731
    want = [run(*r) for r in rows]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in rows]
    for _ in range(5):
        got = []
        for s, r in zip(streams, rows):
            with torch.cuda.stream(s):
                got.append(run(*r))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(got, want) for a, b in zip(x, y))


def test_more_rows_than_32_bits_address(binding):
    """Rows behind 2^33 elements, in more tiles than a launch has workgroups."""
    if binding == "python" or torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("once, and where there is room")
    st, part, times, d = Setup(64, "bf16", n_axes=1), 1 << 20, 135, 64
    n = part * times
    base, pos = normal((part, 1, d), 1, "bf16"), torch.arange(n, dtype=torch.int32, device="cuda")
    x = base.repeat(times, 1, 1)
    z, _ = pa.rotary_fwd(x, None, pos, st.handle)
    at = torch.cat([torch.arange(40), torch.arange(n - 40, n), torch.randint(0, n, (300,), generator=torch.Generator().manual_seed(2))]).cuda()
    check("rows", z[at], *st.forward(x[at], pos[at][None]))
    back = pa.rotary_bwd(z, None, pos, st.handle, dq=z)[0]  # turned back, in place: the rows, rounded twice
    # z is off by 2^-8 of itself, so the rows turned back by 2^-8 (|z_a| + |z_b|) <= 2^-8 sqrt(2) (|a| + |b|) and 2^-8 |a|
    for i in range(0, times, 15):
        err = (back[i * part:(i + 1) * part].float() - base.float()).abs()
        assert bool((err <= 2.0 ** -7 * 1.5 * (base.float().abs() + base.float().roll(32, -1).abs())).all()), i


@pytest.mark.parametrize("which", ["q", "k"])
def test_one_of_the_two(which):
    _say(which)
    st, n, d = Setup(64, "bf16"), 77, 64
    x, g, w = normal((n, 3, d), 1, "bf16"), normal((n, 3, d), 2, "bf16"), normal((d,), 3, "bf16")
    pos = positions(3, n, 4)
    pick = (lambda t: (t, None)) if which == "q" else (lambda t: (None, t))
    z = pa.rotary_fwd(*pick(x), pos, st.handle, *pick(w))
    check("z", z[0 if which == "q" else 1], *st.forward(x, pos, w))
    out = pa.rotary_bwd(*pick(g), pos, st.handle, *pick(x), *pick(w))
    want, tol, dw, dtol = st.backward(g, x, pos, w)
    at = 0 if which == "q" else 1
    check("dx", out[at], want, tol)
    check("dw", out[2 + at], dw, dtol)
    assert out[1 - at] is None and out[3 - at] is None
    # a weight on one side only
    zq, zk = pa.rotary_fwd(x, x, pos, st.handle, *pick(w))
    check("q", zq, *st.forward(x, pos, w if which == "q" else None))
    check("k", zk, *st.forward(x, pos, w if which == "k" else None))
    dq, dk, dwq, dwk = pa.rotary_bwd(g, g, pos, st.handle, *pick(x), *pick(w))
    check("dq", dq, *st.backward(g, x, pos, w if which == "q" else None)[:2])
    check("dk", dk, *st.backward(g, x, pos, w if which == "k" else None)[:2])
    none = pa.rotary_bwd(g, g, pos, st.handle, *pick(x), *pick(w), weight_grads=False)
    assert none[2] is None and none[3] is None
    assert torch.equal(none[0], dq) and torch.equal(none[1], dk)


def test_no_rows():
    st = Setup(64, "bf16")
    x, pos, w = torch.empty((0, 3, 64), dtype=torch.bfloat16, device="cuda"), positions(3, 0, 1), normal((64,), 1, "bf16")
    zq, zk = pa.rotary_fwd(x, x, pos, st.handle, w, w)
    assert zq.shape == (0, 3, 64) and zk.shape == (0, 3, 64)
    dq, dk, dwq, dwk = pa.rotary_bwd(x, x, pos, st.handle, x, x, w, w)
    assert dq.shape == (0, 3, 64) and not dwq.any() and not dwk.any()


def test_values_at_the_edge():
    """Zero rows under a norm, rows of one huge value, infinities and NaN that
    stay in the head (without a norm: in the pair) they are in."""
    st, n, d = Setup(128, "f32", 64, 1), 9, 128
    pos, w = positions(1, n, 1), normal((d,), 2, "f32")
    x = normal((n, 2, d), 3, "f32")
    x[0, 0] = 0
    x[1, 1] = 0
    x[1, 1, 5] = 1e15
    x[2, 0] = 1e-20
    x[3, 0, 100] = float("inf")
    x[4, 1, 3] = float("nan")
    g = normal((n, 2, d), 4, "f32")
    hit = np.zeros((n, 2), bool)
    hit[3, 0] = hit[4, 1] = True
    y = x.clone()
    y[3, 0], y[4, 1] = 0, 0
    z, _ = pa.rotary_fwd(x, None, pos, st.handle, w)
    want, tol = st.forward(y, pos, w)
    check("z", torch.where(torch.from_numpy(hit).cuda()[..., None], 0.0, z), np.where(hit[..., None], 0, want), tol)
    assert not torch.isfinite(z[4, 1]).any() and torch.isnan(z[3, 0, 100])
    dx = pa.rotary_bwd(g, None, pos, st.handle, x, None, w, weight_grads=False)[0]
    want, tol = st.backward(g, y, pos, w)[:2]
    check("dx", torch.where(torch.from_numpy(hit).cuda()[..., None], 0.0, dx), np.where(hit[..., None], 0, want), tol)
    z, _ = pa.rotary_fwd(x, None, pos, st.handle)
    bad = ~np.isfinite(f64(z))
    want = np.zeros_like(bad)
    want[3, 0, 100] = want[4, 1, 3] = want[4, 1, 35] = True
    assert np.array_equal(bad, want)
    assert torch.equal(z[..., 64:], x[..., 64:])  # dimensions that are not rotated keep their bits


def test_runs_are_equal():
    """The weights' gradients are summed in an order that depends on sizes alone."""
    st, n, d = Setup(128, "bf16"), 3000, 128
    q, k, g, h = (normal((n, c, d), c, "bf16") for c in (16, 2, 16, 2))
    pos, w = positions(3, n, 1), normal((d,), 2, "bf16")
    runs = [pa.rotary_bwd(g, h, pos, st.handle, q, k, w, w) for _ in range(3)]
    for other in runs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(runs[0], other))


def test_gradient_against_differences():
    """The backward of the forward as it is: central differences in fp32."""
    st, n, d = Setup(64, "f32", 32, 3, "pairs", scale=0.9), 3, 64
    x, pos, w = normal((n, 2, d), 1, "f32"), positions(3, n, 2), normal((d,), 3, "f32")
    g = normal((n, 2, d), 4, "f32")
    dx, _, dw, _ = pa.rotary_bwd(g, None, pos, st.handle, x, None, w)
    loss = lambda a, b: float((pa.rotary_fwd(a, None, pos, st.handle, b)[0].double() * g.double()).sum())  # noqa: E731
    step = 2.0 ** -7
    for i in range(12):
        v = normal(x.shape, 10 + i, "f32") if i < 8 else torch.zeros_like(x)
        u = normal(w.shape, 30 + i, "f32") if i >= 8 else torch.zeros_like(w)
        slope = (loss(x + step * v, w + step * u) - loss(x - step * v, w - step * u)) / (2 * step)
        want = float((dx.double() * v.double()).sum() + (dw.double() * u.double()).sum())
        # 384 values: third derivatives of order 1, 3 step^2 each at most; values off by 32 u (|y_a| + |y_b|), 64 u / step
        assert abs(slope - want) <= 384 * (3 * step ** 2 + 64 * 2 ** -24 / step), (i, slope, want)


# ------------------------------------------------------------------ append

def _slots(n, nb, seed, block=16):
    rng = np.random.default_rng(seed)
    s = rng.permutation(nb * block)[:n]
    return np.stack([s // block, s % block], 1).astype(np.int32)


def _check_append(st, hq, hkv, d, dtype, slots, nb, norm, seed=0, shift=0, n_q=None, stream=None):
    n = len(slots)
    n_q = n if n_q is None else n_q
    _, q, k, v = _fused(n, hq, hkv, d, dtype, seed + 1, shift)
    if n_q != n:
        q = normal((n_q, hq, d), seed + 2, dtype)
    pos = positions(st.handle.n_axes, n, seed + 3)
    qpos = None if n_q == n else positions(st.handle.n_axes, n_q, seed + 4)
    wq, wk = (normal((d,), seed + 5, dtype), normal((d,), seed + 6, dtype)) if norm else (None, None)
    kc, vc = normal((nb, hkv, d // 8, 16, 8), seed + 7, dtype), normal((nb, hkv, d, 16), seed + 8, dtype)
    k0, v0 = kc.clone(), vc.clone()
    out = pa.rotary_append(q, k, v, pos, torch.from_numpy(slots).cuda(), kc, vc, st.handle, wq, wk, q_positions=qpos)
    torch.cuda.synchronize()
    check("q", out, *st.forward(q, pos if qpos is None else qpos, wq))
    keep = (slots[:, 0] >= 0) & (slots[:, 0] < nb) & (slots[:, 1] >= 0) & (slots[:, 1] < 16)
    b, t = slots[keep, 0], slots[keep, 1]
    want, tol = st.forward(k, pos, wk)
    check("k", k_block_view(kc)[b, :, t], want[keep], tol[keep])
    assert torch.equal(v_block_view(vc)[b, :, t], v[torch.from_numpy(keep).cuda()])
    # everything else as it was
    for now, was in ((k_block_view(kc).clone(), k_block_view(k0).clone()), (v_block_view(vc).clone(), v_block_view(v0).clone())):
        now[b, :, t] = 0
        was[b, :, t] = 0
        assert torch.equal(now, was)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,style,axes,norm", [(128, "halves", 3, True), (128, "pairs", 1, False), (64, "halves", 1, True), (64, "pairs", 3, False)])
@pytest.mark.parametrize("n", [1, 17, 70])
def test_append_scattered(dtype, d, style, axes, norm, n):
    _say(dtype, d, style, axes, norm, n)
    _check_append(Setup(d, dtype, None, axes, style), 6, 2, d, dtype, _slots(n, 30, n), 30, norm, shift=n % 3)


def _runs(lengths, firsts, nb, seed):
    """Slots of streams that append runs of tokens at lengths firsts, in blocks of their own."""
    rng = np.random.default_rng(seed)
    free = list(rng.permutation(nb))
    out = []
    for n, f in zip(lengths, firsts):
        blocks = [free.pop() for _ in range((f + n + 15) // 16)]
        out += [(blocks[p // 16], p % 16) for p in range(f, f + n)]
    return np.array(out, np.int32).reshape(-1, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lengths,firsts", [
    ((16,), (0,)), ((8,), (8,)), ((7,), (9,)), ((64, 64), (0, 0)), ((63, 65, 1, 130), (0, 5, 15, 11)),
    ((1, 1, 40, 1, 9, 8, 8), (0, 8, 3, 7, 15, 0, 1)), ((300, 301), (1, 0))])
def test_append_runs(dtype, d, lengths, firsts):
    _say(dtype, d, lengths, firsts)
    nb = sum((n + f + 15) // 16 for n, f in zip(lengths, firsts)) + 3
    _check_append(Setup(d, dtype), 4, 3, d, dtype, _runs(lengths, firsts, nb, 1), nb, True, n_q=sum(lengths) // 2 + 1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_append_padding_and_order(dtype):
    """Rows left out among runs, a run downwards, slots outside a block."""
    _say(dtype)
    s = _runs((40, 33), (0, 6), 20, 2)
    s[5] = (-1, 3)
    s[20:23, 0] = 20
    s[30, 1] = 16
    s[31, 1] = -1
    s[41:49] = s[41:49][::-1].copy()
    s[60:62] = -1
    _check_append(Setup(128, dtype), 4, 1, 128, dtype, s, 20, True)
    _check_append(Setup(64, dtype), 4, 1, 64, dtype, np.full((9, 2), -1, np.int32), 5, True)


def test_append_long():
    """A prefill of several thousand tokens of three streams."""
    _say("long")
    lengths, firsts = (2557, 1031, 700), (0, 3, 8)
    _check_append(Setup(128, "bf16"), 4, 2, 128, "bf16", _runs(lengths, firsts, 300, 1), 300, True)


def test_append_many_heads_and_queries_in_place():
    _say("many heads")
    _check_append(Setup(64, "bf16"), 70, 33, 64, "bf16", _runs((9, 30), (3, 0), 5, 1), 5, True)
    st, n, d = Setup(128, "bf16", style="pairs"), 20, 128
    buf, q, k, v = _fused(n, 4, 2, d, "bf16", 1)
    pos, w, s = positions(3, n, 2), normal((d,), 3, "bf16"), torch.from_numpy(_slots(n, 4, 4)).cuda()
    kc, vc = torch.zeros((4, 2, 16, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 2, d, 16), dtype=torch.bfloat16, device="cuda")
    want, k0 = st.forward(q, pos, w), k.clone()
    out = pa.rotary_append(q, k, v, pos, s, kc, vc, st.handle, w, w, q_out=q)
    assert out.data_ptr() == q.data_ptr() and torch.equal(k, k0)
    check("q", q, *want)


def test_append_keys_alone():
    st, n, d = Setup(64, "bf16"), 20, 64
    k, v, pos = normal((n, 2, d), 1, "bf16"), normal((n, 1, d), 2, "bf16").expand(n, 2, d), positions(3, n, 3)
    kc, vc = torch.zeros((4, 2, 8, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((4, 2, d, 16), dtype=torch.bfloat16, device="cuda")
    s = _slots(n, 4, 5)
    assert pa.rotary_append(None, k, v, pos, torch.from_numpy(s).cuda(), kc, vc, st.handle) is None
    want, tol = st.forward(k, pos)
    check("k", k_block_view(kc)[s[:, 0], :, s[:, 1]], want, tol)
    assert torch.equal(v_block_view(vc)[s[:, 0], :, s[:, 1]], v)


# ---------------------------------------------------- streams and graphs

def test_on_another_stream_and_in_a_graph():
    """Every call captured into one graph and replayed with new inputs, the
    program's own work between the replays."""
    st, n, hq, hkv, d = Setup(128, "bf16"), 75, 4, 2, 128
    pos, w = positions(3, n, 1), normal((d,), 2, "bf16")
    s = torch.from_numpy(_slots(n, 12, 3)).cuda()
    pairs = torch.tensor([[i, 12 + i] for i in range(12)], dtype=torch.int32, device="cuda")
    buf, q, k, v = _fused(n, hq, hkv, d, "bf16", 4)
    g, h = normal((n, hq, d), 5, "bf16"), normal((n, hkv, d), 6, "bf16")
    kc, vc = torch.zeros((24, hkv, d // 8, 16, 8), dtype=torch.bfloat16, device="cuda"), torch.zeros((24, hkv, d, 16), dtype=torch.bfloat16, device="cuda")

    def run():
        fwd = pa.rotary_fwd(q, k, pos, st.handle, w, w)
        bwd = pa.rotary_bwd(g, h, pos, st.handle, q, k, w, w)
        out = pa.rotary_append(q, k, v, pos, s, kc, vc, st.handle, w, w)
        pa.cache_copy_blocks(kc, vc, pairs)
        return [*fwd, *bwd, out, kc, vc]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for i in range(4):
        buf.copy_(normal(buf.shape, 20 + i, "bf16"))
        g.copy_(normal(g.shape, 40 + i, "bf16"))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        kc.zero_(), vc.zero_()
        want = run()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


def test_a_stream_of_the_callers():
    st, n, d = Setup(64, "bf16"), 5000, 64
    q, g, w, pos = normal((n, 8, d), 1, "bf16"), normal((n, 8, d), 2, "bf16"), normal((d,), 3, "bf16"), positions(3, n, 4)
    want = pa.rotary_fwd(q, None, pos, st.handle, w)[0], *pa.rotary_bwd(g, None, pos, st.handle, q, None, w)
    side = torch.cuda.Stream()
    for _ in range(3):
        side.wait_stream(torch.cuda.current_stream())
        got = pa.rotary_fwd(q, None, pos, st.handle, w, stream=side)[0], *pa.rotary_bwd(g, None, pos, st.handle, q, None, w, stream=side)
        junk = [torch.full((256, 1024), 3.0, device="cuda") for _ in range(4)]  # memory the calls let go of is not theirs yet
        torch.cuda.current_stream().wait_stream(side)
        assert all(a is None and b is None or torch.equal(a, b) for a, b in zip(got, want)) and len(junk) == 4


# ---------------------------------------------------------------- refusals

def _call(what="fwd", **kw):
    st, n, d = kw.pop("st", None) or Setup(64, "bf16"), 6, 64
    a = {"q": normal((n, 4, d), 1, "bf16"), "k": normal((n, 2, d), 2, "bf16"), "v": normal((n, 2, d), 3, "bf16"),
         "positions": positions(3, n, 4), "q_weight": normal((d,), 5, "bf16"), "k_weight": normal((d,), 6, "bf16"),
         "gq": normal((n, 4, d), 7, "bf16"), "gk": normal((n, 2, d), 8, "bf16"), "q_out": None,
         "slots": torch.from_numpy(_slots(n, 3, 1)).cuda(), "q_positions": None,
         "kc": torch.zeros((3, 2, 8, 16, 8), dtype=torch.bfloat16, device="cuda"),
         "vc": torch.zeros((3, 2, d, 16), dtype=torch.bfloat16, device="cuda")}
    a.update(kw)
    if what == "fwd":
        return pa.rotary_fwd(a["q"], a["k"], a["positions"], st.handle, a["q_weight"], a["k_weight"], a["q_out"])
    if what == "bwd":
        return pa.rotary_bwd(a["gq"], a["gk"], a["positions"], st.handle, a["q"], a["k"], a["q_weight"], a["k_weight"], dq=a["q_out"])
    return pa.rotary_append(a["q"], a["k"], a["v"], a["positions"], a["slots"], a["kc"], a["vc"], st.handle, a["q_weight"],
                            a["k_weight"], a["q_positions"], a["q_out"])


BAD = {  # argument: values that no call takes
    "q": [lambda t: t.float(), lambda t: t.cpu(), lambda t: t[:, :, :32], lambda t: t[:5], lambda t: t[0],
          lambda t: torch.empty((64, 4, 6), dtype=t.dtype, device="cuda").permute(2, 1, 0), lambda t: t[0, 0, 0]],
    "k": [lambda t: t.float(), lambda t: t.cpu(), lambda t: t[:5]],
    "positions": [lambda t: t.long(), lambda t: t.cpu(), lambda t: t[:2], lambda t: t[:, :5], lambda t: t[0],
                  lambda t: torch.stack([t, t], -1)[..., 0]],
    "q_weight": [lambda t: t.float(), lambda t: t.cpu(), lambda t: t[:32], lambda t: torch.stack([t, t], -1)[:, 0]],
    "q_out": [lambda t: torch.empty((6, 4, 64), device="cuda"), lambda t: torch.empty((6, 3, 64), dtype=torch.bfloat16, device="cuda"),
              lambda t: torch.empty((6, 1, 64), dtype=torch.bfloat16, device="cuda").expand(6, 4, 64)],
    "gq": [lambda t: t.float(), lambda t: t[:5], lambda t: t[0, 0, 0]],
    "v": [lambda t: t.float(), lambda t: t[:5], lambda t: t[:, :1]],
    "slots": [lambda t: t.long(), lambda t: t[:5], lambda t: t.t().contiguous(), lambda t: t.cpu()],
    "kc": [lambda t: t.float(), lambda t: t[:2], lambda t: t.transpose(2, 3)],
    "vc": [lambda t: t.float(), lambda t: t[:, :1], lambda t: t.transpose(2, 3).contiguous()],
    "q_positions": [lambda t: positions(3, 5, 1)],
}
USED = {"fwd": ("q", "k", "positions", "q_weight", "q_out"), "bwd": ("q", "k", "positions", "q_weight", "q_out", "gq"),
        "append": ("q", "k", "positions", "q_weight", "q_out", "v", "slots", "kc", "vc", "q_positions")}


@pytest.mark.parametrize("what", USED)
def test_refusals(what):
    st = Setup(64, "bf16")
    _call(what, st=st)
    for name in USED[what]:
        for i, spoil in enumerate(BAD[name]):
            if what == "append" and name == "q" and i == 3:
                continue  # fewer queries than new rows: refused for its positions below
            base = {"q": normal((6, 4, 64), 1, "bf16"), "k": normal((6, 2, 64), 2, "bf16"), "v": normal((6, 2, 64), 2, "bf16"),
                    "positions": positions(3, 6, 4), "q_weight": normal((64,), 5, "bf16"), "gq": normal((6, 4, 64), 7, "bf16"),
                    "slots": torch.from_numpy(_slots(6, 3, 1)).cuda(), "kc": torch.zeros((3, 2, 8, 16, 8), dtype=torch.bfloat16, device="cuda"),
                    "vc": torch.zeros((3, 2, 64, 16), dtype=torch.bfloat16, device="cuda")}.get(name)
            with pytest.raises((ValueError, TypeError, pa.PadocError)):
                _call(what, st=st, **{name: spoil(base)})
                print("taken:", what, name, i, flush=True)
    if what == "append":
        with pytest.raises(pa.PadocError, match="q_pos"):
            _call(what, st=st, q=normal((5, 4, 64), 1, "bf16"))
        with pytest.raises((ValueError, AttributeError)):
            _call(what, st=st, v=None)
    with pytest.raises(ValueError, match="stream"):
        class Elsewhere:
            device, cuda_stream = torch.device("cuda", 7), 0
        pa.rotary_fwd(normal((6, 4, 64), 1, "bf16"), None, positions(3, 6, 4), st.handle, stream=Elsewhere)


def test_a_closed_handle_is_refused():
    st = Setup(64, "bf16")
    st.handle.close()
    for what in USED:
        with pytest.raises(ValueError, match="closed"):
            _call(what, st=st)


def test_a_flag_without_a_truth_value():
    st = Setup(64, "bf16")
    q, w, pos = normal((6, 4, 64), 1, "bf16"), normal((64,), 2, "bf16"), positions(3, 6, 3)
    with pytest.raises(RuntimeError, match="ambiguous"):
        pa.rotary_bwd(q, None, pos, st.handle, q, None, w, weight_grads=torch.ones(2))

"""rotary_append into 8-bit caches with a head norm, over rows whose mean square
is 0, infinite, NaN or far from 1, with and without an eps."""
import numpy as np
import pytest
import torch

from oracle import e4m3 as orc
import paper_2608_06146_amd as pa
from _e4m3 import on_gpu, on_host
from _rotary import Setup, f64, normal, positions, torch_dtype

pytestmark = pytest.mark.gpu


def special_rows(n, hkv, d, dtype):
    """Drawn rows, the first ten of a kind each."""
    x = normal((n, hkv, d), 31, dtype, device="cpu", spread=3.0)
    t = torch_dtype(dtype)
    top, low = torch.finfo(t).max, 2.0 ** (-149 if dtype == "f32" else -133)
    sign = torch.where(x < 0, -1.0, 1.0).to(t)
    x[0] = 0
    x[1] = -0.0
    x[2] = sign[2] * top                       # mean square 2^256: past fp32
    x[3] = sign[3] * low                       # the smallest numbers: 2^-298
    x[4] = (x[4].double() * 2.0 ** -80).to(t)  # mean square 2^-160
    x[5] = 0
    x[5, :, 7] = top                           # one number in a row
    x[6, 0, d - 1] = float("inf")
    x[7, hkv - 1, 0] = float("-inf")
    x[8, 0, d // 2] = float("nan")
    x[9, :, 1], x[9, :, 2] = float("inf"), float("-inf")
    return x.cuda()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,style", [(128, "halves"), (64, "halves"), (128, "pairs"), (64, "pairs")])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("n,hkv", [(40, 2), (3100, 2)])
def test_norms_of_every_kind(n, hkv, d, style, eps, dtype):
    """K's codes and scales bit for bit those of the 64-bit formula (z is within 2^-36 of its pair's magnitude, and no
    value that is drawn lies that close to a border: a chance of 800,000 x 2^-36 / 2^-4 = 2e-4); rows without a finite
    value in the formula are NaN, and the rows beside them as ever.  Byte by byte and with V staged."""
    st = Setup(d, dtype, style=style, base=1e6, scale=1.25, eps=eps)
    k, v = special_rows(n, hkv, d, dtype), normal((n, hkv, d), 32, dtype)
    wk, pos = normal((d,), 33, dtype), positions(3, n, 34, far=1)
    blocks = n // 16 + 5
    p = np.random.default_rng(35).permutation(blocks * 16)[:n]
    slots = np.stack([p // 16, p % 16], 1).astype(np.int32)
    before = orc.empty(blocks, hkv, d, 36)
    gpu = on_gpu(before)
    print("[case] append e4m3 norms of every kind", dtype, d, style, eps, n, flush=True)
    pa.rotary_append(None, k, v, pos, torch.from_numpy(slots).cuda(), *gpu[:2], st.handle, None, wk, scales=gpu[2])
    torch.cuda.synchronize()
    want = [w.copy() for w in before]
    with np.errstate(all="ignore"):
        z = st.forward(k, pos, wk)[0]
    finite = np.isfinite(z).all(-1)
    assert (~finite).sum() == (2 * hkv if eps == 0 else 0) + 3 + hkv and finite[2:6].all()
    orc.write(want, slots[:, 0], slots[:, 1], z, f64(v))
    for name, a, w in zip(("k", "v", "scales"), on_host(gpu), want):
        zero = (a & 127 == 0) & (w & 127 == 0) if name == "k" else False  # (of a zero, the sign is free)
        bad = ~((a == w) | zero)
        assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:4].tolist(), a[bad][:4], w[bad][:4])

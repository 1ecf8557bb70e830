"""cache_copy_blocks: whole blocks to other blocks, bit for bit, nothing else
written."""
import numpy as np
import pytest
import torch

import paper_2608_06146_amd as pa
from _rotary import normal

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True, params=["native", "python"])
def binding(request, monkeypatch):
    if request.param == "python":
        monkeypatch.setattr(pa, "_copy_blocks", lambda *a: None)


def _caches(nb, hkv, d, dtype, seed):
    return normal((nb, hkv, d // 8, 16, 8), seed, dtype), normal((nb, hkv, d, 16), seed + 1, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,hkv", [(64, 1), (64, 5), (128, 2), (128, 3)])
@pytest.mark.parametrize("n", [0, 1, 24, 301])
def test_within_a_cache(dtype, d, hkv, n):
    print("[case]", dtype, d, hkv, n, flush=True)
    nb = 2 * n + 5
    kc, vc = _caches(nb, hkv, d, dtype, 1)
    ids = np.random.default_rng(n).permutation(nb)[:2 * n].reshape(-1, 2).astype(np.int32)
    ids[n // 2:, 0] = ids[n // 2:, 0][:1] if n else 0  # one block forked many times
    want = [c.clone() for c in (kc, vc)]
    for c in want:
        c[ids[:, 1]] = c[ids[:, 0]]
    out = pa.cache_copy_blocks(kc, vc, torch.from_numpy(ids).cuda(), pairs_host=ids)
    assert out[0] is kc and out[1] is vc
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])
    back = torch.from_numpy(ids[n // 2:, ::-1].copy()[:1]).cuda()  # one back, without the host's copy
    pa.cache_copy_blocks(kc, vc, back)
    assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])


def test_refusals():
    kc, vc = _caches(4, 2, 64, "bf16", 1)
    pairs = torch.tensor([[0, 1]], dtype=torch.int32, device="cuda")
    for k, v, p in ((kc.float(), vc, pairs), (kc, vc[:3], pairs), (kc, vc, pairs.long()), (kc, vc, pairs[0]), (kc, vc, pairs.cpu()),
                    (kc.transpose(2, 3), vc, pairs), (kc.half(), vc.half(), pairs), (kc, vc.transpose(2, 3).contiguous(), pairs),
                    (vc, kc, pairs), (kc.cpu(), vc, pairs)):
        with pytest.raises((ValueError, TypeError)):
            pa.cache_copy_blocks(k, v, p)
    with pytest.raises(ValueError):
        pa.cache_copy_blocks(kc, vc, pairs, k_dst=kc)
    with pytest.raises(ValueError):
        pa.cache_copy_blocks(kc, vc, pairs, *_caches(4, 1, 64, "bf16", 1))
    with pytest.raises(ValueError):
        pa.cache_copy_blocks(kc, vc, pairs, pairs_host=np.zeros((2, 2), np.int32))


def test_to_another_cache_with_ids_outside():
    """Another pool of another size; pairs outside either pool are left out."""
    a, b = _caches(9, 2, 64, "bf16", 1), _caches(5, 2, 64, "bf16", 7)
    ids = np.array([[8, 0], [-1, 1], [9, 2], [3, 5], [3, -1], [3, 4], [2 ** 31 - 1, 3], [0, -2 ** 31]], np.int32)
    want = [c.clone() for c in b]
    for w, s in zip(want, a):
        w[0], w[4] = s[8], s[3]
    src = [c.clone() for c in a]
    pa.cache_copy_blocks(*a, torch.from_numpy(ids).cuda(), *b)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip([*a, *b], [*src, *want]))
    with pytest.raises(pa.PadocError, match="outside"):
        pa.cache_copy_blocks(*a, torch.from_numpy(ids).cuda(), *b, pairs_host=ids)


def test_a_block_past_32_bits():
    """Blocks whose first byte lies behind 2^32."""
    hkv, d = 8, 128
    nb = 2 ** 32 // (hkv * 16 * d * 4) + 70  # fp32: one tensor is a little more than 4 GiB
    kc = torch.zeros((nb, hkv, d // 8, 16, 8), device="cuda")
    vc = torch.zeros((nb, hkv, d, 16), device="cuda")
    kc[3], vc[3] = 1.5, 2.5
    pairs = np.array([[3, nb - 1], [3, nb - 66]], np.int32)
    pa.cache_copy_blocks(kc, vc, torch.from_numpy(pairs).cuda(), pairs_host=pairs)
    assert bool((kc[nb - 1] == 1.5).all()) and bool((vc[nb - 66] == 2.5).all())
    assert float(kc.sum(dtype=torch.float64)) == 3 * 1.5 * hkv * 16 * d and float(vc.sum(dtype=torch.float64)) == 3 * 2.5 * hkv * 16 * d
    # and rows appended there
    rot = pa.Rotary(d, "f32")
    k, v = torch.ones((2, hkv, d), device="cuda"), torch.full((2, hkv, d), 7.0, device="cuda")
    slots = torch.tensor([[nb - 2, 15], [nb - 1, 0]], dtype=torch.int32, device="cuda")
    pa.rotary_append(None, k, v, torch.zeros((1, 2), dtype=torch.int32, device="cuda"), slots, kc, vc, rot)
    assert bool((vc[nb - 2, :, :, 15] == 7).all()) and bool((vc[nb - 1, :, :, 0] == 7).all())
    assert bool((kc[nb - 2, :, :, 15] == 1).all()) and bool((kc[nb - 1, :, :, 0] == 1).all())

"""Cases and bounds shared by the rotary tests.

Bounds (u = 2^-24, half a step of fp32, relative).  A norm: the square sum of a
row adds 16 values in a lane and 2 or 3 levels over lanes (19 roundings and
one of each square, halved by the root: 10), rsqrt and two products 4.  A
cosine or sine is off by 7 at most (angle 3, polynomial 4), its scale 1, the
two products and their sum 3.  Together below 32, times scale (|y_a| + |y_b|).
The reference's angles are products in 64 bits of a position and a frequency
that the library computed itself: 3 half steps (2^-53) of the largest angle.
A bf16 result is rounded once more, by 2^-8 of itself at most.

A weight's gradient adds its terms (off by 28 each) in fp32: in a lane, over
the lanes, wavefronts and workgroups, in these tests at most 160 in a row.
"""
import numpy as np
import torch

from oracle import rotary as orc

U = 2.0 ** -24
AXES = {1: lambda p: [0] * p, 3: lambda p: [0] * (p - 3 * p // 4) + [1 + i % 2 for i in range(3 * p // 4)],
        4: lambda p: [i % 4 for i in range(p)]}


def torch_dtype(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def normal(shape, seed, dtype, device="cuda", spread=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * spread).to(torch_dtype(dtype)).to(device)


def f64(t):
    return t.detach().double().cpu().numpy()


def positions(n_axes, n, seed, far=0):
    g = torch.Generator().manual_seed(seed)
    return (far + torch.randint(0, 5000, (n_axes, n), generator=g)).to(torch.int32).to("cuda")


def bound(mag, z, dtype, pos, freq, roundings=32):
    far = 3 * 2.0 ** -53 * float(np.abs(pos.cpu().numpy().astype(np.float64)).max(initial=0)) * float(np.abs(freq).max())
    b = (roundings * U + far) * mag
    if dtype == "bf16":
        b = b + 2.0 ** -8 * (np.abs(z) + b)
    return b + 1e-38  # the smallest normal number: results below it round coarser


def check(name, got, want, tol):
    got = f64(got)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[:3].tolist(), got[bad][:3], want[bad][:3], tol[bad][:3])


class Setup:
    """A handle and everything the reference needs to know of it."""

    def __init__(self, d, dtype, rotary_dim=None, n_axes=3, style="halves", base=10000.0, scale=1.0, eps=1e-6):
        import paper_2608_06146_amd as pa
        self.rd, self.style, self.scale, self.eps, self.dtype = rotary_dim or d, style, scale, eps, dtype
        self.axis = AXES[n_axes](self.rd // 2)
        self.freq = orc.frequencies(self.rd, base)
        self.handle = pa.Rotary(d, dtype, rotary_dim=self.rd, axis=self.axis, base=base, style=style, scale=scale, eps=eps)

    def forward(self, x, pos, w=None):
        z, mag = orc.rotary_forward(f64(x), pos.cpu().numpy(), self.axis, self.freq, self.rd, self.style, self.scale,
                                    None if w is None else f64(w), self.eps)
        return z, bound(mag, z, self.dtype, pos, self.freq)

    def backward(self, dz, x, pos, w=None):
        dx, mag, dw, dwmag = orc.rotary_backward(f64(dz), None if x is None else f64(x), pos.cpu().numpy(), self.axis,
                                                 self.freq, self.rd, self.style, self.scale,
                                                 None if w is None else f64(w), self.eps)
        tol = bound(mag, dx, self.dtype, pos, self.freq)
        return dx, tol, dw, None if dw is None else bound(dwmag, dw, "f32", pos, self.freq, 28 + 160)


def k_block_view(kc):
    """K cache [blocks, Hkv, d/8, 16, 8] as [blocks, Hkv, 16 tokens, d]."""
    slot = [0, 1, 2, 3, 8, 9, 10, 11, 4, 5, 6, 7, 12, 13, 14, 15]
    nb, h, c, _, _ = kc.shape
    return kc[:, :, :, slot].permute(0, 1, 3, 2, 4).reshape(nb, h, 16, 8 * c)


def v_block_view(vc):
    """V cache [blocks, Hkv, d, 16] as [blocks, Hkv, 16 tokens, d]."""
    return vc.transpose(2, 3)

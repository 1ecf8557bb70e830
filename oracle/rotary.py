"""Head norms and rotary positions in 64 bits (numpy), from their formulas.

A head's row x of d values: y = w x / sqrt(mean x^2 + eps) (y = x without a
weight); pair i of the first ``rotary_dim`` dimensions, members (a, b), is
turned by the angle pos[axis[i]] * inv_freq[i] and scaled.  Beside each result
stands the magnitude its rounding errors scale with.
"""
from __future__ import annotations

import numpy as np


def members(rotary_dim: int, style: str):
    """Dimensions of the two members of every pair."""
    i = np.arange(rotary_dim // 2)
    return (i, i + rotary_dim // 2) if style == "halves" else (2 * i, 2 * i + 1)


def frequencies(rotary_dim: int, base: float) -> np.ndarray:
    return np.array([float(base) ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)])


def _turn(y, pos, axis, freq, rotary_dim, style, scale, sign):
    """Rotated rows, and per element scale * (|y_a| + |y_b|) (|y| where not
    rotated).  pos [n_axes, n]; y [n, H, d]."""
    ang = (pos[np.asarray(axis)].astype(np.float64).T * freq)[:, None, :]   # [n, 1, pairs]
    c, s = np.cos(ang) * scale, sign * np.sin(ang) * scale
    a, b = members(rotary_dim, style)
    z, mag = y.copy(), np.abs(y)
    z[..., a] = y[..., a] * c - y[..., b] * s
    z[..., b] = y[..., b] * c + y[..., a] * s
    both = abs(scale) * (np.abs(y[..., a]) + np.abs(y[..., b]))
    mag[..., a] = both
    mag[..., b] = both
    return z, mag


def rotary_forward(x, pos, axis, freq, rotary_dim, style="halves", scale=1.0, weight=None, eps=1e-6):
    """``(z, magnitude)`` of rows x [n, H, d]."""
    y = np.asarray(x, np.float64)
    if weight is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    return _turn(y, np.asarray(pos), axis, freq, rotary_dim, style, scale, 1.0)


def rotary_backward(dz, x, pos, axis, freq, rotary_dim, style="halves", scale=1.0, weight=None, eps=1e-6):
    """``(dx, magnitude, dw, magnitude)`` of sum(dz * z)."""
    dy, mag = _turn(np.asarray(dz, np.float64), np.asarray(pos), axis, freq, rotary_dim, style, scale, -1.0)
    if weight is None:
        return dy, mag, None, None
    x, w = np.asarray(x, np.float64), np.asarray(weight, np.float64)
    rho = 1.0 / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps)
    n = x * rho
    g = dy * w
    dx = rho * (g - n * (g * n).mean(-1, keepdims=True))
    gm = mag * np.abs(w)
    dmag = rho * (gm + 3.0 * np.abs(n) * (gm * np.abs(n)).mean(-1, keepdims=True))
    return dx, dmag, (dy * n).sum((0, 1)), (mag * np.abs(n)).sum((0, 1))

"""Rows in 8 bits, in 64 bits (numpy), from the format: e4m3 codes (a sign, 4
exponent bits with a bias of 7, 3 fraction bits; exponent 0: subnormals of 2^-9;
0x7f and 0xff: NaN) and one power of two for each row, kept as exponent + 127.
"""
from __future__ import annotations

import numpy as np

MIN_EXPONENT, NAN = -64, 255


def _grid():
    """The value of every code."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, (8.0 + m) * 2.0 ** (e - 10.0), m * 2.0 ** -9)
    v[(c & 127) == 127] = np.nan
    return np.where(c >> 7, -v, v)


VALUES = _grid()
_POSITIVE = VALUES[:127]  # ascending


def encode(x, nan_code=0):
    """Rows x [..., d] as ``(codes [..., d], bytes [...])``, uint8: the smallest
    e >= -64 with max |x| <= 448 * 2^e, codes of x * 2^-e rounded to the nearest
    value, ties to the even code.  Rows that are not finite, or that would not stay
    so in fp32: ``nan_code``, 255."""
    x = np.asarray(x, np.float64)
    bad = ~(np.abs(x) < 248 * 2.0 ** 120).all(-1)  # (248 * 2^120 rounds to 2^128)
    y = np.where(bad[..., None], 0.0, x)
    a = np.abs(y).max(-1, initial=0.0)
    e = np.full(a.shape, MIN_EXPONENT)
    while (grow := a > 448.0 * np.exp2(e.astype(np.float64))).any():
        e = e + grow
    y = y * np.exp2(-e.astype(np.float64))[..., None]
    mag = np.abs(y)
    hi = np.clip(np.searchsorted(_POSITIVE, mag), 0, 126)  # first value >= mag
    lo = np.maximum(hi - 1, 0)
    dl, dh = mag - _POSITIVE[lo], _POSITIVE[hi] - mag
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi) | np.where(np.signbit(y), 128, 0)
    return (np.where(bad[..., None], nan_code, code).astype(np.uint8), np.where(bad, NAN, e + 127).astype(np.uint8))


def decode(codes, scale):
    """The values that rows of codes and their bytes stand for."""
    s = np.where(scale == NAN, np.nan, np.exp2(scale.astype(np.float64) - 127))
    return VALUES[codes] * s[..., None]


def empty(blocks, hkv, d, seed):
    """An 8-bit cache of anything: uint8 arrays ``(k, v, scales)``."""
    rng = np.random.default_rng([seed, 77])
    draw = lambda *shape: rng.integers(0, 256, size=shape, dtype=np.uint8)  # noqa: E731
    return draw(blocks, hkv, d // 16, 16, 16), draw(blocks, hkv, d, 16), draw(blocks, hkv, 2, 16)


def write(cache, blk, slot, k, v):
    """Rows k, v [n, Hkv, d] (64 bits) into (block, slot) places."""
    kc, vc, sc = cache
    n, hkv, d = np.shape(k)
    codes, s = encode(k, nan_code=0x7f)
    kc[blk, :, :, slot] = codes.reshape(n, hkv, d // 16, 16)
    sc[blk, :, 0, slot] = s
    codes, s = encode(v)
    vc[blk, :, :, slot] = codes
    sc[blk, :, 1, slot] = s


def read(cache, blk, slot):
    """The rows' values at (block, slot) places: ``(k, v)`` [n, Hkv, d]."""
    kc, vc, sc = cache
    k = kc[blk, :, :, slot]
    return (decode(k.reshape(*k.shape[:2], -1), sc[blk, :, 0, slot]), decode(vc[blk, :, :, slot], sc[blk, :, 1, slot]))

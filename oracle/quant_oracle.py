"""Caches held in 4 or 8 bits, in float64 numpy, from the definition: a group of 32
elements along the head dimension is a power of two times elements of a small float
format.  Test infrastructure only.
"""
from __future__ import annotations

import math

import numpy as np

GROUP = 32
# bits: (mantissa bits, exponent bias, what a group's largest magnitude may be in steps of
# its scale, largest scale exponent)
FORMATS = {4: (1, 1, 7.0, 125), 8: (3, 7, 448.0, 119)}
LEAST = -111


def elements(bits):
    """Values of the elements' codes, sign and all (e4m3: 127 and 255 are NaN)."""
    mant, bias, _, _ = FORMATS[bits]
    out = np.zeros(2 ** bits)
    for code in range(2 ** bits):
        sign, rest = divmod(code, 2 ** (bits - 1))
        exp, frac = divmod(rest, 2 ** mant)
        mag = math.ldexp(frac, 1 - bias - mant) if exp == 0 else \
            math.ldexp(2 ** mant + frac, exp - bias - mant)
        if bits == 8 and rest == 127:
            mag = math.nan
        out[code] = -mag if sign else mag
    return out


def quantise(x, bits):
    """x [.., d] float64 -> codes [.., d] (one each) and scale bytes [.., d / 32]."""
    _, _, fits, most = FORMATS[bits]
    grid = elements(bits)[:2 ** (bits - 1)]
    grid = grid[np.isfinite(grid)]
    borders = (grid[1:] + grid[:-1]) / 2
    shape = x.shape
    x = x.reshape(-1, GROUP)
    codes = np.zeros(x.shape, dtype=np.uint8)
    scales = np.zeros(len(x), dtype=np.uint8)
    top = np.abs(x).max(-1)
    ok = np.isfinite(top)
    scales[~ok] = 255
    X = np.full(len(x), LEAST)
    for e in range(LEAST, most):           # the least that holds the group
        X[ok & (top > fits * 2.0 ** e)] = e + 1
    scales[ok] = X[ok] + 127
    with np.errstate(invalid="ignore"):
        y = np.abs(x) / np.exp2(X)[:, None]
    y = np.where(ok[:, None], y, 0.0)
    low = np.searchsorted(borders, y, side="left")      # one at a border stays below it ..
    high = np.searchsorted(borders, y, side="right")    # .. or goes above
    codes = np.where(low % 2 == 0, low, high).astype(np.uint8)
    codes = codes + np.where(np.signbit(x), 2 ** (bits - 1), 0).astype(np.uint8)
    return codes.reshape(shape), scales.reshape(shape[:-1] + (shape[-1] // GROUP,))


def values(codes, scales, bits):
    """codes [.., d], scale bytes [.., d / 32] -> [.., d] float64 (NaN where scales are 255)."""
    s = scales.astype(np.float64)
    power = np.where(s == 255, math.nan, np.exp2(s - 127))
    return elements(bits)[codes] * np.repeat(power, GROUP, axis=-1)


def pack(codes, bits):
    return codes if bits == 8 else (codes[..., 0::2] | codes[..., 1::2] << 4).astype(np.uint8)


def unpack(held, bits):
    if bits == 8:
        return held
    return np.stack([held & 15, held >> 4], -1).reshape(held.shape[:-1] + (-1,))

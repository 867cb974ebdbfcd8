"""Microscaled 4-bit rows in float64 NumPy: format, quantisation, product.

e2m1 codes (sign, two exponent bits, one mantissa bit), two per byte, the first in the low half; one power-of-two scale
2^(b - 127) per 32 elements. Codes are found by searching the eight magnitudes, not by bit arithmetic.
"""
from __future__ import annotations

import math

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
BLOCK = 32


def exponent_byte(amax: float) -> int:
    """Smallest b in 1..252 with amax <= 7 2^(b - 127), 252 where none is; 127 for 0."""
    if amax == 0:
        return 127
    b = 1
    while b < 252 and amax > math.ldexp(7.0, b - 127):
        b += 1
    return b


def quantize(x):
    """(codes [rows][cols / 2], scale bytes [rows][cols / 32]) of x [rows][cols]."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    v = x.reshape(rows, cols // BLOCK, BLOCK)
    fine = np.isfinite(v).all(axis=2)
    amax = np.abs(np.where(fine[:, :, None], v, 0.0)).max(axis=2)
    known = {a: exponent_byte(float(a)) for a in np.unique(amax)}
    exps = np.vectorize(known.get, otypes=[np.int64])(amax) if amax.size else np.zeros(amax.shape, np.int64)
    y = np.abs(np.where(fine[:, :, None], v, 0.0)) / np.ldexp(1.0, exps - 127)[:, :, None]
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    down, up = np.searchsorted(mid, y, "left"), np.searchsorted(mid, y, "right")
    code = np.where(down % 2 == 0, down, up)              # they differ on a midpoint only
    code = np.where(fine[:, :, None], code + 8 * np.signbit(v), 0).reshape(rows, cols)
    return (code[:, 0::2] | code[:, 1::2] << 4).astype(np.uint8), np.where(fine, exps, 255).astype(np.uint8)


def values(codes, scales):
    """float64 values of codes [rows][cols / 2] with scale bytes [rows][cols / 32]."""
    codes = np.asarray(codes)
    c = np.stack([codes & 15, codes >> 4], axis=2).reshape(codes.shape[0], -1)
    b = np.asarray(scales).astype(np.int64)
    s = np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))
    return np.concatenate([MAGNITUDES, -MAGNITUDES])[c] * np.repeat(s, BLOCK, axis=1)


def gelu(x):
    return 0.5 * x * (1.0 + np.vectorize(math.erf, otypes=[np.float64])(np.asarray(x) * math.sqrt(0.5)))


def linear(a, w, bias, resid=None, use_gelu=False):
    """(out, sum of |a w| + |bias|) of values a [M][K] and w [N][K]."""
    z = a @ w.T + bias
    size = np.abs(a) @ np.abs(w).T + np.abs(bias)
    if use_gelu:
        z = gelu(z)
    return (z if resid is None else z + resid), size

"""The 8-bit K/V cache in float64 NumPy: format, quantisation, rewriting of rows, attention.

e4m3 codes (sign, four exponent bits with bias 7, three mantissa bits, no infinities, NaN at 0x7f / 0xff) with one
power-of-two scale 2^(b - 127) per (cache, block of tokens, K or V, head). Every code is found by searching the table
of the 127 magnitudes, not by bit arithmetic.
"""
from __future__ import annotations

import math

import numpy as np


def _magnitudes() -> np.ndarray:
    """The 127 finite magnitudes, ascending: code c < 8 is c 2^-9, else (8 + c % 8) 2^(c // 8 - 10)."""
    return np.array([math.ldexp(c % 8, -9) if c < 8 else math.ldexp(8 + c % 8, c // 8 - 10) for c in range(127)])


MAGNITUDES = _magnitudes()


def code_values() -> np.ndarray:
    """The values of the 256 codes."""
    v = np.append(MAGNITUDES, np.nan)
    return np.concatenate([v, -v])


def scale_value(b) -> np.ndarray:
    """2^(b - 127) of exponent bytes, NaN at 255."""
    b = np.asarray(b).astype(np.int64)
    return np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))


def exponent_byte(amax: float) -> int:
    """Smallest b >= 1 with amax <= 448 2^(b - 127); 127 for 0."""
    if amax == 0:
        return 127
    b = 1
    while amax > math.ldexp(448.0, b - 127):
        b += 1
    return b


def encode(x, b: int) -> np.ndarray:
    """Codes of x at the scale 2^(b - 127): nearest magnitude, ties to the even code; NaN and infinities -> NaN."""
    x = np.asarray(x, np.float64)
    fine = np.isfinite(x)
    y = np.abs(np.where(fine, x, 0.0)) / math.ldexp(1.0, b - 127)
    mid = (MAGNITUDES[1:] + MAGNITUDES[:-1]) / 2
    down, up = np.searchsorted(mid, y, "left"), np.searchsorted(mid, y, "right")
    code = np.where(down % 2 == 0, down, up)          # they differ on a midpoint only
    code = np.where(fine, code, 127)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def quantize(x, block: int):
    """(codes like x, exponent bytes [blocks][2][H]) of x [T][2][H][hd]."""
    T, _, H, _ = x.shape
    codes = np.zeros(x.shape, np.uint8)
    exps = np.zeros((-(-T // block), 2, H), np.uint8)
    for k, t in enumerate(range(0, T, block)):
        for w in range(2):
            for h in range(H):
                tile = np.asarray(x[t:t + block, w, h], np.float64)
                fine = np.abs(tile[np.isfinite(tile)])
                b = exponent_byte(float(fine.max()) if fine.size else 0.0)
                exps[k, w, h] = b
                codes[t:t + block, w, h] = encode(tile, b)
    return codes, exps


def values(codes, exps, block: int) -> np.ndarray:
    """float64 values of codes [T][2][H][hd] with exponent bytes [blocks][2][H]."""
    return code_values()[codes] * np.repeat(scale_value(exps), block, axis=0)[:codes.shape[0], ..., None]


def rewrite(codes, exps, block: int, kv, src_row):
    """Tokens with 0 <= src_row[t] < len(kv) take that row; blocks without such a token stay as they are."""
    codes, exps = codes.copy(), exps.copy()
    x = values(codes, exps, block)
    new = (src_row >= 0) & (src_row < len(kv))
    x[new] = np.asarray(kv, np.float64)[src_row[new]]
    for k, t in enumerate(range(0, len(codes), block)):
        if new[t:t + block].any():
            c, e = quantize(x[t:t + block], block)
            codes[t:t + block], exps[k] = c, e[0]
    return codes, exps


def attention(q, k, v, scale: float):
    """(out, spread) of q [M][H][hd] over k, v [n][Hkv][hd]: out = sum w v / sum w with w = exp(scale q.k - max), zeros
    without keys; spread = sum w |v - out| / sum w, what relative errors of the weights act on."""
    M, H, hd = q.shape
    n, G = k.shape[0], H // k.shape[1]
    out, spread = np.zeros((M, H, hd)), np.zeros((M, H, hd))
    if n == 0:
        return out, spread
    with np.errstate(invalid="ignore", over="ignore"):
        for h in range(H):
            s = scale * (q[:, h] @ k[:, h // G].T)
            w = np.exp(s - s.max(1, keepdims=True))
            w /= w.sum(1, keepdims=True)
            out[:, h] = w @ v[:, h // G]
            for m in range(M):
                spread[m, h] = w[m] @ np.abs(v[:, h // G] - out[m, h])
    return out, spread

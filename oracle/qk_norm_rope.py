"""Per-head norms, position rotation and K/V scatter in float64 NumPy."""
from __future__ import annotations

import numpy as np


def norm(x, gain, eps):
    """x [rows][heads][hd] over its heads' root mean square, times gain; x itself without one."""
    return x if gain is None else x / np.sqrt((x * x).mean(axis=2, keepdims=True) + eps) * gain


def rotate(x, table, pos, halves):
    """(result, |x_i| + |x_j| of every element's pair) of x [rows][heads][hd] with (cos, sin) = table[pos[m]][p]; rows without
    a position in the table stay."""
    out, size = x.copy(), np.abs(x)
    if table is None:
        return out, size
    half = table.shape[1]
    for m, p in enumerate(pos):
        if not 0 <= p < table.shape[0]:
            continue
        for k in range(half):
            i, j = (k, k + half) if halves else (2 * k, 2 * k + 1)
            c, s = table[p, k]
            a, b = x[m, :, i], x[m, :, j]
            out[m, :, i], out[m, :, j] = a * c - b * s, b * c + a * s
            size[m, :, i] = size[m, :, j] = np.abs(a) + np.abs(b)
    return out, size


def qk_norm_rope(qkv, heads, kv_heads, hd, q_gain, k_gain, eps, table, pos, halves):
    """((q, its sizes), (k, its sizes), v) of rows [rows][(heads + 2 kv_heads) hd]."""
    x = qkv.reshape(qkv.shape[0], heads + 2 * kv_heads, hd)
    pos = np.arange(x.shape[0]) if pos is None else pos
    q = rotate(norm(x[:, :heads], q_gain, eps), table, pos, halves)
    k = rotate(norm(x[:, heads:heads + kv_heads], k_gain, eps), table, pos, halves)
    return q, k, x[:, heads + kv_heads:]

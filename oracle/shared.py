"""Attention of a batch over one shared prefix in float64 NumPy."""
from __future__ import annotations

import numpy as np


def attention(q, kv, hidden, seg_start, fresh, fresh_start, scale):
    """(out, spread, size, reach) of q [rows][heads][hd] over kv [tokens][2][kv_heads][hd], hidden bool [batch][tokens] or
    None, own rows fresh [..][2][kv_heads][hd] by fresh_start, or None. spread = sum w |v - out| / sum w and size = sum w |v| /
    sum w per output element, reach = the largest sum |q k| |scale| of the row and head: what errors are bounded with. Rows of
    no request and rows without a key are zeros."""
    M, H, hd = q.shape
    G = kv.shape[2]
    out, spread, size = (np.zeros(q.shape) for _ in range(3))
    reach = np.zeros((M, H, 1))
    for b in range(len(seg_start) - 1):
        r0, r1 = seg_start[b], seg_start[b + 1]
        rows = kv if hidden is None else kv[~hidden[b]]
        if fresh is not None:
            rows = np.concatenate([rows, fresh[fresh_start[b]:fresh_start[b + 1]]])
        if r1 <= r0 or len(rows) == 0:
            continue
        for h in range(H):
            k, v = rows[:, 0, h * G // H], rows[:, 1, h * G // H]
            with np.errstate(invalid="ignore"):
                z = q[r0:r1, h] @ k.T * scale
                top = z.max(axis=1, keepdims=True)
                w = np.exp(z - np.where(top == -np.inf, 0.0, top))
                total = w.sum(axis=1, keepdims=True)
                o = np.where(total == 0, 0.0, w @ v / np.where(total == 0, 1.0, total))
            out[r0:r1, h] = o
            w = w / np.where(total == 0, 1.0, total)
            size[r0:r1, h] = w @ np.abs(v)
            for c in range(hd):
                spread[r0:r1, h, c] = (w * np.abs(v[None, :, c] - o[:, None, c])).sum(axis=1)
            reach[r0:r1, h, 0] = (np.abs(q[r0:r1, h]) @ np.abs(k).T).max(axis=1) * abs(scale)
    return out, spread, size, reach

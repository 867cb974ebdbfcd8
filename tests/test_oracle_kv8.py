"""Pins of the 8-bit cache oracle: torch's e4m3 conversion, closed forms, brute force."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8


def test_code_table_is_torchs():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(kv8.code_values(), t, equal_nan=True)


def test_encode_matches_torchs_conversion():
    """float32 values over the whole range, every midpoint between codes and its neighbours."""
    mid = (kv8.MAGNITUDES[1:] + kv8.MAGNITUDES[:-1]) / 2
    x = np.concatenate([mid, np.nextafter(mid.astype(np.float32), np.float32(0)), np.nextafter(mid.astype(np.float32), np.float32(1e9)),
                        kv8.MAGNITUDES, np.random.default_rng(0).normal(0, 60, 5000)]).astype(np.float32)
    x = np.clip(np.concatenate([x, -x]), -448, 448)
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(kv8.encode(x, 127), want)


@pytest.mark.parametrize("amax,byte", [(0.0, 127), (448.0, 127), (448.0001, 128), (224.0, 126), (224.0001, 127), (1.75, 119), (1.0, 119),
                                       (1.7500001, 120), (2.0 ** -140, 1), (448 * 2.0 ** -126, 1), (449 * 2.0 ** -126, 2),
                                       (float(np.finfo(np.float32).max), 247)])
def test_exponent_byte(amax, byte):
    assert kv8.exponent_byte(amax) == byte


def test_quantised_values_are_within_half_a_code():
    """|x - value| <= 2^-4 |x| for x at or above the smallest normal code 2^-6 s, 2^-10 s below it; at most 448 s."""
    x = np.random.default_rng(1).normal(0, 1, (37, 2, 3, 16)) * np.exp(np.random.default_rng(2).normal(0, 2, (2, 3, 1)))
    c, e = kv8.quantize(x, 16)
    s = np.repeat(kv8.scale_value(e), 16, axis=0)[:37, ..., None]
    assert np.all(np.abs(kv8.values(c, e, 16) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * s))
    assert np.all(np.abs(x) <= 448 * s)
    largest = np.maximum.reduceat(np.abs(x).max(-1), [0, 16, 32])
    assert np.all(largest > 224 * kv8.scale_value(e))


def test_not_finite_values_become_nan_and_leave_the_scale_alone():
    x = np.ones((4, 2, 1, 8))
    x[1, 0, 0, 3], x[2, 0, 0, 1], x[2, 0, 0, 2] = np.nan, np.inf, -np.inf
    c, e = kv8.quantize(x, 4)
    v = kv8.values(c, e, 4)
    assert np.array_equal(np.isnan(v), ~np.isfinite(x)) and np.all(v[np.isfinite(x)] == 1)
    assert np.array_equal(e, kv8.quantize(np.ones_like(x), 4)[1])


def test_rewrite_of_every_row_is_a_new_cache_and_of_none_the_same():
    g = np.random.default_rng(3)
    old, new = g.normal(0, 1, (21, 2, 2, 8)), g.normal(0, 30, (21, 2, 2, 8))
    c, e = kv8.quantize(old, 8)
    c2, e2 = kv8.rewrite(c, e, 8, new, np.arange(21))
    assert all(np.array_equal(a, b) for a, b in zip((c2, e2), kv8.quantize(new, 8)))
    c3, e3 = kv8.rewrite(c, e, 8, new, np.full(21, -1))
    assert np.array_equal(c3, c) and np.array_equal(e3, e)
    src = np.full(21, -1)
    src[9] = 4
    c4, e4 = kv8.rewrite(c, e, 8, new, src)
    assert np.array_equal(c4[:8], c[:8]) and np.array_equal(c4[16:], c[16:]) and np.all(e4[1] > e[1])
    kept = [8, 10, 11, 12, 13, 14, 15]
    s = kv8.scale_value(e4[1])[None, ..., None]
    off = np.abs(kv8.values(c4, e4, 8)[kept] - kv8.values(c, e, 8)[kept])
    assert np.all(off <= 2.0 ** -10 * s)                  # only values below the smallest normal code move
    assert not off[np.abs(kv8.values(c, e, 8)[kept]) >= 2.0 ** -6 * np.broadcast_to(s, off.shape)].any()


def test_attention_matches_torch_softmax_and_closed_forms():
    g = np.random.default_rng(4)
    q, k, v = g.normal(0, 1, (5, 6, 8)), g.normal(0, 1, (9, 2, 8)), g.normal(0, 1, (9, 2, 8))
    out, spread = kv8.attention(q, k, v, 0.3)
    for h in range(6):
        p = torch.softmax(torch.from_numpy(q[:, h] @ k[:, h // 3].T) * 0.3, dim=1).numpy()
        assert np.allclose(out[:, h], p @ v[:, h // 3], rtol=1e-13, atol=1e-15)
    one, sp = kv8.attention(q, k[:1], v[:1], 0.3)
    assert np.allclose(one, np.repeat(v[:1], 3, axis=1)) and np.allclose(sp, 0)
    none, _ = kv8.attention(q, k[:0], v[:0], 0.3)
    assert np.array_equal(none, np.zeros_like(q))
    assert math.isclose(kv8.attention(0 * q, k, v, 0.3)[0][2, 4, 1], v[:, 1, 1].mean(), rel_tol=1e-12)

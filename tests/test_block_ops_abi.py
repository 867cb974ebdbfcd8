"""Refusals of the 4-bit products, the per-head norms with rotation and the shared attention, before any device work (no GPU
needed), and the oracle's pins."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import mx4, qk_norm_rope, shared
from paper_2505_20600_amd import maskstep as MS

P = 4096    # an address that is checked but never read
BF, F32 = MS.MS_BF16, MS.MS_FP32
_id = lambda v: "-".join(f"{k}={w}" for k, w in v.items()) if isinstance(v, dict) else None


def _refused(status, want):
    assert status == want and MS.load().mask_last_error()


# ------------------------------------------------------------------ 4 bits

ROWS = dict(dtype=BF, x=P, rows=5, cols=64, ld=64, codes=P, scales=P)
BAD_ROWS = [
    (dict(dtype=2), MS.MS_EDTYPE), (dict(dtype=-1), MS.MS_EDTYPE), (dict(rows=-1), MS.MS_ESHAPE), (dict(rows=(1 << 26) + 1), MS.MS_ESHAPE),
    (dict(cols=0), MS.MS_ESHAPE), (dict(cols=48, ld=48), MS.MS_ESHAPE), (dict(cols=-32), MS.MS_ESHAPE), (dict(cols=(1 << 20) + 32, ld=1 << 21), MS.MS_ESHAPE),
    (dict(ld=63), MS.MS_ESHAPE), (dict(ld=68), MS.MS_ESHAPE), (dict(ld=(1 << 32) + 8), MS.MS_ESHAPE), (dict(dtype=F32, ld=66), MS.MS_ESHAPE),
    (dict(x=None), MS.MS_EINVAL), (dict(codes=None), MS.MS_EINVAL), (dict(scales=None), MS.MS_EINVAL),
    (dict(x=P + 8), MS.MS_EALIGN), (dict(codes=P + 4), MS.MS_EALIGN)]


@pytest.mark.parametrize("kw,status", BAD_ROWS, ids=_id)
def test_bad_rows_are_refused(kw, status):
    a = {**ROWS, **kw}
    lib = MS.load()
    _refused(lib.ms_mx4_quantize(a["dtype"], a["x"], a["rows"], a["cols"], a["ld"], a["codes"], a["scales"], None), status)
    _refused(lib.ms_mx4_dequantize(a["dtype"], a["codes"], a["scales"], a["rows"], a["cols"], a["x"], a["ld"], None), status)


PRODUCT = dict(dtype=BF, M=3, N=8, K=64, a=P, sa=P, w=P, sw=P, bias=P, resid=P, out=P, epi=1, ws=P, n=0)
BAD_PRODUCT = [
    (dict(dtype=7), MS.MS_EDTYPE), (dict(M=-1), MS.MS_ESHAPE), (dict(M=(1 << 26) + 1), MS.MS_ESHAPE), (dict(N=0), MS.MS_ESHAPE),
    (dict(N=6), MS.MS_ESHAPE), (dict(N=(1 << 20) + 4), MS.MS_ESHAPE), (dict(K=0), MS.MS_ESHAPE), (dict(K=40), MS.MS_ESHAPE),
    (dict(K=(1 << 20) + 32), MS.MS_ESHAPE), (dict(M=1 << 20, N=1 << 12), MS.MS_ESHAPE), (dict(epi=3), MS.MS_EINVAL), (dict(epi=-1), MS.MS_EINVAL),
    (dict(a=None), MS.MS_EINVAL), (dict(sa=None), MS.MS_EINVAL), (dict(w=None), MS.MS_EINVAL), (dict(sw=None), MS.MS_EINVAL),
    (dict(bias=None), MS.MS_EINVAL), (dict(out=None), MS.MS_EINVAL), (dict(resid=None), MS.MS_EINVAL),
    (dict(a=P + 8), MS.MS_EALIGN), (dict(w=P + 2), MS.MS_EALIGN), (dict(bias=P + 4), MS.MS_EALIGN), (dict(out=P + 8), MS.MS_EALIGN),
    (dict(resid=P + 8), MS.MS_EALIGN), (dict(ws=P + 4), MS.MS_EALIGN)]


@pytest.mark.parametrize("kw,status", BAD_PRODUCT, ids=_id)
def test_bad_products_are_refused(kw, status):
    a = {**PRODUCT, **kw}
    lib = MS.load()
    _refused(lib.ms_mx4_linear(a["dtype"], a["M"], a["N"], a["K"], a["a"], a["sa"], a["w"], a["sw"], a["bias"], a["resid"], a["out"], a["epi"],
                               a["ws"], a["n"], None), status)
    if set(kw) <= {"M", "N", "K"}:
        assert lib.ms_mx4_linear_workspace_bytes(a["M"], a["N"], a["K"]) == 0 and lib.mask_last_error()


def test_product_workspace_clears_the_error():
    lib = MS.load()
    assert lib.ms_mx4_linear_workspace_bytes(-1, 8, 64) == 0 and lib.mask_last_error()
    lib.ms_mx4_linear_workspace_bytes(300, 8, 64)
    assert not lib.mask_last_error()


# ------------------------------------------------------------------ norms and rotation

def _qk(**kw):
    a = MS.QkNormRopeArgs(BF, 7, 4, 2, 64, P, 512, P, P, 1e-6, P, 100, 64, 0, P, P, P, 20, P)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_QK = [
    (dict(dtype=3), MS.MS_EDTYPE), (dict(rows=-1), MS.MS_ESHAPE), (dict(rows=(1 << 26) + 1), MS.MS_ESHAPE), (dict(n_heads=0), MS.MS_ESHAPE),
    (dict(n_heads=1025, ld=1 << 20), MS.MS_ESHAPE), (dict(n_kv_heads=0), MS.MS_ESHAPE), (dict(n_kv_heads=1025, ld=1 << 20), MS.MS_ESHAPE),
    (dict(head_dim=0), MS.MS_ESHAPE), (dict(head_dim=12), MS.MS_ESHAPE), (dict(head_dim=136, ld=4096), MS.MS_ESHAPE),
    (dict(ld=511), MS.MS_ESHAPE), (dict(ld=516), MS.MS_ESHAPE), (dict(ld=1 << 33), MS.MS_ESHAPE), (dict(kv_rows=-1), MS.MS_ESHAPE),
    (dict(rot=0), MS.MS_ESHAPE), (dict(rot=7), MS.MS_ESHAPE), (dict(rot=66), MS.MS_ESHAPE), (dict(n_pos=-1), MS.MS_ESHAPE),
    (dict(pairing=2), MS.MS_EINVAL), (dict(eps=-1.0), MS.MS_EINVAL), (dict(eps=math.nan), MS.MS_EINVAL), (dict(eps=math.inf), MS.MS_EINVAL),
    (dict(qkv=None), MS.MS_EINVAL), (dict(q=None), MS.MS_EINVAL), (dict(kv=None), MS.MS_EINVAL),
    (dict(qkv=P + 8), MS.MS_EALIGN), (dict(q=P + 8), MS.MS_EALIGN), (dict(kv=P + 8), MS.MS_EALIGN), (dict(q_gain=P + 2), MS.MS_EALIGN),
    (dict(k_gain=P + 2), MS.MS_EALIGN), (dict(table=P + 8), MS.MS_EALIGN), (dict(pos=P + 2), MS.MS_EALIGN), (dict(dst_rows=P + 1), MS.MS_EALIGN)]


@pytest.mark.parametrize("kw,status", BAD_QK, ids=_id)
def test_bad_norm_and_rotation_arguments_are_refused(kw, status):
    a = _qk(**kw)
    _refused(MS.load().ms_qk_norm_rope(C.byref(a), None), status)


# ------------------------------------------------------------------ shared attention

def _attn(**kw):
    a = MS.SharedAttn(P, P, 10, 8, 4, 64, P, 100, 3, P, P, P, 10, P, 0.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_ATTN = [
    (dict(rows=-1), MS.MS_ESHAPE), (dict(rows=(1 << 26) + 1), MS.MS_ESHAPE), (dict(rows=(1 << 24) + 1), MS.MS_ESHAPE),
    (dict(n_heads=0), MS.MS_ESHAPE), (dict(n_heads=6), MS.MS_ESHAPE), (dict(n_heads=2048), MS.MS_ESHAPE),
    (dict(n_kv_heads=0), MS.MS_ESHAPE), (dict(n_kv_heads=1025), MS.MS_ESHAPE), (dict(head_dim=0), MS.MS_ESHAPE), (dict(head_dim=20), MS.MS_ESHAPE),
    (dict(head_dim=136), MS.MS_ESHAPE), (dict(batch=0), MS.MS_ESHAPE), (dict(batch=129), MS.MS_ESHAPE),
    (dict(tokens=-1), MS.MS_ESHAPE), (dict(tokens=(1 << 20) + 1), MS.MS_ESHAPE), (dict(tokens=1 << 20, n_kv_heads=8, head_dim=128), MS.MS_ESHAPE),
    (dict(seg_start=None), MS.MS_EINVAL), (dict(q=None), MS.MS_EINVAL), (dict(out=None), MS.MS_EINVAL), (dict(kv=None), MS.MS_EINVAL),
    (dict(fresh_start=None), MS.MS_EINVAL), (dict(fresh_rows=-1), MS.MS_ESHAPE), (dict(fresh_rows=1 << 22), MS.MS_ESHAPE),
    (dict(q=P + 8), MS.MS_EALIGN), (dict(out=P + 8), MS.MS_EALIGN), (dict(kv=P + 8), MS.MS_EALIGN), (dict(fresh=P + 8), MS.MS_EALIGN),
    (dict(bits=P + 4), MS.MS_EALIGN), (dict(seg_start=P + 2), MS.MS_EALIGN), (dict(fresh_start=P + 1), MS.MS_EALIGN),
    (dict(scale=math.nan), MS.MS_EINVAL), (dict(scale=math.inf), MS.MS_EINVAL), (dict(scale=3e38), MS.MS_EINVAL)]


@pytest.mark.parametrize("kw,status", BAD_ATTN, ids=_id)
def test_bad_attention_arguments_are_refused(kw, status):
    a, lib = _attn(**kw), MS.load()
    _refused(lib.ms_shared_attention(BF, C.byref(a), None, 0, None), status)
    assert lib.ms_shared_attention_workspace_bytes(BF, C.byref(a)) == 0 and lib.mask_last_error()


def test_other_attention_refusals():
    lib, a = MS.load(), _attn()
    _refused(lib.ms_shared_attention(5, C.byref(a), None, 0, None), MS.MS_EDTYPE)
    _refused(lib.ms_shared_attention(F32, C.byref(_attn(head_dim=72)), None, 0, None), MS.MS_ESHAPE)
    _refused(lib.ms_shared_attention(BF, None, None, 0, None), MS.MS_EINVAL)
    _refused(lib.ms_shared_attention(BF, C.byref(a), P + 8, 64, None), MS.MS_EALIGN)
    for args in [(None, 1, 1, P), (P, 1, 1, None), (P, 0, 1, P), (P, 129, 1, P), (P, 1, 0, P), (P, 1, (1 << 20) + 1, P), (P, 1, 1, P + 4)]:
        assert lib.ms_shared_bits(*args, None) != MS.MS_OK
    assert lib.ms_shared_attention_workspace_bytes(BF, C.byref(_attn(rows=5))) >= 0 and not lib.mask_last_error()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("heads,group,hd", [(1, 1, 8), (4, 8, 64), (1024, 1, 16)])
def test_key_ranges_stay_within_one_launch(dtype, heads, group, hd):
    """Whatever the sizes, the planned ranges are launches below 2^32 threads: 256 per 16 query slots (or more), K/V head and
    range, and a wave per row and head for the join."""
    lib = MS.load()
    for bits in range(27):
        rows = 1 << bits
        if rows * heads * group > 1 << 27:
            break
        for tokens in (1, 4096, min(1 << 20, ((4095 << 20) - 1) // (2 * heads * hd * 4))):
            a = _attn(rows=rows, n_heads=heads * group, n_kv_heads=heads, head_dim=hd, tokens=tokens, fresh=None)
            need = lib.ms_shared_attention_workspace_bytes(dtype, C.byref(a))
            n = need // (4 * rows * heads * group * (hd + 2))
            assert n <= 64
            assert (rows * group // 16 + 1) * max(1, n) * heads * 256 < 1 << 32 or n <= 1


# ------------------------------------------------------------------ binding

def test_binding_refuses_what_is_not_on_a_gpu_or_of_another_shape():
    t = lambda *s, dt=torch.bfloat16: torch.zeros(*s, dtype=dt)
    u8 = torch.uint8
    for call in [lambda: MS.ms_mx4_quantize(t(3, 64), t(3, 32, dt=u8), t(3, 2, dt=u8)),
                 lambda: MS.ms_mx4_quantize(t(3, 64, dt=torch.float16), t(3, 32, dt=u8), t(3, 2, dt=u8)),
                 lambda: MS.ms_mx4_dequantize(t(3, 32, dt=u8), t(3, 2, dt=u8), t(3, 64)),
                 lambda: MS.ms_mx4_linear(t(3, 32, dt=u8), t(3, 2, dt=u8), t(8, 32, dt=u8), t(8, 2, dt=u8), t(8), t(3, 8)),
                 lambda: MS.ms_qk_norm_rope(t(3, 48), t(3, 4, 8), t(3, 2, 1, 8)),
                 lambda: MS.ms_shared_bits(t(3, 64, dt=u8), t(3, 1, dt=torch.int64)),
                 lambda: MS.ms_shared_attention(t(3, 4, 8), t(9, 2, 4, 8), t(3, 4, 8)),
                 lambda: MS.ms_shared_attention(t(3, 4, 8), t(9, 2, 4, 8), t(3, 4, 8), scale=0.0),
                 lambda: MS.ms_shared_attention(t(3, 4, 8), t(9, 2, 4, 8), t(3, 4, 8), scale=1e-60),
                 lambda: MS.ms_shared_attention(t(3, 4, 8, dt=torch.float16), t(9, 2, 4, 8), t(3, 4, 8)),
                 lambda: MS.ms_shared_attention_workspace_bytes(t(3, 4, 12), t(9, 2, 4, 12)),
                 lambda: MS.ms_mx4_linear_workspace_bytes(t(3, 20, dt=u8), t(8, 20, dt=u8))]:
        with pytest.raises(MS.MaskStepError):
            call()


# ------------------------------------------------------------------ the oracle

def test_oracle_codes_and_scales():
    """Hand-worked blocks: the scale's border at seven times it, ties to even, saturation, NaN blocks."""
    x = np.zeros((6, 32))
    x[0, :8] = [7, 0.25, 0.75, 1.25, 2.5, 3.5, 5, -5]
    x[1, 0] = 7.03125
    x[2, 0], x[2, 1] = 6, -0.0
    x[3, 0] = math.inf
    x[4, 0] = 2.0 ** 127 * 1.99
    x[5, 0] = 2.0 ** -130
    codes, scales = mx4.quantize(x)
    assert scales[:, 0].tolist() == [127, 128, 127, 255, 252, 1]
    v = mx4.values(codes, scales)
    assert v[0, :8].tolist() == [6, 0, 1, 1, 2, 4, 4, -4] and v[1, 0] == 8 and v[2, 0] == 6 and codes[2, 0] == 0x87
    assert np.isnan(v[3]).all() and v[4, 0] == 6 * 2.0 ** 125 and v[5, 0] == 0.0
    assert mx4.exponent_byte(0.0) == 127 and mx4.exponent_byte(1.0) == 125
    g = np.random.default_rng(1)
    y = g.standard_normal((4, 96))
    c, s = mx4.quantize(y)
    # the widest step is 2 s, so no value is off by more than s, and a block's largest is above 3.5 s (or s / 2 would do)
    assert np.abs(mx4.values(c, s) - y).max() <= np.abs(y).max() / 3.5


def test_oracle_product_against_torch():
    g = torch.Generator().manual_seed(2)
    a, w, b, r = (torch.randn(*n, generator=g, dtype=torch.float64) for n in ((5, 64), (8, 64), (8,), (5, 8)))
    z = torch.nn.functional.linear(a, w, b)
    assert np.allclose(mx4.linear(a.numpy(), w.numpy(), b.numpy(), r.numpy())[0], (z + r).numpy())
    assert np.allclose(mx4.linear(a.numpy(), w.numpy(), b.numpy(), None, True)[0], torch.nn.functional.gelu(z).numpy())


@pytest.mark.parametrize("halves", [False, True])
def test_oracle_rotation(halves):
    """Norms of one, a turn by the angle of the position, inner products that depend on the difference of positions alone."""
    g = np.random.default_rng(3)
    x = g.standard_normal((2, 3, 16))
    y = qk_norm_rope.norm(x, np.ones(16), 0.0)
    assert np.allclose((y * y).mean(axis=2), 1.0)
    ang = np.arange(50)[:, None] * np.exp(-np.arange(6))
    table = np.stack([np.cos(ang), np.sin(ang)], axis=2)
    dots = []
    for p in (0, 7, 30):
        r, _ = qk_norm_rope.rotate(x, table, [p, p + 11], halves)
        assert np.allclose((r * r).sum(2), (x * x).sum(2)) and np.array_equal(r[..., 12:], x[..., 12:])
        dots.append((r[0] * r[1]).sum(1))
    assert np.allclose(dots[0], dots[1]) and np.allclose(dots[0], dots[2])
    assert np.array_equal(qk_norm_rope.rotate(x, table, [-1, 50], halves)[0], x)


def test_oracle_attention_against_torch():
    g = torch.Generator().manual_seed(4)
    q, kv, own = (torch.randn(*n, generator=g, dtype=torch.float64) for n in ((7, 4, 8), (20, 2, 2, 8), (9, 2, 2, 8)))
    hidden = np.random.default_rng(5).random((3, 20)) < 0.4
    seg, start = [0, 3, 3, 6], [0, 4, 5, 9]
    out, _, _, _ = shared.attention(q.numpy(), kv.numpy(), hidden, seg, own.numpy(), start, 0.5)
    for b in range(3):
        rows = torch.cat([kv[torch.from_numpy(~hidden[b])], own[start[b]:start[b + 1]]]).repeat_interleave(2, dim=2)
        ref = torch.nn.functional.scaled_dot_product_attention(q[seg[b]:seg[b + 1]].transpose(0, 1), rows[:, 0].transpose(0, 1),
                                                               rows[:, 1].transpose(0, 1), scale=0.5).transpose(0, 1)
        assert np.allclose(out[seg[b]:seg[b + 1]], ref.numpy())
    assert (out[6] == 0).all()

"""Refusals of the 8-bit cache calls, before any device work (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2505_20600_amd import maskstep as MS

P = 4096    # an address that is checked but never read


def _cache(**kw):
    c = MS.Kv8Cache(MS.MS_BF16, 2, 100, 4, 64, 16, P, P)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _select(**kw):
    s = MS.Kv8Select(2, 100, None, P, P)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def _attn(**kw):
    a = MS.Kv8Attn(P, P, 10, 8, 2, P, None, P, 10, None, 0, P, 0.0)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


BAD_CACHE = [
    (dict(dtype=2), MS.MS_EDTYPE), (dict(dtype=-1), MS.MS_EDTYPE),
    (dict(n_caches=0), MS.MS_ESHAPE), (dict(n_caches=(1 << 20) + 1), MS.MS_ESHAPE),
    (dict(tokens=0), MS.MS_ESHAPE), (dict(tokens=(1 << 20) + 1), MS.MS_ESHAPE),
    (dict(n_kv_heads=0), MS.MS_ESHAPE), (dict(n_kv_heads=1025), MS.MS_ESHAPE),
    (dict(head_dim=0), MS.MS_ESHAPE), (dict(head_dim=12), MS.MS_ESHAPE), (dict(head_dim=136), MS.MS_ESHAPE),
    (dict(dtype=MS.MS_FP32, head_dim=72), MS.MS_ESHAPE),
    (dict(block=0), MS.MS_ESHAPE), (dict(block=24), MS.MS_ESHAPE), (dict(block=256), MS.MS_ESHAPE), (dict(block=-16), MS.MS_ESHAPE),
    (dict(tokens=1 << 20, n_kv_heads=32), MS.MS_ESHAPE),          # 2^20 x 2 x 32 x 64 = 2^32 bytes
    (dict(tokens=4095 << 7, n_kv_heads=32, head_dim=128), MS.MS_ESHAPE),   # 4095 MiB
    (dict(codes=None), MS.MS_EINVAL), (dict(scales=None), MS.MS_EINVAL), (dict(codes=P + 8), MS.MS_EALIGN),
]
BAD_SELECT = [
    (dict(batch=0), MS.MS_ESHAPE), (dict(batch=129, cache_of=P), MS.MS_ESHAPE), (dict(batch=3), MS.MS_ESHAPE),
    (dict(ld_keys=-1), MS.MS_ESHAPE), (dict(ld_keys=(1 << 20) + 1), MS.MS_ESHAPE),
    (dict(keys=P + 2), MS.MS_EALIGN), (dict(n_keys=P + 1), MS.MS_EALIGN), (dict(cache_of=P + 3), MS.MS_EALIGN),
]
BAD_ATTN = [
    (dict(rows=-1), MS.MS_ESHAPE), (dict(rows=(1 << 26) + 1), MS.MS_ESHAPE),
    (dict(rows=(1 << 24) + 1), MS.MS_ESHAPE),                        # x 8 heads above 2^27
    (dict(n_heads=0), MS.MS_ESHAPE), (dict(n_heads=6), MS.MS_ESHAPE), (dict(n_heads=2048), MS.MS_ESHAPE),
    (dict(n_seg=0), MS.MS_ESHAPE), (dict(n_seg=129, seg_req=P), MS.MS_ESHAPE), (dict(n_seg=3), MS.MS_ESHAPE),
    (dict(q=None), MS.MS_EINVAL), (dict(out=None), MS.MS_EINVAL), (dict(seg_start=None), MS.MS_EINVAL),
    (dict(q=P + 8), MS.MS_EALIGN), (dict(out=P + 4), MS.MS_EALIGN), (dict(fresh=P + 2), MS.MS_EALIGN),
    (dict(seg_start=P + 2), MS.MS_EALIGN), (dict(seg_req=P + 1), MS.MS_EALIGN), (dict(fresh_start=P + 2), MS.MS_EALIGN),
    (dict(fresh_list=P + 1), MS.MS_EALIGN),
    (dict(fresh_start=None), MS.MS_EINVAL), (dict(fresh_rows=-1), MS.MS_ESHAPE), (dict(fresh_list=P, fresh_entries=-1), MS.MS_ESHAPE),
    (dict(scale=float("nan")), MS.MS_EINVAL), (dict(scale=float("inf")), MS.MS_EINVAL),
    (dict(scale=3e38), MS.MS_EINVAL),                                # x log2 e is no float32
]
_id = lambda v: "-".join(f"{k}={x}" for k, x in v.items()) if isinstance(v, dict) else str(v)


def _attention(c, s, a, ws=None, n=0):
    return MS.load().ms_kv8_attention(C.byref(c), C.byref(s), C.byref(a), ws, n, None)


@pytest.mark.parametrize("kw,status", BAD_CACHE, ids=_id)
def test_bad_cache_is_refused_by_every_call(kw, status):
    lib = MS.load()
    c = _cache(**kw)
    assert lib.ms_kv8_quantize(C.byref(c), P, 1 << 21, 1 << 20, None, None) == status
    assert lib.mask_last_error()
    assert lib.ms_kv8_dequantize(C.byref(c), C.byref(_select()), P, 1 << 20, None) == status
    assert _attention(c, _select(), _attn(n_heads=4)) == status
    assert lib.ms_kv8_attention_workspace_bytes(C.byref(c), C.byref(_select()), C.byref(_attn(n_heads=4))) == 0
    assert lib.mask_last_error()


@pytest.mark.parametrize("kw,status", BAD_SELECT, ids=_id)
def test_bad_selection_is_refused(kw, status):
    lib = MS.load()
    s = _select(**kw)
    assert lib.ms_kv8_dequantize(C.byref(_cache()), C.byref(s), P, 100, None) == status
    assert _attention(_cache(), s, _attn()) == status


@pytest.mark.parametrize("kw,status", BAD_ATTN, ids=_id)
def test_bad_attention_arguments_are_refused(kw, status):
    assert _attention(_cache(), _select(), _attn(**kw)) == status
    assert MS.load().mask_last_error()


def test_null_descriptions_rows_and_strides_are_refused():
    lib = MS.load()
    c, s, a = _cache(), _select(), _attn()
    assert lib.ms_kv8_attention(None, C.byref(s), C.byref(a), None, 0, None) == MS.MS_EINVAL
    assert lib.ms_kv8_attention(C.byref(c), None, C.byref(a), None, 0, None) == MS.MS_EINVAL
    assert lib.ms_kv8_attention(C.byref(c), C.byref(s), None, None, 0, None) == MS.MS_EINVAL
    assert _attention(c, s, a, P + 8, 1 << 20) == MS.MS_EALIGN
    assert lib.ms_kv8_quantize(None, P, 200, 100, None, None) == MS.MS_EINVAL
    for kv, rows, stride, src, status in ((None, 200, 100, None, MS.MS_EINVAL), (P + 4, 200, 100, None, MS.MS_EALIGN),
                                          (P, 0, 100, None, MS.MS_ESHAPE), (P, 200, 99, None, MS.MS_ESHAPE),
                                          (P, 199, 100, None, MS.MS_ESHAPE), (P, 200, 101, None, MS.MS_ESHAPE),
                                          (P, 200, 1 << 62, None, MS.MS_ESHAPE), (P, 1 << 62, 100, None, MS.MS_ESHAPE),
                                          (P, 200, 100, P + 2, MS.MS_EALIGN)):
        assert lib.ms_kv8_quantize(C.byref(c), kv, rows, stride, src, None) == status
    for kv, stride, status in ((None, 100, MS.MS_EINVAL), (P + 2, 100, MS.MS_EALIGN), (P, 99, MS.MS_ESHAPE),
                               (P, 1 << 62, MS.MS_ESHAPE)):
        assert lib.ms_kv8_dequantize(C.byref(c), C.byref(s), kv, stride, None) == status
    for mask, b, t, keys, ld, n, status in ((None, 1, 8, P, 8, P, MS.MS_EINVAL), (P, 0, 8, P, 8, P, MS.MS_ESHAPE),
                                            (P, 129, 8, P, 8, P, MS.MS_ESHAPE), (P, 1, 0, P, 8, P, MS.MS_ESHAPE),
                                            (P, 1, 8, P, 7, P, MS.MS_ESHAPE), (P, 1, 8, None, 8, P, MS.MS_EINVAL),
                                            (P, 1, 8, P, 8, None, MS.MS_EINVAL), (P, 1, 8, P + 1, 8, P, MS.MS_EALIGN)):
        assert lib.ms_kv8_keys(mask, b, t, keys, ld, n, None) == status


@pytest.mark.parametrize("dtype,block,caches,tokens", [(MS.MS_BF16, 1, 1 << 20, 1), (MS.MS_BF16, 128, 1 << 17, 128),
                                                       (MS.MS_FP32, 32, 1 << 18, 31)])
def test_more_than_one_launch_can_write_is_refused(dtype, block, caches, tokens):
    """At 1024 heads of 8: 16 (bf16) or 32 (float32) KiB-pieces per row, K and V, tokens up to whole blocks of 16 or more."""
    lib = MS.load()
    at = _cache(dtype=dtype, n_caches=caches, tokens=tokens, n_kv_heads=1024, head_dim=8, block=block)
    assert caches * 2 * (16 if dtype == MS.MS_BF16 else 32) * max(16, block) >= 1 << 28
    for src in (None, P):
        assert lib.ms_kv8_quantize(C.byref(at), P, 1 << 30, tokens, src, None) == MS.MS_ESHAPE
        assert b"one call" in lib.mask_last_error()


def test_no_rows_is_not_an_error():
    assert _attention(_cache(), _select(), _attn(rows=0, q=None, out=None)) == MS.MS_OK
    assert MS.load().ms_kv8_attention_workspace_bytes(C.byref(_cache()), C.byref(_select()), C.byref(_attn(rows=0))) == 0
    assert not MS.load().mask_last_error()


def test_binding_refuses_wrong_tensors():
    """Shapes, types and places that the C interface cannot see (host tensors: every call refuses them)."""
    codes, scales = torch.zeros(2, 40, 2, 4, 64, dtype=torch.uint8), torch.zeros(2, 3, 2, 4, dtype=torch.uint8)
    kv, q = torch.zeros(2, 40, 2, 4, 64, dtype=torch.bfloat16), torch.zeros(10, 8, 64, dtype=torch.bfloat16)
    start = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(MS.MaskStepError, match="one GPU"):
        MS.ms_kv8_quantize(kv, codes, scales, block=16)
    with pytest.raises(MS.MaskStepError, match="one GPU"):
        MS.ms_kv8_dequantize(codes, scales, kv, block=16)
    with pytest.raises(MS.MaskStepError, match="one GPU"):
        MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start, block=16)
    with pytest.raises(MS.MaskStepError, match="mask must be"):
        MS.ms_kv8_keys(torch.zeros(2, 40, dtype=torch.uint8), torch.zeros(2, 40, dtype=torch.int32), start[:2])
    for c, s, block in ((codes[:, :, :1], scales, 16), (codes.float(), scales, 16), (codes.transpose(1, 2), scales, 16),
                        (codes, scales, 32), (codes, scales, 0), (codes, scales[:1], 16), (codes, scales.float(), 16)):
        with pytest.raises(MS.MaskStepError, match="must be contiguous bytes"):
            MS.ms_kv8_quantize(kv, c, s, block=block)
    with pytest.raises(MS.MaskStepError, match="bfloat16 or float32"):
        MS.ms_kv8_quantize(kv.half(), codes, scales, block=16)

"""What the Python binding of the 8-bit cache refuses before it hands addresses to the library (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2505_20600_amd import maskstep as MS

L, B, N, H, HD, BLOCK, S = 3, 2, 40, 4, 16, 16, 5


class _Reached(Exception):
    pass


class _Library:
    def mask_stack_forward_kv8(self, *a):
        raise _Reached


def _step():
    """A context as far as the binding's checks look at it."""
    s = MS.MaskStep.__new__(MS.MaskStep)
    s.desc = MS.ModelDesc(L, H * HD, H, 4, 5, 8, 3, 0, B, MS.MS_BF16, 1e-5)
    s.batch, s.handle, s._lib = B, None, _Library()
    return s


def _bytes(*shape):
    return torch.zeros(*shape, dtype=torch.uint8)


def _call(step=None, **kw):
    a = dict(codes=[_bytes(S, N, 2, H, HD) for _ in range(L)], scales=[_bytes(S, 3, 2, H) for _ in range(L)], block=BLOCK)
    a.update(kw)
    (step or _step()).stack_forward_kv8(None, 0, 0, a.pop("codes"), a.pop("scales"), 0, stream=1, **a)


def _pinned(**kw):
    a = dict(codes=[_bytes(B, N, 2, H, HD) for _ in range(L)], pinned=True, slots=[_bytes(B, N, 2, H, HD)], copy_stream=2)
    a.update(kw)
    _call(**a)


def _with(n, at, t):
    return [t if i == at else x for i, x in enumerate(n)]


CODES = [_bytes(S, N, 2, H, HD) for _ in range(L)]
SCALES = [_bytes(S, 3, 2, H) for _ in range(L)]
HOST = [_bytes(B, N, 2, H, HD) for _ in range(L)]


@pytest.mark.parametrize("kw", [
    dict(scales=SCALES[:2]), dict(codes=CODES[:2]), dict(codes=CODES + CODES[:1]),
    dict(block=8), dict(block=32), dict(block=0), dict(block=-16), dict(block=16.0),
    dict(scales=_with(SCALES, 1, _bytes(S - 1, 3, 2, H))), dict(scales=_with(SCALES, 2, _bytes(S, 2, 2, H))),
    dict(scales=_with(SCALES, 0, SCALES[0].float())), dict(scales=_with(SCALES, 1, _bytes(3, S, 2, H).transpose(0, 1))),
    dict(codes=_with(CODES, 1, _bytes(S - 1, N, 2, H, HD))), dict(codes=_with(CODES, 2, _bytes(S, N - 1, 2, H, HD))),
    dict(codes=_with(CODES, 0, _bytes(S, N, 2, H, HD // 2))), dict(codes=_with(CODES, 0, CODES[0].to(torch.bfloat16))),
    dict(codes=_with(CODES, 1, _bytes(S, 2, N, H, HD).transpose(1, 2)))], ids=lambda kw: "-".join(kw))
def test_step_refuses_caches_that_are_not_as_large_as_said(kw):
    with pytest.raises(MS.MaskStepError, match="layer|block|contiguous"):
        _call(**kw)


@pytest.mark.parametrize("kw", [
    dict(codes=_with(HOST, 1, _bytes(B - 1, N, 2, H, HD))), dict(codes=_with(HOST, 1, HOST[0].float())),
    dict(slots=[_bytes(B, N, 2, H, HD - 1)]), dict(slots=[_bytes(B, N, 2, H, HD), _bytes(B, N, H, HD)]),
    dict(slots=[_bytes(B, 2, N, H, HD).transpose(1, 2)]),
    dict(codes=None, per_request=[[_bytes(N, 2, H, HD)] * B] * (L - 1)), dict(codes=None, per_request=[[_bytes(N, 2, H, HD)]] * L),
    dict(codes=None, per_request=[[_bytes(N - 1, 2, H, HD), None]] * L)], ids=lambda kw: "-".join(kw))
def test_streamed_step_refuses_buffers_that_are_too_small(kw):
    with pytest.raises(MS.MaskStepError, match="layer|contiguous"):
        _pinned(**kw)


def test_step_refuses_host_scales():
    for f in (_call, _pinned, lambda: _pinned(codes=None, per_request=[[None, _bytes(N, 2, H, HD)]] * L),
              lambda: _pinned(slots=[torch.zeros(B, N, 2, H, HD, dtype=torch.bfloat16)])):
        with pytest.raises(MS.MaskStepError, match="on one GPU"):
            f()


# ------------------------------------------------------------------ workspace

@pytest.mark.parametrize("rows", [1, 150, 600])
@pytest.mark.parametrize("by", ["cache_of", "n_keys", "keys", "fresh_start", "codes"])
def test_workspace_is_planned_for_the_calls_requests(rows, by):
    """Two and three segments per request: the bytes that the library plans for the call's own batch, whichever table says
    how many requests there are."""
    lib, T, fresh_rows = MS.load(), 3000, 7000
    codes = torch.empty(2 if by == "codes" else 9, T, 2, 3, 64, dtype=torch.uint8)
    start, req = torch.zeros(6, dtype=torch.int32), torch.zeros(5, dtype=torch.int32)
    q, fresh = torch.empty(5 * rows, 6, 64, dtype=torch.bfloat16), torch.empty(fresh_rows, 2, 3, 64, dtype=torch.bfloat16)
    tables = {"cache_of": torch.zeros(2, dtype=torch.int32), "n_keys": torch.zeros(2, dtype=torch.int32),
              "keys": torch.zeros(2, 2000, dtype=torch.int32), "fresh_start": torch.zeros(3, dtype=torch.int32)}
    kw = {"fresh": fresh} if by == "codes" else {by: tables[by], "fresh": fresh}
    cache = MS.Kv8Cache(MS.MS_BF16, codes.shape[0], T, 3, 64, 64, 16, 16)
    ld = 2000 if by == "keys" else 0
    args = MS.Kv8Attn(16, 16, 5 * rows, 6, 5, 16, 16, 16, fresh_rows, None, 0, 16, 0.0)

    def planned(batch):
        sel = MS.Kv8Select(batch, ld, 16, 16 if ld else None, None)
        return lib.ms_kv8_attention_workspace_bytes(C.byref(cache), C.byref(sel), C.byref(args))
    assert MS.ms_kv8_attention_workspace_bytes(q, codes, start, seg_req=req, **kw) == planned(2)
    if rows == 150:
        assert planned(2) != planned(5)
    one = MS.ms_kv8_attention_workspace_bytes(q, codes, start, fresh=fresh)
    assert by == "keys" or one == planned(5)


# ------------------------------------------------------------------ score scale

@pytest.mark.parametrize("scale", [0, 0.0, -0.0, 1e-60])
def test_a_score_scale_of_zero_is_refused(scale):
    """The library takes 0 as 1 / sqrt(head_dim)."""
    codes, scales = torch.zeros(1, 40, 2, 4, 64, dtype=torch.uint8), torch.zeros(1, 3, 2, 4, dtype=torch.uint8)
    q, start = torch.zeros(10, 8, 64, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(MS.MaskStepError, match="is 0 in float32"):
        MS.ms_kv8_attention(q, codes, scales, q, start, block=16, scale=scale)
    with pytest.raises(MS.MaskStepError, match="one GPU"):
        MS.ms_kv8_attention(q, codes, scales, q, start, block=16, scale=1e-40)


# ------------------------------------------------------------------ launch sizes

@pytest.mark.parametrize("dtype,heads,group,hd", [(MS.MS_BF16, 1, 1, 8), (MS.MS_BF16, 64, 8, 64), (MS.MS_BF16, 1024, 1, 16),
                                                  (MS.MS_FP32, 1, 1, 8), (MS.MS_FP32, 1024, 1, 64)])
@pytest.mark.parametrize("segments", [1, 8, 128])
def test_key_ranges_stay_within_one_launch(dtype, heads, group, hd, segments):
    """However many keys are to be expected (here a list of up to 2^28 entries), the planned ranges are launches below
    2^32 threads: 256 per 16 query slots (or more), K/V head and range, and a wave per row and head for the join."""
    lib, split = MS.load(), 0
    cache = MS.Kv8Cache(dtype, 128, 64, heads, hd, 64, 16, 16)
    sel = MS.Kv8Select(segments, 0, 16, None, None)
    for bits in range(27):
        rows = 1 << bits
        if rows * heads * group > 1 << 27:
            break
        for entries in (1 << 20, 1 << 28):
            a = MS.Kv8Attn(16, 16, rows, heads * group, segments, 16, 16, 16, 1, 16, entries, 16, 0.0)
            n = lib.ms_kv8_attention_workspace_bytes(C.byref(cache), C.byref(sel), C.byref(a)) // (rows * heads * group * (hd + 2) * 4)
            assert not lib.mask_last_error()
            split = max(split, n)
            if n:
                tile = 128 if dtype == MS.MS_BF16 and rows * group > 8 * 128 * segments else 16   # many rows: the form for many
                assert (rows * group // tile * n) * heads * 256 < 1 << 32
                assert rows * heads * group * 64 < 1 << 32
    assert split > 1

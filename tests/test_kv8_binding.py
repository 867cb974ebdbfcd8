"""What the Python binding of the 8-bit cache refuses before it hands addresses to the library (no GPU needed)."""
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

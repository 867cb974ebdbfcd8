"""4-bit row products on the GPU at the sizes, epilogues and scale bytes at the edges of what they take, against the float64
oracle."""
import numpy as np
import pytest
import torch

from oracle import mx4
from paper_2505_20600_amd import maskstep as MS
from tests import block_ops_forms as F
from tests.test_gpu_block_ops import DEV, DT, _np, _operand, _product_bound, _randn, _within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N", [(1 << 20, 1 << 11), (1 << 26, 20)])
def test_product_of_most_outputs(M, N):
    """2^31 outputs, and 2^26 rows: offsets that pass 32 bits. Rows at both ends, around the middle and at random."""
    g = torch.Generator().manual_seed(N)
    K = 32
    w, bias = _operand(g, N, K), _randn(g, (N,), "bf16")
    dg = torch.Generator(device=DEV).manual_seed(N)
    codes = torch.randint(0, 256, (M, K // 2), generator=dg, device=DEV, dtype=torch.uint8)
    scales = torch.randint(120, 130, (M, 1), generator=dg, device=DEV, dtype=torch.uint8)
    out = torch.empty(M, N, dtype=torch.bfloat16, device=DEV)
    out[-300:] = 7.0
    MS.ms_mx4_linear(codes, scales, *w, bias, out)
    at = torch.cat([torch.arange(300), torch.arange(M // 2 - 150, M // 2 + 150), torch.arange(M - 300, M), torch.randint(0, M, (300,), generator=g)])
    a = [t[at.to(DEV)].cpu().numpy() for t in (codes, scales)]
    want, size = mx4.linear(mx4.values(*a), mx4.values(w[0].cpu().numpy(), w[1].cpu().numpy()), _np(bias))
    _within(_np(out[at.to(DEV)]), want, _product_bound(want, size, K, "bf16"), f"{M}x{N}")


def _values(codes, scales):
    """float64 values of codes on the GPU."""
    c = torch.stack([codes & 15, codes >> 4], dim=2).flatten(1).long()
    grid = torch.tensor(np.concatenate([mx4.MAGNITUDES, -mx4.MAGNITUDES]), device=DEV)
    s = torch.exp2(scales.double() - 127.0)
    return grid[c] * torch.where(scales == 255, torch.full_like(s, np.nan), s).repeat_interleave(32, 1)


def _random_operand(g, rows, K, exponent):
    """Any codes, scale bytes of a few sizes around an exponent."""
    return (torch.randint(0, 256, (rows, K // 2), generator=g, device=DEV, dtype=torch.uint8),
            torch.randint(126 + exponent, 130 + exponent, (rows, K // 32), generator=g, device=DEV, dtype=torch.uint8))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("epilogue", ["bias", "resid", "gelu"])
@pytest.mark.parametrize("tile,split", F.PRODUCT_FORMS)
def test_every_form_with_every_epilogue(dtype, epilogue, tile, split):
    """Residuals from a buffer of their own and in place, with the workspace and without."""
    M, N, K = F.product_of(tile, split)
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    a, w = _random_operand(g, M, K, -1), _random_operand(g, N, K, -2 - K.bit_length() // 2)
    bias, resid = (torch.randn(*n, generator=g, device=DEV).to(DT[dtype]) for n in ((N,), (M, N)))
    av, wv = _values(*a), _values(*w)
    want, size = av @ wv.t().contiguous() + bias.double(), av.abs() @ wv.abs().t().contiguous() + bias.double().abs()
    r = resid if epilogue == "resid" else None
    if epilogue == "gelu":
        want = 0.5 * want * (1.0 + torch.special.erf(want * 0.5 ** 0.5))
    elif r is not None:
        want = want + r.double()
    want, size = want.cpu().numpy(), size.cpu().numpy()
    bound = _product_bound(want, size, K, dtype, None if r is None else _np(r))
    need = MS.ms_mx4_linear_workspace_bytes(a[0], w[0])
    assert MS.ms_mx4_linear_plan(a[0], w[0], need)[0] == tile and (need > 0) == split
    for ws in [None] + [torch.full((need + 16,), 0xff, dtype=torch.uint8, device=DEV)] * (need > 0):
        out = torch.full((M + 1, N), 7.0, dtype=DT[dtype], device=DEV)
        MS.ms_mx4_linear(*a, *w, bias, out[:M], resid=r, gelu=epilogue == "gelu", workspace=ws)
        _within(_np(out[:M]), want, bound, f"{M}x{N}x{K} {'one range' if ws is None else 'ranges'}")
        assert bool((out[M] == 7.0).all())
        if r is not None:       # onto the residual stream: the same sums, so the same bits
            onto = torch.cat([r, torch.full_like(r[:1], 7.0)])
            MS.ms_mx4_linear(*a, *w, bias, onto[:M], resid=onto[:M], workspace=ws)
            assert torch.equal(onto, out)


@pytest.mark.parametrize("M,N", [(20, 24), (300, 264)])
@pytest.mark.parametrize("K", [32, 640])
def test_products_of_the_outermost_scales(M, N, K):
    """Scale bytes 0, 1, 2, 252, 253, 254, which the codes' own writer leaves out at the ends, against the ones that bring the
    products near 1; others fall to nothing. Products beyond float32 are infinite (or NaN where infinities cancel)."""
    g = torch.Generator(device=DEV).manual_seed(K)
    a, w = _random_operand(g, M, K, 0), _random_operand(g, N, K, 0)
    ends = torch.tensor([0, 1, 2, 252, 253, 254], dtype=torch.uint8, device=DEV)
    a[1][:] = ends[torch.randint(0, 6, (M, 1), generator=g, device=DEV)]
    w[1][:] = ends[torch.randint(0, 6, (N, 1), generator=g, device=DEV)]
    out = torch.empty(M, N, device=DEV)
    MS.ms_mx4_linear(*a, *w, torch.zeros(N, device=DEV), out)
    av, wv = _values(*a), _values(*w)
    want, size = (av @ wv.t().contiguous()).cpu().numpy(), (av.abs() @ wv.abs().t().contiguous()).cpu().numpy()
    got, near = _np(out), size < 2.0 ** 100
    assert 0.5 < near.mean() < 0.9      # a third or so meets one of the same end
    assert bool((np.abs(got - want)[near] <= _product_bound(want, size, K, "fp32")[near]).all())
    assert not np.isfinite(got[np.abs(want) > 2.0 ** 130]).any()


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_outermost_scales_are_read_back(dtype):
    """Every code under scale bytes 0, 253 and 254: exact where the type holds it (subnormals too), infinite beyond."""
    exps = [0, 253, 254]
    codes = torch.arange(256, dtype=torch.uint8).repeat(len(exps), 1).to(DEV)
    scales = torch.tensor(exps, dtype=torch.uint8)[:, None].repeat(1, 16).to(DEV)
    x = torch.empty(len(exps), 512, dtype=DT[dtype], device=DEV)
    MS.ms_mx4_dequantize(codes, scales, x)
    want = torch.from_numpy(mx4.values(codes.cpu().numpy(), scales.cpu().numpy()))
    want = torch.where(want.abs() >= 2.0 ** 128, want.sign() * np.inf, want)
    assert np.array_equal(_np(x), want.numpy())

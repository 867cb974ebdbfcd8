"""4-bit row products on the GPU at the edges of what they take, against the float64 oracle."""
import pytest
import torch

from oracle import mx4
from paper_2505_20600_amd import maskstep as MS
from tests.test_gpu_block_ops import DEV, _np, _operand, _product_bound, _randn, _within

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

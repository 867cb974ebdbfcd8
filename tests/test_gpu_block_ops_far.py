"""Per-head norms with rotation at the far ends of their types, against the float64 oracle."""
import numpy as np
import pytest
import torch

from tests.test_gpu_block_ops import DT, _qk_case, _qk_check

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------ norms

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,H,G,hd,rot,halves", [(6, 5, 2, 72, 72, False), (70, 4, 4, 64, 64, True), (9, 3, 3, 40, 18, True), (3, 33, 1, 128, 96, False),
                                                 (5000, 2, 1, 24, 24, False)])
@pytest.mark.parametrize("eps", [0.0, 2.0 ** -149, 2.0 ** -130, 2.0 ** -100, 2.0 ** -80, 1e-6, 2.0 ** 100])
def test_norms_of_heads_far_from_one(dtype, M, H, G, hd, rot, halves, eps):
    """Heads from the smallest subnormals to the type's largest values side by side: each has a root mean square of its own, which
    float32 holds though it may not hold the squares. Within a head values spread over 2^40."""
    g = torch.Generator().manual_seed(M + hd)
    s = _qk_case(g, dtype, M, H, G, hd, rot, 8, 300, M + 50)
    n = H + 2 * G
    far = torch.tensor([-133.0, -126.0, -110.0, -75.0, -64.0, -62.0, -40.0, 0.0, 40.0, 62.0, 64.0, 66.0, 100.0, 122.0], dtype=torch.float64)
    x = torch.randn(M, n, hd, generator=g, dtype=torch.float64) * torch.exp2(torch.randint(-40, 1, (M, n, hd), generator=g).double())
    x[..., 0] = torch.where(torch.rand(M, n, generator=g) < 0.5, 2.0, -3.0).double()      # of the head's own size, so that none is all zeros
    x *= torch.exp2(far[torch.randint(0, len(far), (M, n), generator=g)])[:, :, None]
    s["qkv"].copy_(x.view(M, -1).to(DT[dtype]))
    assert bool(torch.isfinite(s["qkv"].float()).all()) and bool((s["qkv"].view(M, n, hd)[..., 0] != 0).all())
    _qk_check(s, dtype, H, G, hd, halves, float(np.float32(eps)))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("eps", [0.03, 1.0, 4.0, 300.0])
@pytest.mark.parametrize("M", [3, 5000])
def test_norms_with_eps_of_the_size_of_the_mean_square(dtype, eps, M):
    """The heads' mean square is near 4: eps is inside the root, and it is the caller's."""
    g = torch.Generator().manual_seed(M)
    s = _qk_case(g, dtype, M, 6, 2, 64, 64, 0, 60, M + 5)
    _qk_check(s, dtype, 6, 2, 64, True, float(np.float32(eps)))

"""Per-head norms with rotation and attention over a shared prefix at the far ends of their types, against the float64
oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import shared
from tests.test_gpu_block_ops import DEV, DT, _attend, _attend_bound, _batch, _np, _qk_case, _qk_check, _within

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


# ------------------------------------------------------------------ attention

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [(3,), (20, 9), (60, 140), (800, 7)], ids=lambda r: f"{sum(r)}")
@pytest.mark.parametrize("values", ["one", "both signs", "few"])
@pytest.mark.parametrize("ws", [None, "need"])
def test_values_near_the_largest_of_the_type(dtype, rows, values, ws):
    """Results are means of the values, so they are finite where the values are, whatever the weights sum to."""
    g = torch.Generator().manual_seed(sum(rows))
    s = _batch(g, dtype, rows, 700, 2, 64, 1, hide=0.2)
    big = 3e38
    for kv in (s["kv"], s["fresh"]):
        v = kv[:, 1]
        if values == "one":
            v.fill_(big)
        elif values == "both signs":
            v.copy_(torch.where(torch.rand(v.shape, generator=g) < 0.5, big, -big).to(DT[dtype]).to(DEV))
        else:
            v[::97] = big
    hd = s["q"].shape[2]
    want, spread, size, reach = shared.attention(_np(s["q"]), _np(s["kv"]), s["hidden"].numpy(), s["seg"], _np(s["fresh"]), s["own"], 1 / math.sqrt(hd))
    keys = len(s["kv"]) + len(s["fresh"])
    _within(_np(_attend(s, ws)), want, _attend_bound(want, spread, size, reach, keys, hd, dtype), f"{values} {ws}")

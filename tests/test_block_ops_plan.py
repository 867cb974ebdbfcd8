"""The forms that the 4-bit product and the shared attention choose (no GPU needed)."""
import ctypes as C

import pytest
import torch

from paper_2505_20600_amd import maskstep as MS
from tests import block_ops_forms as F

BF, F32 = MS.MS_BF16, MS.MS_FP32


@pytest.mark.parametrize("tile,split", F.PRODUCT_FORMS)
def test_every_form_of_the_product_has_a_size(tile, split):
    M, N, K = F.product_of(tile, split)
    t, r = F.product_plan(M, N, K)
    assert t == tile and (r > 1) == split
    need = MS.load().ms_mx4_linear_workspace_bytes(M, N, K)
    assert need == (4 * r * M * N if r > 1 else 0)
    assert F.product_plan(M, N, K, need) == (t, r) and F.product_plan(M, N, K, 0)[1] == 1


@pytest.mark.parametrize("dtype,hd,tile,split", [(d, hd, *f) for d in F.HEAD_DIMS for hd in F.HEAD_DIMS[d] for f in F.ATTENTION_FORMS[d]])
def test_every_form_of_the_attention_has_a_size(dtype, hd, tile, split):
    rows, G, group, T = F.attention_of(dtype, hd, tile, split)
    t, r = F.attention_plan(dtype, rows, G, group, hd, T, rows)
    assert t == tile and (r > 1) == split
    assert F.attention_plan(dtype, rows, G, group, hd, T, rows, 0) == (t, 1)
    one = 4 * rows * G * group * (hd + 2)
    assert F.attention_plan(dtype, rows, G, group, hd, T, rows, r * one) == (t, r)
    assert F.attention_plan(dtype, rows, G, group, hd, T, rows, r * one - 1) == (t, max(1, r - 1))


def test_plans_of_shapes():
    """The binding's calls for tensors, which need not be on a GPU, and of sizes without rows."""
    e = lambda *s, dt=torch.bfloat16: torch.empty(*s, dtype=dt)
    codes = lambda rows, cols: e(rows, cols // 2, dt=torch.uint8)
    M, N, K = F.product_of(64, True)
    assert MS.ms_mx4_linear_plan(codes(M, K), codes(N, K), F.PLENTY) == F.product_plan(M, N, K)
    assert MS.ms_mx4_linear_plan(codes(M, K), codes(N, K)) == F.product_plan(M, N, K, 0)
    assert MS.ms_mx4_linear_plan(codes(0, K), codes(N, K), F.PLENTY)[1] == 1
    rows, G, group, T = F.attention_of("bf16", 64, 128, True)
    q, kv, fresh = e(rows, G * group, 64), e(T, 2, G, 64), e(rows, 2, G, 64)
    assert MS.ms_shared_attention_plan(q, kv, fresh=fresh, workspace_bytes=F.PLENTY) == F.attention_plan("bf16", rows, G, group, 64, T, rows)
    assert MS.ms_shared_attention_plan(q[:0], kv, workspace_bytes=F.PLENTY)[1] == 1


def test_refusals_of_plans():
    lib, t, r = MS.load(), C.c_int32(), C.c_int32()
    tp, rp = C.byref(t), C.byref(r)
    assert lib.ms_mx4_linear_plan(5, 6, 64, 0, tp, rp) == MS.MS_ESHAPE
    assert lib.ms_mx4_linear_plan(5, 8, 64, 0, None, rp) == MS.MS_EINVAL and lib.ms_mx4_linear_plan(5, 8, 64, 0, tp, None) == MS.MS_EINVAL
    a = MS.SharedAttn(F.P, F.P, 10, 8, 4, 64, F.P, 100, 1, None, F.P, None, 0, None, 0.0)
    assert lib.ms_shared_attention_plan(BF, C.byref(a), 0, None, rp) == MS.MS_EINVAL
    assert lib.ms_shared_attention_plan(BF, C.byref(a), 0, tp, None) == MS.MS_EINVAL
    assert lib.ms_shared_attention_plan(9, C.byref(a), 0, tp, rp) == MS.MS_EDTYPE and lib.mask_last_error()
    assert lib.ms_shared_attention_plan(BF, None, 0, tp, rp) == MS.MS_EINVAL
    assert lib.ms_shared_attention_plan(F32, C.byref(a), 0, tp, rp) == MS.MS_OK and not lib.mask_last_error()
    with pytest.raises(MS.MaskStepError):
        MS.ms_shared_attention_plan(torch.empty(3, 4, 12), torch.empty(9, 2, 4, 12))
    with pytest.raises(MS.MaskStepError):
        MS.ms_mx4_linear_plan(torch.empty(3, 20, dtype=torch.uint8), torch.empty(8, 20, dtype=torch.uint8))

"""The documented limits of the 4-bit product, on both sides, before any device work (no GPU needed)."""
import pytest

from paper_2505_20600_amd import maskstep as MS


@pytest.mark.parametrize("M,N", [(1 << 20, 1 << 11), (1 << 11, 1 << 20), (1 << 26, 32), (1 << 26, 20), (1 << 26, 4), ((1 << 31) // 36, 36), (1, 1 << 20)])
@pytest.mark.parametrize("K", [32, 1 << 20])
def test_products_of_up_to_2_to_the_31_outputs_are_taken(M, N, K):
    lib = MS.load()
    lib.ms_mx4_linear_workspace_bytes(M, N, K)
    assert not lib.mask_last_error(), lib.mask_last_error()


@pytest.mark.parametrize("M,N", [((1 << 20) + 1, 1 << 11), ((1 << 11) + 1, 1 << 20), (1 << 26, 36), ((1 << 31) // 36 + 1, 36)])
def test_products_of_more_outputs_are_refused(M, N):
    lib = MS.load()
    assert lib.ms_mx4_linear_workspace_bytes(M, N, 64) == 0 and b"2^31" in lib.mask_last_error()
    P = 4096    # an address that is checked but never read
    assert lib.ms_mx4_linear(MS.MS_BF16, M, N, 64, P, P, P, P, P, None, P, MS.MS_EPI_BIAS, None, 0, None) == MS.MS_ESHAPE

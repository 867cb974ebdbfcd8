"""Sizes at which the 4-bit product and the shared attention take each of their forms, found by asking the library, so that a test of
a form still tests it after the choice has changed."""
import ctypes as C
import functools

from paper_2505_20600_amd import maskstep as MS

P = 4096            # an address that is checked but never read
PLENTY = 1 << 60    # bytes of workspace

# (tile, several ranges) of the product
PRODUCT_FORMS = [(16, False), (64, False), (64, True), (128, False), (128, True), (256, False), (256, True)]
# (tile, several ranges) of the attention
ATTENTION_FORMS = {"bf16": [(16, False), (16, True), (32, False), (32, True), (128, False), (128, True)],
                   "fp32": [(16, False), (16, True), (32, False)]}
HEAD_DIMS = {"bf16": range(8, 129, 8), "fp32": range(8, 65, 8)}


def product_plan(M, N, K, ws=PLENTY):
    t, r = C.c_int32(), C.c_int32()
    assert MS.load().ms_mx4_linear_plan(M, N, K, ws, C.byref(t), C.byref(r)) == MS.MS_OK, MS.load().mask_last_error()
    return t.value, r.value


@functools.lru_cache(None)
def product_of(tile, split):
    """Least work (M, N, K), ragged where the form allows it, of a product in this form."""
    sizes = [(M, N, K) for M in (5, 33, 270, 1030, 1500, 2049) for N in (100, 772, 1028, 2052, 4036) for K in (288, 672, 1056, 4128, 12832, 24608)]
    for M, N, K in sorted(sizes, key=lambda s: s[0] * s[1] * s[2]):
        t, r = product_plan(M, N, K)
        if t == tile and (r > 1) == split:
            return M, N, K
    raise AssertionError(f"no size takes tiles of {tile} with {'several ranges' if split else 'one range'}")


def attention_plan(dtype, rows, kv_heads, group, head_dim, tokens, own, ws=PLENTY):
    a = MS.SharedAttn(P, P, rows, kv_heads * group, kv_heads, head_dim, P, tokens, 1, None, P, P, own, P, 0.0)
    t, r = C.c_int32(), C.c_int32()
    code = MS.MS_BF16 if dtype == "bf16" else MS.MS_FP32
    assert MS.load().ms_shared_attention_plan(code, C.byref(a), ws, C.byref(t), C.byref(r)) == MS.MS_OK, MS.load().mask_last_error()
    return t.value, r.value


@functools.lru_cache(None)
def attention_of(dtype, head_dim, tile, split):
    """Least work (rows, kv_heads, group, tokens) of a batch with as many own rows in this form."""
    sizes = [(rows, G, group, T) for rows in (3, 17, 200, 403, 701, 931) for G in (1, 2, 8, 16, 24) for group in (1, 2) for T in (70, 131, 331, 700, 1500)]
    for rows, G, group, T in sorted(sizes, key=lambda s: s[0] * s[1] * s[2] * (s[3] + s[0] // 4)):
        t, r = attention_plan(dtype, rows, G, group, head_dim, T, rows)
        if t == tile and (r > 1) == split:
            return rows, G, group, T
    raise AssertionError(f"no size takes {tile} slots with {'several ranges' if split else 'one range'} at head_dim {head_dim} in {dtype}")

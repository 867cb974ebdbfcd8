"""4-bit row products, per-head norms with rotation, and attention over a shared prefix on the GPU against the float64
oracle: codes, scales, read-back values and copied rows are exact, everything else is held to the roundings it makes."""
import math

import numpy as np
import pytest
import torch

from oracle import mx4, qk_norm_rope, shared
from paper_2505_20600_amd import maskstep as MS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}      # half a step, relative


def _np(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _randn(g, shape, dtype, width=1.0):
    return (torch.randn(*shape, generator=g) * width).to(DT[dtype]).to(DEV)


def _within(got, want, bound, what=""):
    off = np.abs(got - want)
    worst = float((off / np.maximum(bound, 1e-300)).max()) if off.size else 0.0
    print(f"[bound] {what}: largest error {float(off.max()) if off.size else 0:.3e}, {worst:.3f} of its bound", flush=True)
    assert np.isfinite(got).all() and bool((off <= bound).all()), f"{what}: {worst:.3f} times the bound"


# ------------------------------------------------------------------ 4-bit codes

def _empty_codes(rows, cols, fill=0x55):
    return (torch.full((rows, cols // 2), fill, dtype=torch.uint8, device=DEV),
            torch.full((rows, cols // 32), fill, dtype=torch.uint8, device=DEV))


def _same_codes(got, want):
    return bool(np.array_equal(got.cpu().numpy(), want))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 32), (3, 64), (5, 1056), (130, 96), (33, 4096), (1, 16384), (1000, 160), (4099, 2080)])
def test_codes_are_exact_and_read_back(dtype, rows, cols):
    g = torch.Generator().manual_seed(rows + cols)
    x = _randn(g, (rows, cols), dtype) * torch.exp(2 * torch.randn(rows, cols // 32, generator=g)).repeat_interleave(32, 1).to(DEV).to(DT[dtype])
    codes, scales = _empty_codes(rows + 1, cols)
    MS.ms_mx4_quantize(x, codes[:rows], scales[:rows])
    c, s = mx4.quantize(_np(x))
    assert _same_codes(scales[:rows], s) and _same_codes(codes[:rows], c)
    assert bool((codes[rows] == 0x55).all()) and bool((scales[rows] == 0x55).all())       # nothing past the last row
    back = torch.full((rows + 1, cols), 7.0, dtype=DT[dtype], device=DEV)
    MS.ms_mx4_dequantize(codes[:rows], scales[:rows], back[:rows])
    assert np.array_equal(_np(back[:rows]), mx4.values(c, s)) and bool((back[rows] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_codes_of_special_values(dtype):
    """Zeros of both signs, NaN, infinities, the type's largest and smallest values, ties, the border of seven times the scale."""
    big, tiny = torch.finfo(DT[dtype]).max, torch.finfo(DT[dtype]).tiny
    g = torch.Generator().manual_seed(4)
    x = torch.randn(16, 64, generator=g)
    x[0] = 0.0
    x[0, ::2] = -0.0
    x[1, 3], x[1, 40] = math.nan, math.inf
    x[2, 5] = -math.inf
    x[3] = math.nan
    x[4] *= big / 8
    x[4, 1], x[4, 33] = -big, big
    x[5] *= tiny
    x[6] = tiny * 2.0 ** -6 * torch.randint(-8, 9, (64,), generator=g)                    # subnormal
    x[7] = torch.randint(-28, 29, (64,), generator=g) * 0.25                              # ties
    x[7, 0], x[7, 32] = 7.0, -7.0
    x[8] = torch.randint(-28, 29, (64,), generator=g) * 0.25
    x[8, 0], x[8, 32] = 6.0, 4.0
    x[9] = 1.0
    x[9, 0], x[9, 40] = 7.0 + 2.0 ** -5, 7.0
    x[10] *= 2.0 ** -120
    x[11] = 5.0
    x[12], x[12, 7] = 1e-9, 3.0
    x[13] = -big
    x[14] = torch.where(torch.arange(64) % 2 == 0, 3.5, -3.5)
    x = x.to(DT[dtype]).to(DEV)
    codes, scales = _empty_codes(16, 64)
    MS.ms_mx4_quantize(x, codes, scales)
    c, s = mx4.quantize(_np(x))
    assert _same_codes(scales, s) and _same_codes(codes, c)
    back = torch.empty_like(x)
    MS.ms_mx4_dequantize(codes, scales, back)
    assert np.array_equal(_np(back), mx4.values(c, s), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_every_code_and_scale_byte_is_read(dtype):
    """All 256 bytes of codes under scale bytes from 1 to 252 and 255."""
    exps = [1, 2, 60, 126, 127, 128, 200, 251, 252, 255]
    codes = torch.arange(256, dtype=torch.uint8).repeat(len(exps), 1).to(DEV)
    scales = torch.tensor(exps, dtype=torch.uint8)[:, None].repeat(1, 16).to(DEV)
    x = torch.empty(len(exps), 512, dtype=DT[dtype], device=DEV)
    MS.ms_mx4_dequantize(codes, scales, x)
    assert np.array_equal(_np(x), mx4.values(codes.cpu().numpy(), scales.cpu().numpy()), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_rows_that_lie_apart(dtype):
    g = torch.Generator().manual_seed(8)
    wide = _randn(g, (9, 200), dtype)
    codes, scales = _empty_codes(9, 96)
    MS.ms_mx4_quantize(wide[:, 8:104], codes, scales)
    c, s = mx4.quantize(_np(wide[:, 8:104]))
    assert _same_codes(scales, s) and _same_codes(codes, c)
    back = wide.clone()
    MS.ms_mx4_dequantize(codes, scales, back[:, 8:104])
    assert np.array_equal(_np(back[:, 8:104]), mx4.values(c, s))
    assert torch.equal(back[:, :8], wide[:, :8]) and torch.equal(back[:, 104:], wide[:, 104:])


# ------------------------------------------------------------------ products

def _operand(g, rows, cols, width=1.0):
    c, s = mx4.quantize((torch.randn(rows, cols, generator=g) * width * torch.exp(torch.randn(rows, 1, generator=g))).double().numpy())
    return torch.from_numpy(c).to(DEV), torch.from_numpy(s).to(DEV)


def _product_bound(want, size, K, dtype, resid=None):
    """float32 sums of K exact products and a bias in any order, GELU's slope (below 1.13) and 3.3e-7, one rounding."""
    e = 1.13 * (K + 2) * 2.0 ** -24 * size + 3.3e-7
    if resid is not None:
        e = e + 2.0 ** -24 * (np.abs(resid) + np.abs(want))
    return e + HALF[dtype] * (np.abs(want) + e)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("epilogue", ["bias", "resid", "gelu"])
@pytest.mark.parametrize("M,N,K", [(1, 4, 32), (1, 260, 1056), (3, 100, 64), (16, 64, 256), (17, 132, 288), (33, 68, 2048),
                                   (65, 1000, 96), (128, 128, 512), (129, 132, 544), (200, 300, 1152), (257, 520, 800), (300, 264, 4128)])
def test_product(dtype, epilogue, M, N, K):
    g = torch.Generator().manual_seed(M + N + K)
    a, w = _operand(g, M, K), _operand(g, N, K, 1.0 / math.sqrt(K))
    bias, resid = _randn(g, (N,), dtype), _randn(g, (M, N), dtype)
    out = torch.full((M + 1, N), 7.0, dtype=DT[dtype], device=DEV)
    r = resid if epilogue == "resid" else None
    want, size = mx4.linear(mx4.values(a[0].cpu().numpy(), a[1].cpu().numpy()), mx4.values(w[0].cpu().numpy(), w[1].cpu().numpy()),
                            _np(bias), None if r is None else _np(r), epilogue == "gelu")
    need = MS.ms_mx4_linear_workspace_bytes(a[0], w[0])
    for ws in (None, torch.empty(need + 16, dtype=torch.uint8, device=DEV)):
        MS.ms_mx4_linear(*a, *w, bias, out[:M], resid=r, gelu=epilogue == "gelu", workspace=ws)
        _within(_np(out[:M]), want, _product_bound(want, size, K, dtype, None if r is None else _np(r)), f"{M}x{N}x{K}")
        assert bool((out[M] == 7.0).all())
    if r is not None:       # onto the residual stream in place
        MS.ms_mx4_linear(*a, *w, bias, r, resid=r)
        assert torch.equal(r, out[:M]) or need


@pytest.mark.parametrize("M,N,K", [(5, 36, 96), (140, 260, 320), (1, 64, 4096)])
def test_nan_scales_stay_in_their_rows_and_columns(M, N, K):
    """Rows of A and W behind a NaN block, also in a last step that K does not fill: nothing leaks past a row's end."""
    g = torch.Generator().manual_seed(M)
    a, w = _operand(g, M, K), _operand(g, N, K)
    bias = torch.zeros(N, device=DEV)
    clean = torch.empty(M, N, device=DEV)
    MS.ms_mx4_linear(*a, *w, bias, clean)
    a[1][M - 1, 0] = 255
    w[1][1, K // 32 - 1] = 255
    w[1][N - 1, 0] = 255
    out = torch.empty(M, N, device=DEV)
    MS.ms_mx4_linear(*a, *w, bias, out)
    nan = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    nan[M - 1] = True
    nan[:, 1] = nan[:, N - 1] = True
    assert torch.equal(torch.isnan(out), nan) and torch.equal(out[~nan], clean[~nan])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K,shift", [(300, 264, 128, 0), (300, 264, 256, 0), (300, 264, 384, 0), (300, 264, 4096, 0), (270, 200, 4224, 0),
                                         (4100, 4100, 384, 0), (4097, 4004, 512, 0), (2000, 4100, 640, 0), (2049, 4036, 1024, 0),
                                         (1030, 2052, 2080, 0), (1900, 2052, 1056, 0), (600, 640, 12800, 0), (2000, 4100, 672, 0), (300, 264, 384, 1), (2000, 4100, 640, 2), (33, 68, 2048, 3)])
def test_product_of_every_tile_size(dtype, M, N, K, shift):
    """Sizes that take small and large tiles, whole and half steps, K ranges; scales that start at any byte."""
    g = torch.Generator().manual_seed(M + K)
    a, w = _operand(g, M, K), _operand(g, N, K, 1.0 / math.sqrt(K))
    bias, out = _randn(g, (N,), dtype), torch.empty(M + 1, N, dtype=DT[dtype], device=DEV)
    want, size = mx4.linear(mx4.values(a[0].cpu().numpy(), a[1].cpu().numpy()), mx4.values(w[0].cpu().numpy(), w[1].cpu().numpy()), _np(bias))
    bound = _product_bound(want, size, K, dtype)
    store = [torch.full((shift + t.numel() + 8,), 255, dtype=torch.uint8, device=DEV) for t in (a[1], w[1])]
    sa, sw = (m[shift:shift + t.numel()].view(t.shape) for m, t in zip(store, (a[1], w[1])))
    sa.copy_(a[1])
    sw.copy_(w[1])
    need = MS.ms_mx4_linear_workspace_bytes(a[0], w[0])
    for size in sorted({0, need // 2, need}):
        ws = torch.full((size + 16,), 0xff, dtype=torch.uint8, device=DEV) if size else None
        out.fill_(7.0)
        MS.ms_mx4_linear(a[0], sa, w[0], sw, bias, out[:M], workspace=ws)
        _within(_np(out[:M]), want, bound, f"{M}x{N}x{K} workspace {size}")
        assert bool((out[M] == 7.0).all())
    MS.ms_mx4_linear(a[0], sa, w[0], sw, bias, out[:M])
    sa[M - 1, 0] = sw[1, K // 32 - 1] = sw[N - 1, 0] = 255
    nan = torch.zeros(M, N, dtype=torch.bool, device=DEV)
    nan[M - 1] = True
    nan[:, 1] = nan[:, N - 1] = True
    got = torch.empty(M, N, dtype=DT[dtype], device=DEV)
    MS.ms_mx4_linear(a[0], sa, w[0], sw, bias, got)
    assert torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], out[:M][~nan])


def test_scales_of_every_size():
    """Scale bytes from 2 to 250 on both sides, products within float32."""
    g = torch.Generator().manual_seed(9)
    M, N, K = 20, 24, 640
    a, w = _operand(g, M, K), _operand(g, N, K)
    sa = torch.randint(2, 250, (M, 1), generator=g)
    a[1][:] = sa.to(torch.uint8).to(DEV)
    for n in range(N):      # 2^(a - 127) 2^(w - 127) near 1 for the row that it meets
        w[1][n] = int(254 - sa[n % M])
    out = torch.empty(M, N, device=DEV)
    MS.ms_mx4_linear(*a, *w, torch.zeros(N, device=DEV), out)
    want, size = mx4.linear(mx4.values(a[0].cpu().numpy(), a[1].cpu().numpy()), mx4.values(w[0].cpu().numpy(), w[1].cpu().numpy()), np.zeros(N))
    got, bound = _np(out), _product_bound(want, size, K, "fp32")
    near = size < 2.0 ** 100
    assert bool((np.abs(got - want)[near] <= bound[near]).all())
    for m in range(M):
        assert abs(got[m, m] - want[m, m]) <= bound[m, m]


# ------------------------------------------------------------------ norms, rotation, scatter

def _table(n_pos, rot, dtype=torch.float32):
    f = torch.exp(torch.arange(rot // 2, dtype=torch.float64) * (-2 * math.log(1e4) / rot))
    a = torch.arange(n_pos, dtype=torch.float64)[:, None] * 31.0 * f
    return torch.stack([a.cos(), a.sin()], 2).to(dtype).contiguous().to(DEV)


def _qk_case(g, dtype, M, H, G, hd, rot, extra, n_pos, kv_rows):
    wide = _randn(g, (M, (H + 2 * G) * hd + extra), dtype, 2.0)
    s = {"qkv": wide[:, :(H + 2 * G) * hd], "q": torch.full((M + 1, H, hd), 5.0, dtype=DT[dtype], device=DEV),
         "kv": _randn(g, (kv_rows, 2, G, hd), dtype), "q_gain": 1 + _randn(g, (hd,), dtype, 0.3), "k_gain": 1 + _randn(g, (hd,), dtype, 0.3),
         "table": _table(n_pos, rot) if rot else None, "pos": torch.randint(0, n_pos, (M,), generator=g).int().to(DEV),
         "rows": torch.randperm(kv_rows, generator=g)[:M].int().to(DEV)}
    return s


def _qk_check(s, dtype, H, G, hd, halves, eps=1e-6):
    M = s["qkv"].shape[0]
    before = s["kv"].clone()
    MS.ms_qk_norm_rope(s["qkv"], s["q"][:M], s["kv"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=eps, table=s["table"], pos=s["pos"],
                       halves=halves, rows=s["rows"])
    gain = [None if s[k] is None else _np(s[k]) for k in ("q_gain", "k_gain")]
    (q, qs), (k, ks), v = qk_norm_rope.qk_norm_rope(_np(s["qkv"]), H, G, hd, *gain, eps, None if s["table"] is None else _np(s["table"]),
                                                    None if s["pos"] is None else s["pos"].cpu().numpy(), halves)
    # float32: the sum of hd squares, root, quotient, two gains' products, the rotation's two products and sum
    e = (hd / 2 + 12) * 2.0 ** -24
    _within(_np(s["q"][:M]), q, e * qs + HALF[dtype] * (np.abs(q) + e * qs) + 1e-38, "q")
    assert bool((s["q"][M] == 5.0).all())
    rows = np.arange(M) if s["rows"] is None else s["rows"].cpu().numpy()
    there = (rows >= 0) & (rows < before.shape[0])
    _within(_np(s["kv"])[rows[there], 0], k[there], (e * ks + HALF[dtype] * (np.abs(k) + e * ks) + 1e-38)[there], "k")
    assert np.array_equal(_np(s["kv"])[rows[there], 1], v[there])
    left = np.ones(before.shape[0], bool)
    left[rows[there]] = False
    assert torch.equal(s["kv"][torch.from_numpy(left).to(DEV)], before[torch.from_numpy(left).to(DEV)])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("halves", [False, True], ids=["pairs", "halves"])
@pytest.mark.parametrize("M,H,G,hd,rot,extra", [(1, 1, 1, 8, 8, 0), (1, 24, 24, 128, 128, 0), (5, 4, 2, 64, 64, 8), (37, 16, 16, 72, 72, 0),
                                                (9, 8, 1, 128, 64, 72), (13, 3, 3, 40, 18, 0), (130, 6, 2, 104, 104, 0), (70, 5, 5, 24, 10, 16),
                                                (3, 33, 1, 96, 2, 0), (257, 12, 12, 64, 32, 0), (20, 7, 7, 120, 114, 0)])
def test_qk_norm_rope(dtype, halves, M, H, G, hd, rot, extra):
    g = torch.Generator().manual_seed(M + hd + rot)
    _qk_check(_qk_case(g, dtype, M, H, G, hd, rot, extra, 300, M + 50), dtype, H, G, hd, halves)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("without", ["q_gain", "k_gain", "gains", "table", "pos", "rows", "all"])
def test_qk_norm_rope_without(dtype, without):
    g = torch.Generator().manual_seed(12)
    s = _qk_case(g, dtype, 40, 6, 3, 80, 48, 0, 60, 45)
    for k in {"gains": ("q_gain", "k_gain"), "all": ("q_gain", "k_gain", "table", "pos", "rows")}.get(without, (without,)):
        s[k] = None
    _qk_check(s, dtype, 6, 3, 80, False)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_numbers_outside_their_tables(dtype):
    """Positions outside the table are not rotated, rows outside kv not written; a table without rows rotates nothing."""
    g = torch.Generator().manual_seed(13)
    s = _qk_case(g, dtype, 40, 6, 3, 64, 64, 0, 60, 45)
    s["pos"][:6] = torch.tensor([-1, 60, 59, 0, -(1 << 31), (1 << 31) - 1], dtype=torch.int32)
    s["rows"][3:7] = torch.tensor([-1, 45, -(1 << 31), (1 << 31) - 1], dtype=torch.int32)
    _qk_check(s, dtype, 6, 3, 64, True)
    s["table"] = torch.empty(0, 32, 2, device=DEV)
    _qk_check(s, dtype, 6, 3, 64, True)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_qk_specials_stay_in_their_heads(dtype):
    """Rows of zeros, a NaN and an infinity in one head of one row."""
    g = torch.Generator().manual_seed(14)
    M, H, G, hd = 9, 5, 2, 72
    s = _qk_case(g, dtype, M, H, G, hd, hd, 0, 60, 45)
    MS.ms_qk_norm_rope(s["qkv"], s["q"][:M], s["kv"], q_gain=s["q_gain"], k_gain=s["k_gain"], table=s["table"], pos=s["pos"], rows=s["rows"])
    q, kv = s["q"].clone(), s["kv"].clone()
    s["qkv"][2, 3 * hd + 5], s["qkv"][4, (H + 1) * hd] = math.nan, math.inf
    s["qkv"][6] = 0.0
    MS.ms_qk_norm_rope(s["qkv"], s["q"][:M], s["kv"], q_gain=s["q_gain"], k_gain=s["k_gain"], table=s["table"], pos=s["pos"], rows=s["rows"])
    assert bool(torch.isnan(s["q"][2, 3]).all()) and bool(torch.isnan(s["kv"][s["rows"][4].long(), 0, 1]).any())
    assert bool((s["q"][6] == 0).all()) and bool((s["kv"][s["rows"][6].long()] == 0).all())
    same = torch.ones(M, H, dtype=torch.bool, device=DEV)
    same[2, 3] = same[6] = False
    assert torch.equal(s["q"][:M][same], q[:M][same])


# ------------------------------------------------------------------ attention over a shared prefix

def _batch(g, dtype, rows, T, G, hd, group, own=None, hide=0.2, lead=0, tail=0):
    """rows: packed rows of each request; own: own rows of each (None: as many); lead, tail: packed rows of no request."""
    B, own = len(rows), rows if own is None else own
    M = lead + sum(rows) + tail
    s = {"q": _randn(g, (M, G * group, hd), dtype, 1.5), "kv": _randn(g, (T, 2, G, hd), dtype),
         "out": torch.full((M, G * group, hd), 7.0, dtype=DT[dtype], device=DEV),
         "seg": [lead + sum(rows[:b]) for b in range(B + 1)], "own": [sum(own[:b]) for b in range(B + 1)],
         "hidden": torch.rand(B, T, generator=g) < hide if hide else None, "fresh": _randn(g, (sum(own), 2, G, hd), dtype) if sum(own) else None}
    return s


def _bits(hidden):
    bits = torch.empty(hidden.shape[0], -(-hidden.shape[1] // 64), dtype=torch.int64, device=DEV)
    MS.ms_shared_bits(hidden.to(DEV), bits)
    return bits


def _int(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _attend(s, ws="need", scale=None, out=None):
    need = MS.ms_shared_attention_workspace_bytes(s["q"], s["kv"], fresh=s["fresh"])
    size = {"need": need, None: 0, "some": need // 2}[ws]
    workspace = torch.full((size + 16,), 0xff, dtype=torch.uint8, device=DEV) if size else None
    MS.ms_shared_attention(s["q"], s["kv"], s["out"] if out is None else out, seg_start=_int(s["seg"]),
                           bits=None if s["hidden"] is None or s["kv"].shape[0] == 0 else _bits(s["hidden"]), fresh=s["fresh"],
                           fresh_start=None if s["fresh"] is None else _int(s["own"]), scale=scale, workspace=workspace)
    return s["out"] if out is None else out


def _attend_bound(want, spread, size, reach, keys, hd, dtype):
    """Weights: scores in float32 (hd products summed, the running maximum taken off, the scale), the exponential to 2^-22 and
    in bf16 the operand's rounding; numerator and denominator in float32 over `keys` terms; one rounding of the result."""
    e = ((2 * hd + 8) * 2.0 ** -24 * reach + 2.0 ** -22 + (2.0 ** -8 if dtype == "bf16" else 0.0)) * 1.02
    e = e * spread + 2 * (keys + 64) * 2.0 ** -24 * size
    return e + HALF[dtype] * (np.abs(want) + e) + 1e-30


def _check(s, dtype, *each, scale=None):
    """The call with each of these workspaces against the oracle."""
    hd = s["q"].shape[2]
    want, spread, size, reach = shared.attention(_np(s["q"]), _np(s["kv"]), None if s["hidden"] is None else s["hidden"].numpy(), s["seg"],
                                                 None if s["fresh"] is None else _np(s["fresh"]), s["own"],
                                                 1 / math.sqrt(hd) if scale is None else scale)
    lo, hi = s["seg"][0], s["seg"][-1]
    keys = s["kv"].shape[0] + (0 if s["fresh"] is None else s["fresh"].shape[0])
    bound = _attend_bound(want, spread, size, reach, keys, hd, dtype)[lo:hi]
    for ws in each or ("need",):
        s["out"].fill_(7.0)
        got = _attend(s, ws, scale)
        _within(_np(got[lo:hi]), want[lo:hi], bound, f"T={s['kv'].shape[0]} hd={hd} ws={ws}")
        assert bool((got[:lo] == 7.0).all()) and bool((got[hi:] == 7.0).all())


@pytest.mark.parametrize("T", [1, 63, 64, 65, 1000])
def test_bits(T):
    g = torch.Generator().manual_seed(T)
    hidden = torch.rand(5, T, generator=g) < 0.4
    bits = _bits(hidden).cpu()
    for b in range(5):
        for t in range(64 * bits.shape[1]):
            assert bool((int(bits[b, t // 64]) >> (t % 64)) & 1) == (bool(hidden[b, t]) if t < T else True)


@pytest.mark.parametrize("dtype,hd", [("bf16", h) for h in range(8, 129, 8)] + [("fp32", h) for h in range(8, 65, 8)])
@pytest.mark.parametrize("rows", [(3,), (9, 0, 14), (60, 1, 90, 7)], ids=["3", "23", "158"])
def test_attention_at_every_head_dim(dtype, hd, rows):
    g = torch.Generator().manual_seed(hd + len(rows))
    s = _batch(g, dtype, rows, 331, 2, hd, 1, lead=2, tail=3)
    _check(s, dtype, None, "need")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [(1,), (16,), (1,) * 16, (17,), (32,), (5, 28), (129,), (1,) * 128, (40, 200, 3, 90)], ids=lambda r: f"{len(r)}x{r[0]}")
@pytest.mark.parametrize("T", [0, 1, 31, 64, 65, 127, 700])
def test_attention_lengths(dtype, rows, T):
    g = torch.Generator().manual_seed(T + sum(rows))
    s = _batch(g, dtype, rows, T, 3, 64, 1)
    _check(s, dtype, None, "need", "some")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("own", ["none", "more", "fewer"])
@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("hide", [0.0, 0.5, 1.0])
def test_attention_heads_own_rows_and_hidden_tokens(dtype, own, group, hide):
    """Own rows of their own number (none at all, or some of a request without query rows), every token hidden."""
    g = torch.Generator().manual_seed(group + int(10 * hide))
    rows = (6, 30, 0, 1, 17)
    n = {"none": (0,) * 5, "more": (70, 0, 33, 5, 129), "fewer": (0, 2, 1, 0, 3)}[own]
    s = _batch(g, dtype, rows, 260, 2, 40, group, own=n, hide=hide)
    _check(s, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [2, 30, 150])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 3e38])
def test_what_a_row_does_not_see_has_no_effect(dtype, rows, value):
    """Hidden tokens and other requests' own rows of NaN, infinities and the largest values."""
    g = torch.Generator().manual_seed(rows)
    s = _batch(g, dtype, (rows, rows + 3, rows), 200, 2, 72 if dtype == "bf16" else 64, 1, hide=0.3)
    s["hidden"][1] = s["hidden"][0]
    s["hidden"][:2, 64:128] = True
    for ws in (None, "need"):
        want = _attend(s, ws).clone()
        bad = {k: v.clone() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
        bad["kv"][s["hidden"][0].to(DEV) & s["hidden"][2].to(DEV)] = value
        only = s["hidden"][0].to(DEV) & ~s["hidden"][2].to(DEV)       # the third request sees these
        bad["kv"][only] = value
        bad["fresh"][s["own"][2]:] = value
        got = _attend(bad, ws)
        seen = slice(0, s["seg"][2])
        w, p = _np(want[seen]), _np(got[seen])
        # recomputed slots sum in another order and keep their weights in float32
        assert np.isfinite(p).all() and np.abs(p - w).max() <= (2.0 ** -6 if dtype == "bf16" else 1e-5) * np.abs(w).max()
        _check_rows(bad, dtype, got, seen)
        if value != value:
            assert bool(torch.isnan(got[s["seg"][2]:]).all())


def _check_rows(s, dtype, got, rows):
    clean = {k: s[k] for k in s}
    kv, fresh = _np(s["kv"]), _np(s["fresh"])
    kv[~np.isfinite(kv) | (np.abs(kv) > 1e38)] = 0.0
    fresh[~np.isfinite(fresh) | (np.abs(fresh) > 1e38)] = 0.0
    hd = s["q"].shape[2]
    want, spread, size, reach = shared.attention(_np(s["q"]), kv, s["hidden"].numpy(), s["seg"], fresh, s["own"], 1 / math.sqrt(hd))
    bound = _attend_bound(want, spread, size, reach, len(kv) + len(fresh), hd, dtype)
    _within(_np(got)[rows], want[rows], bound[rows], "rows that do not see it")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 25, 200])
@pytest.mark.parametrize("ws", [None, "need"])
def test_scores_of_infinity(dtype, rows, ws):
    """Scores of -infinity weigh nothing, alone they give zeros; one of +infinity, or a NaN in a query, makes its row NaN."""
    g = torch.Generator().manual_seed(rows)
    s = _batch(g, dtype, (rows,), 1500, 1, 32, 1, own=(10,), hide=0.0)
    s["q"][:, 0, 0] = 1.0
    s["kv"][700:, 0, 0, 0] = -math.inf
    s["fresh"][:, 0, 0, 0] = -math.inf
    want = {k: v for k, v in s.items()}
    want["kv"], want["fresh"] = s["kv"][:700].contiguous(), None
    ref, spread, size, reach = shared.attention(_np(s["q"]), _np(want["kv"]), None, s["seg"], None, None, 1 / math.sqrt(32))
    _within(_np(_attend(s, ws)), ref, _attend_bound(ref, spread, size, reach, 1510, 32, dtype), "-inf")
    s["kv"][:, 0, 0, 0] = -math.inf
    assert bool((_attend(s, ws) == 0).all())
    s["q"][rows - 1, 0, 0] = -1.0
    s["q"][0, 0, 3] = math.nan
    got = _attend(s, ws)
    assert bool(torch.isnan(got[rows - 1]).all()) and bool(torch.isnan(got[0]).all())
    assert rows < 3 or bool((got[1:rows - 1] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("scale", [-0.3, 2.0, 1e-6, 1e-44])
def test_attention_scales(dtype, scale):
    g = torch.Generator().manual_seed(3)
    _check(_batch(g, dtype, (20, 5), 300, 2, 64, 2), dtype, scale=scale)
    _check(_batch(g, dtype, (150, 5), 300, 2, 64, 2), dtype, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [(4,), (20, 9), (70, 90)])
def test_output_over_the_queries(dtype, rows):
    g = torch.Generator().manual_seed(sum(rows))
    s = _batch(g, dtype, rows, 500, 2, 64, 1)
    for ws in (None, "need"):
        want = _attend(s, ws).clone()
        q = s["q"].clone()
        t = dict(s, q=q)
        assert torch.equal(_attend(t, ws, out=q), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [(4,), (20, 9), (30, 70), (70, 90)])
def test_output_over_the_queries_with_hidden_nan(dtype, rows):
    """Results that are computed again read queries that the output has not replaced."""
    g = torch.Generator().manual_seed(sum(rows))
    s = _batch(g, dtype, rows, 500, 2, 64, 1)
    s["hidden"][:, 40:44] = True
    s["kv"][40:44] = math.nan
    for ws in (None, "need"):
        want = _attend(s, ws).clone()
        _check_rows(s, dtype, want, slice(0, sum(rows)))
        t = dict(s, q=s["q"].clone())
        assert torch.equal(_attend(t, ws, out=t["q"]), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tables_out_of_range_are_bounded(dtype):
    """Starts that do not ascend or lie outside the rows: every access stays within the buffers, rows of no request stay."""
    g = torch.Generator().manual_seed(2)
    s = _batch(g, dtype, (30, 40, 30), 300, 2, 64, 1)
    for seg, own in [([0, 70, 30, 100], s["own"]), ([-5, 10, 1 << 30, 200], [-7, 40, 1 << 30, 500]), (s["seg"], [90, 20, 70, 0]),
                     ([50, 50, 50, 50], s["own"]), ([100, 60, 20, 0], s["own"])]:
        s["out"].fill_(7.0)
        got = _attend(dict(s, seg=seg, own=own))
        lo, hi = min(max(seg[0], 0), 100), min(max(seg[-1], 0), 100)
        assert bool(torch.isfinite(got).all())
        assert bool((got[:lo] == 7.0).all()) and (hi < lo or bool((got[hi:] == 7.0).all()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_large_scores_and_far_maxima(dtype):
    """A first tile of scores near the lowest values, later ones far above them, and growing ones."""
    g = torch.Generator().manual_seed(6)
    s = _batch(g, dtype, (40,), 512, 1, 64, 1, own=(0,), hide=0.0)
    s["q"][:] = 0.0
    s["q"][:, 0, 0] = 1.0
    step = torch.arange(512, device=DEV).float()
    for height in (-1e30 * (step < 100), 40.0 * step, -40.0 * step, 1e4 * (step == 300)):
        s["kv"][:, 0, 0, 0] = height.to(DT[dtype])
        z = _np(s["kv"])[:, 0, 0, 0] / 8.0
        w = np.exp(z - z.max())
        want = (w[:, None] * _np(s["kv"])[:, 1, 0]).sum(0) / w.sum()
        got = _np(_attend(s, None))[:, 0]
        # a score's own float32 digits beside a maximum of this size
        e = 2.0 ** -8 + 2.0 ** -22 * np.abs(z[w > 1e-9]).max() + 2.0 ** -10 * (dtype == "bf16")
        assert np.abs(got - want).max() <= e * 8.0


# ------------------------------------------------------------------ together

def _run_block(s, stream=None):
    """The first half of a block: rows -> 4 bits -> Q, K, V -> norms, rotation, own K/V -> attention over the template -> 4 bits ->
    output projection onto the rows."""
    kw = {"stream": stream}
    MS.ms_mx4_quantize(s["x"], *s["xq"], **kw)
    MS.ms_mx4_linear(*s["xq"], *s["w_qkv"], s["b_qkv"], s["qkv"], workspace=s["ws"], **kw)
    MS.ms_qk_norm_rope(s["qkv"], s["q"], s["fresh"], q_gain=s["q_gain"], k_gain=s["k_gain"], table=s["table"], pos=s["pos"], **kw)
    MS.ms_shared_attention(s["q"], s["kv"], s["o"], seg_start=s["seg"], bits=s["bits"], fresh=s["fresh"], fresh_start=s["seg"],
                           workspace=s["ws"], **kw)
    MS.ms_mx4_quantize(s["o"].view(s["x"].shape), *s["oq"], **kw)
    MS.ms_mx4_linear(*s["oq"], *s["w_o"], s["b_o"], s["y"], resid=s["x"], workspace=s["ws"], **kw)


def _block(dtype, seed=1, rows=(9, 40, 1), T=200, H=4, hd=32):
    g = torch.Generator().manual_seed(seed)
    d, M = H * hd, sum(rows)
    seg = [sum(rows[:b]) for b in range(len(rows) + 1)]
    hidden = torch.zeros(len(rows), T, dtype=torch.bool)
    pos = []
    for b, n in enumerate(rows):
        at = torch.randperm(T, generator=g)[:n].sort().values
        hidden[b, at] = True
        pos += at.tolist()
    s = {"x": _randn(g, (M, d), dtype), "xq": _empty_codes(M, d), "w_qkv": _operand(g, 3 * d, d, d ** -0.5), "b_qkv": _randn(g, (3 * d,), dtype),
         "qkv": torch.empty(M, 3 * d, dtype=DT[dtype], device=DEV), "q": torch.empty(M, H, hd, dtype=DT[dtype], device=DEV),
         "fresh": torch.empty(M, 2, H, hd, dtype=DT[dtype], device=DEV), "q_gain": 1 + _randn(g, (hd,), dtype, 0.2),
         "k_gain": 1 + _randn(g, (hd,), dtype, 0.2), "table": _table(T, hd), "pos": _int(pos), "kv": _randn(g, (T, 2, H, hd), dtype),
         "o": torch.empty(M, H, hd, dtype=DT[dtype], device=DEV), "seg": _int(seg), "segs": seg, "hidden": hidden, "bits": _bits(hidden),
         "oq": _empty_codes(M, d), "w_o": _operand(g, d, d, d ** -0.5), "b_o": _randn(g, (d,), dtype),
         "y": torch.empty(M, d, dtype=DT[dtype], device=DEV)}
    s["ws"] = torch.empty(max(16, MS.ms_shared_attention_workspace_bytes(s["q"], s["kv"], fresh=s["fresh"]),
                              MS.ms_mx4_linear_workspace_bytes(s["xq"][0], s["w_qkv"][0]),
                              MS.ms_mx4_linear_workspace_bytes(s["oq"][0], s["w_o"][0])), dtype=torch.uint8, device=DEV)
    return s


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_a_run_of_them_together(dtype):
    """Each operator against the oracle of what the one before it left on the GPU."""
    H, hd = 4, 32
    s = _block(dtype)
    _run_block(s)
    vals = lambda t: mx4.values(t[0].cpu().numpy(), t[1].cpu().numpy())
    c, e = mx4.quantize(_np(s["x"]))
    assert _same_codes(s["xq"][0], c) and _same_codes(s["xq"][1], e)
    want, size = mx4.linear(vals(s["xq"]), vals(s["w_qkv"]), _np(s["b_qkv"]))
    _within(_np(s["qkv"]), want, _product_bound(want, size, H * hd, dtype), "qkv")
    (q, qs), (k, ks), v = qk_norm_rope.qk_norm_rope(_np(s["qkv"]), H, H, hd, _np(s["q_gain"]), _np(s["k_gain"]), 1e-6, _np(s["table"]),
                                                    s["pos"].cpu().numpy(), False)
    f = 28 * 2.0 ** -24
    _within(_np(s["q"]), q, f * qs + HALF[dtype] * (np.abs(q) + f * qs), "q")
    _within(_np(s["fresh"][:, 0]), k, f * ks + HALF[dtype] * (np.abs(k) + f * ks), "k")
    want, spread, size, reach = shared.attention(_np(s["q"]), _np(s["kv"]), s["hidden"].numpy(), s["segs"], _np(s["fresh"]), s["segs"], hd ** -0.5)
    _within(_np(s["o"]), want, _attend_bound(want, spread, size, reach, 250, hd, dtype), "o")
    want, size = mx4.linear(vals(s["oq"]), vals(s["w_o"]), _np(s["b_o"]), _np(s["x"]))
    _within(_np(s["y"]), want, _product_bound(want, size, H * hd, dtype, _np(s["x"])), "y")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_the_run_captured_and_on_another_stream(dtype):
    """A captured run replayed over new inputs, with eager runs and synchronizations between: bit for bit what an eager run gives."""
    s = _block(dtype)
    _run_block(s)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        _run_block(s)
    for seed in range(2, 6):
        t = _block(dtype, seed)
        s["x"].copy_(t["x"])
        s["kv"].copy_(t["kv"])
        _run_block(s)
        torch.cuda.synchronize()
        want = {k: s[k].clone() for k in ("qkv", "q", "fresh", "o", "y")}
        for k in want:
            s[k].fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(s[k], want[k]) for k in want)
        with torch.cuda.stream(side):
            for k in want:
                s[k].fill_(3.0)
            _run_block(s)
        torch.cuda.synchronize()
        assert all(torch.equal(s[k], want[k]) for k in want)
        other = torch.cuda.Stream()
        other.wait_stream(torch.cuda.current_stream())
        _run_block(s, stream=other)
        torch.cuda.synchronize()
        assert all(torch.equal(s[k], want[k]) for k in want)


def test_runs_are_repeatable():
    """Two calls give the same bits."""
    for dtype in ("bf16", "fp32"):
        s = _block(dtype, rows=(70, 5, 130), T=900)
        _run_block(s)
        first = {k: s[k].clone() for k in ("qkv", "q", "fresh", "o", "y")}
        for _ in range(3):
            s["ws"].fill_(0xff)
            _run_block(s)
            assert all(torch.equal(s[k], first[k]) for k in first)


def test_nothing_to_do():
    """No rows and no tokens are no errors."""
    e = lambda *shape, dt=torch.bfloat16: torch.empty(*shape, dtype=dt, device=DEV)
    u8 = torch.uint8
    MS.ms_mx4_quantize(e(0, 64), e(0, 32, dt=u8), e(0, 2, dt=u8))
    MS.ms_mx4_dequantize(e(0, 32, dt=u8), e(0, 2, dt=u8), e(0, 64))
    MS.ms_mx4_linear(e(0, 32, dt=u8), e(0, 2, dt=u8), e(8, 32, dt=u8), e(8, 2, dt=u8), e(8), e(0, 8))
    MS.ms_qk_norm_rope(e(0, 48), e(0, 4, 8), e(5, 2, 1, 8))
    MS.ms_shared_attention(e(0, 4, 8), e(9, 2, 4, 8), e(0, 4, 8))
    q, out = torch.ones(3, 4, 8, device=DEV), torch.full((3, 4, 8), 7.0, device=DEV)
    MS.ms_shared_attention(q, torch.empty(0, 2, 4, 8, device=DEV), out)
    assert bool((out == 0).all())

"""The 8-bit K/V cache on the GPU against the float64 oracle: writing, rewriting and reading back are exact (codes,
scales and values), attention is held to bounds derived from the roundings it makes (_bound)."""
import math

import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2505_20600_amd import maskstep as MS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}


def _np(t):
    return t.detach().to(torch.float64).cpu().numpy()


def _rows(g, shape, dtype, width=1.0):
    """K/V rows whose (K or V, head) blocks have magnitudes e^(+-2) apart."""
    x = torch.randn(*shape, generator=g) * torch.exp(torch.randn(*shape[-3:-1], 1, generator=g)) * width
    return x.to(DT[dtype]).to(DEV)


def _empty_cache(S, T, H, hd, block, fill=0x55):
    return (torch.full((S, T, 2, H, hd), fill, dtype=torch.uint8, device=DEV),
            torch.full((S, -(-T // block), 2, H), fill, dtype=torch.uint8, device=DEV))


def _oracle_cache(kv, block):
    both = [kv8.quantize(_np(kv[s]), block) for s in range(kv.shape[0])]
    return np.stack([c for c, _ in both]), np.stack([e for _, e in both])


def _cache(g, S, T, H, hd, block, dtype):
    """(codes, scales) on the GPU of random rows, by the oracle."""
    c, e = _oracle_cache(_rows(g, (S, T, 2, H, hd), dtype), block)
    return torch.from_numpy(c).to(DEV), torch.from_numpy(e).to(DEV)


def _same_codes(got, want):
    """Equal codes, any NaN code for NaN; the sign of zero counts."""
    nan = (want & 0x7f) == 0x7f
    return bool(np.array_equal((got & 0x7f) == 0x7f, nan) and np.array_equal(got[~nan], want[~nan]))


# ------------------------------------------------------------------ writing

@pytest.mark.parametrize("dtype,S,T,H,hd,block", [
    ("bf16", 1, 1, 1, 8, 1), ("bf16", 2, 37, 3, 8, 16), ("bf16", 1, 130, 2, 128, 128), ("bf16", 3, 65, 5, 72, 64),
    ("bf16", 1, 64, 16, 64, 64), ("bf16", 2, 33, 2, 40, 1), ("bf16", 1, 300, 1, 104, 32), ("bf16", 1, 50, 4, 120, 2),
    ("bf16", 1, 257, 2, 128, 4), ("fp32", 1, 1, 1, 8, 64), ("fp32", 2, 100, 3, 64, 128), ("fp32", 1, 77, 4, 32, 8),
    ("fp32", 1, 129, 2, 56, 64), ("fp32", 1, 40, 3, 48, 1)])
def test_quantize_is_exact(dtype, S, T, H, hd, block):
    g = torch.Generator().manual_seed(T + hd)
    kv = _rows(g, (S, T, 2, H, hd), dtype)
    codes, scales = _empty_cache(S + 1, T, H, hd, block)
    MS.ms_kv8_quantize(kv, codes[:S], scales[:S], block=block)
    c, e = _oracle_cache(kv, block)
    assert np.array_equal(scales[:S].cpu().numpy(), e)
    assert _same_codes(codes[:S].cpu().numpy(), c)
    assert bool((codes[S] == 0x55).all()) and bool((scales[S] == 0x55).all())     # nothing past the last cache


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_quantize_of_special_values(dtype):
    """Zeros of both signs, NaN and infinities, the type's largest and smallest values, ties between codes, blocks of
    zeros and of no finite value."""
    big, tiny = torch.finfo(DT[dtype]).max, torch.finfo(DT[dtype]).tiny
    g = torch.Generator().manual_seed(5)
    kv = torch.randn(1, 8 * 12, 2, 1, 16, generator=g)
    v = kv.view(12, 8, 2, 1, 16)
    v[0] = 0.0
    v[0, ::2] = -0.0
    v[1, 3, 0, 0, 2], v[1, 4, 0, 0, 3], v[1, 5, 1, 0, 1] = math.nan, math.inf, -math.inf
    v[2] = math.nan
    v[3, 0] = -math.inf
    v[4] *= big / 8
    v[4, 1, 0, 0, 0] = -big
    v[5] = tiny * torch.randn(8, 2, 1, 16, generator=g)
    v[6] = tiny * 2.0 ** -6 * torch.randint(-8, 9, (8, 2, 1, 16), generator=g)           # subnormal
    v[7] = torch.randint(-40, 41, (8, 2, 1, 16), generator=g).float()                    # ties: 17 between 16 and 18
    v[7, 0, :, 0, 0] = 448.0
    v[8] = torch.randn(8, 2, 1, 16, generator=g) * 2.0 ** -12                            # below the smallest normal code
    v[8, 0, :, 0, 0] = 448.0
    v[9], v[9, 0, :, 0, 0] = 1.0, 1.75
    v[10], v[10, 0, :, 0, 0] = 1.0, 1.765625
    v[11] *= 2.0 ** -120
    kv = kv.to(DT[dtype]).to(DEV)
    codes, scales = _empty_cache(1, 96, 1, 16, 8)
    MS.ms_kv8_quantize(kv, codes, scales, block=8)
    c, e = _oracle_cache(kv, 8)
    assert np.array_equal(scales.cpu().numpy(), e)
    assert _same_codes(codes.cpu().numpy(), c)


def test_quantize_rows_of_a_working_buffer():
    """Image rows behind text rows, requests further apart than the cache's tokens."""
    g = torch.Generator().manual_seed(6)
    full = _rows(g, (3, 100, 2, 2, 64), "bf16")
    img = full[:, 20:90]
    codes, scales = _empty_cache(3, 70, 2, 64, 32)
    MS.ms_kv8_quantize(img, codes, scales, block=32)
    c, e = _oracle_cache(img, 32)
    assert np.array_equal(scales.cpu().numpy(), e) and _same_codes(codes.cpu().numpy(), c)
    wide = _rows(g, (2, 80, 2, 2, 64), "bf16")          # only the first 70 rows of each are the caches' tokens
    MS.ms_kv8_quantize(wide, codes[:2], scales[:2], block=32)
    c, e = _oracle_cache(wide[:, :70], 32)
    assert np.array_equal(scales[:2].cpu().numpy(), e) and _same_codes(codes[:2].cpu().numpy(), c)


@pytest.mark.parametrize("dtype,S,T,H,hd,block", [("bf16", 2, 150, 3, 64, 64), ("bf16", 1, 70, 2, 72, 16), ("bf16", 1, 33, 1, 8, 1),
                                                  ("bf16", 1, 260, 2, 128, 128), ("fp32", 2, 100, 2, 40, 32), ("fp32", 1, 5, 1, 64, 4)])
@pytest.mark.parametrize("share", [0.0, 0.1, 1.0])
def test_rewrite_is_exact(dtype, S, T, H, hd, block, share):
    """New rows 30 times larger or smaller than the kept ones; blocks without a new row untouched; a row used twice;
    numbers outside kv keep the token; a second pass with the same rows changes nothing."""
    g = torch.Generator().manual_seed(T + hd + int(10 * share))
    codes, scales = _cache(g, S, T, H, hd, block, dtype)
    n = max(2, int(S * T * share))
    kv = _rows(g, (n, 2, H, hd), dtype, width=30.0 if T % 4 else 1 / 30)
    src = torch.full((S, T), -1, dtype=torch.int32)
    hit = torch.randperm(S * T, generator=g)[:int(S * T * share)]
    src.view(-1)[hit] = torch.arange(hit.numel(), dtype=torch.int32) % n
    if share == 0.1 and hit.numel():
        src.view(-1)[hit[0]] = 1
        src[0, T // 2] = n
        src[0, T // 3] = -(1 << 31)
    want = [kv8.rewrite(codes[s].cpu().numpy(), scales[s].cpu().numpy(), block, _np(kv), src[s].numpy()) for s in range(S)]
    for _ in range(2):
        MS.ms_kv8_quantize(kv, codes, scales, block=block, src_row=src.to(DEV))
        assert np.array_equal(scales.cpu().numpy(), np.stack([e for _, e in want]))
        assert _same_codes(codes.cpu().numpy(), np.stack([c for c, _ in want]))


def test_rewrite_keeps_values_of_the_smallest_scales():
    """Kept values between 2^-135 and 2^-118, below what bf16 holds as a normal number."""
    g = torch.Generator().manual_seed(11)
    codes = torch.randint(0, 127, (1, 64, 2, 1, 16), generator=g, dtype=torch.uint8).to(DEV)
    scales = torch.ones(1, 1, 2, 1, dtype=torch.uint8, device=DEV)
    kv = torch.zeros(1, 2, 1, 16, dtype=torch.bfloat16, device=DEV)
    src = torch.full((1, 64), -1, dtype=torch.int32, device=DEV)
    src[0, 5] = 0
    c, e = kv8.rewrite(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 64, _np(kv), src[0].cpu().numpy())
    MS.ms_kv8_quantize(kv, codes, scales, block=64, src_row=src)
    assert np.array_equal(scales[0].cpu().numpy(), e) and _same_codes(codes[0].cpu().numpy(), c)


# ------------------------------------------------------------------ reading

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_dequantize_every_code_and_scale(dtype):
    """All 256 codes at every exponent byte. bf16: values are the oracle's rounded to bf16 (only those below 2^-126 or
    beyond the largest need it); values below 2^-126 may come out as zero."""
    codes = torch.arange(256, dtype=torch.uint8, device=DEV).view(1, 1, 1, 1, 256)
    codes = codes.view(1, 1, 1, 4, 64).expand(1, 256, 2, 4, 64).contiguous()
    scales = torch.arange(256, dtype=torch.uint8, device=DEV).view(1, 256, 1, 1).expand(1, 256, 2, 4).contiguous()
    kv = torch.zeros(1, 256, 2, 4, 64, dtype=DT[dtype], device=DEV)
    MS.ms_kv8_dequantize(codes, scales, kv, block=1)
    want = torch.from_numpy(kv8.values(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 1)).to(DT[dtype]).double().numpy()
    got = _np(kv[0])
    small = np.abs(want) < 2.0 ** -126
    assert np.array_equal(got[~small], want[~small], equal_nan=True)
    assert np.all((got[small] == want[small]) | (got[small] == 0))


@pytest.mark.parametrize("dtype,S,T,H,hd,block", [("bf16", 3, 130, 2, 64, 64), ("bf16", 2, 65, 3, 72, 16), ("bf16", 1, 1, 1, 8, 1),
                                                  ("bf16", 2, 300, 2, 128, 128), ("fp32", 2, 90, 3, 40, 32), ("fp32", 1, 64, 4, 64, 64)])
def test_dequantize_listed_tokens(dtype, S, T, H, hd, block):
    """Lists in any order, a token twice, numbers outside the cache, requests sharing a cache, an empty list, a cache
    number outside: the listed rows are exact and no other row changes."""
    g = torch.Generator().manual_seed(T)
    codes, scales = _cache(g, S, T, H, hd, block, dtype)
    B = 5
    of = torch.tensor([S - 1, 0, S - 1, S, -1], dtype=torch.int32)
    counts = torch.tensor([min(T, T // 2 + 1), 0, T, T, T], dtype=torch.int32)
    keys = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]).int()
    if T > 4:
        keys[2, 1], keys[2, 2], keys[2, 3] = keys[2, 0], T, -5
    kv = _rows(g, (B, T + 3, 2, H, hd), dtype)
    want = _np(kv)
    for b in range(3):
        vals = kv8.values(codes[int(of[b])].cpu().numpy(), scales[int(of[b])].cpu().numpy(), block)
        for t in keys[b, :int(counts[b])].tolist():
            if 0 <= t < T:
                want[b, t] = vals[t]
    MS.ms_kv8_dequantize(codes, scales, kv, block=block, cache_of=of.to(DEV), keys=keys.to(DEV), n_keys=counts.to(DEV))
    assert np.array_equal(_np(kv), want)
    # no tables: every token of cache b
    kv2 = torch.full((S, T, 2, H, hd), 7.0, dtype=DT[dtype], device=DEV)
    MS.ms_kv8_dequantize(codes, scales, kv2, block=block)
    assert np.array_equal(_np(kv2), np.stack([kv8.values(codes[s].cpu().numpy(), scales[s].cpu().numpy(), block) for s in range(S)]))
    # counts without lists: the first tokens; counts beyond the list and below zero are limited
    kv3 = torch.full((S, T, 2, H, hd), 7.0, dtype=DT[dtype], device=DEV)
    n = torch.tensor([T // 2, T + 100, -3][:S], dtype=torch.int32, device=DEV)
    MS.ms_kv8_dequantize(codes, scales, kv3, block=block, n_keys=n)
    for s in range(S):
        m = min(max(int(n[s]), 0), T)
        assert torch.equal(kv3[s, :m], kv2[s, :m]) and bool((kv3[s, m:] == 7.0).all())


@pytest.mark.parametrize("B,T", [(1, 1), (3, 64), (2, 1023), (2, 1025), (1, 70001), (128, 5)])
def test_keys_are_the_unmasked_tokens(B, T):
    g = torch.Generator().manual_seed(T)
    mask = (torch.rand(B, T, generator=g) < torch.linspace(0, 1, B)[:, None]).to(torch.uint8) * 3
    keys = torch.full((B, T + 2), -7, dtype=torch.int32, device=DEV)
    n = torch.full((B,), -7, dtype=torch.int32, device=DEV)
    MS.ms_kv8_keys(mask.to(DEV), keys, n)
    for b in range(B):
        want = (mask[b] == 0).nonzero().flatten().int()
        assert int(n[b]) == want.numel()
        assert torch.equal(keys[b, :want.numel()].cpu(), want) and bool((keys[b, want.numel():] == -7).all())


def test_offsets_past_32_bits():
    """A pool whose last cache starts beyond 4 GiB of codes: written, read back, attended over."""
    S, T, H, hd, block = 10, 1 << 19, 4, 128, 128
    codes = torch.zeros(S, T, 2, H, hd, dtype=torch.uint8, device=DEV)          # half a GiB per cache
    scales = torch.full((S, T // block, 2, H), 127, dtype=torch.uint8, device=DEV)
    assert codes[:S - 1].numel() > 2 ** 32
    g = torch.Generator(device=DEV).manual_seed(1)
    kv = torch.randn(1, T, 2, H, hd, device=DEV, generator=g, dtype=torch.bfloat16)
    MS.ms_kv8_quantize(kv, codes[S - 1:], scales[S - 1:], block=block)
    back = torch.zeros(1, T, 2, H, hd, dtype=torch.bfloat16, device=DEV)
    of = torch.tensor([S - 1], dtype=torch.int32, device=DEV)
    MS.ms_kv8_dequantize(codes, scales, back, block=block, cache_of=of)
    err = (back.float() - kv.float()).abs()
    assert bool((err <= 2.0 ** -4 * kv.float().abs() + 2.0 ** -10 * 2.0 ** -5).all())
    tail = torch.tensor([[T - 1, T - 64, T - 200]], dtype=torch.int32, device=DEV)
    q = torch.randn(2, H, hd, device=DEV, generator=g, dtype=torch.bfloat16)
    out = torch.zeros_like(q)
    MS.ms_kv8_attention(q, codes, scales, out, torch.tensor([0, 2], dtype=torch.int32, device=DEV), block=block, cache_of=of,
                        keys=tail)
    k = _np(back[0][tail[0].long()])
    ref, spread = kv8.attention(_np(q), k[:, 0], k[:, 1], hd ** -0.5)
    assert np.all(np.abs(_np(out) - ref) <= _bound(q, k, ref, spread, hd ** -0.5, "bf16"))


# ------------------------------------------------------------------ attention

def _bound(q, kv, ref, spread, scale, dtype):
    """Element-wise bound on |out - ref| for n keys.

    float32: a score is hd products and sums in float32 and one multiplication into the log2 domain, off by at most
    (hd + 4) 2^-24 times sum |q k| |scale| (a magnitude: the sign of the scale plays no part); exp2 and its argument's rounding add 2^-22 plus 2^-24 times the exponent, which
    is at most twice the largest score; relative errors e of the weights move the result by at most 2 max e spread, with
    spread = sum w |v - out| / sum w. The sums over the keys round n times, each by 2^-24 of sum w |v| / sum w <=
    spread + |out|; independent roundings add up to 8 sqrt(n) 2^-24 with eight standard deviations. Range joins add a
    few more roundings of that size (16). bf16 adds the weights' own rounding, at most 2^-8 each (numerator and
    denominator take the same rounded weights), and the output's, 2^-8."""
    M, H, hd = q.shape
    n = kv.shape[0]
    if n == 0:
        return np.zeros(ref.shape)
    G = H // kv.shape[2]
    k = np.abs(kv[:, 0])
    big = np.stack([(np.abs(_np(q))[:, h] @ k[:, h // G].T).max(1) for h in range(H)], 1)[..., None] * abs(scale)
    e = (hd + 4) * 2.0 ** -24 * big + 2.0 ** -22 + 2.0 ** -24 * 2 * 1.4427 * big
    sums = (8 * math.sqrt(n) + 16) * 2.0 ** -24 * (spread + np.abs(ref))
    tol = 2 * e * spread + sums
    if dtype == "bf16":
        tol = tol + 2.0 ** -8 * (1 + 2.0 ** -7) * (spread + np.abs(ref) + tol)
    return tol + 1e-30


def _tensors(*a):
    return [None if t is None else torch.tensor(t, dtype=torch.int32, device=DEV) for t in a]


def _check(g, dtype, H, G, hd, block, S, T, rows, *, lists="all", fresh="rows", of=None, seg_req=None, pad=0, scale=None,
           ws="need", spread_q=1.5, edit=None):
    """One call against the oracle. rows: packed rows per segment; lists: "all" (no tables), "counts" (the first tokens),
    "keys" (random lists, some empty); fresh: "none", "rows" (as many as the request's rows), "list" (through a list)."""
    n_seg = len(rows)
    B = n_seg if seg_req is None else max(seg_req) + 1
    M = sum(rows) + pad
    codes, scales = _cache(g, S, T, H, hd, block, dtype)
    q = (spread_q * torch.randn(M, H * G, hd, generator=g)).to(DT[dtype]).to(DEV)
    start = np.concatenate([[0], np.cumsum(rows)]).tolist()
    counts = {"all": [T] * B, "counts": [(b * 37) % (T + 1) for b in range(B)],
              "keys": [T if b == 0 else 0 if b == 1 else max(1, T * (b + 1) // (B + 2)) for b in range(B)]}[lists]
    keys = torch.stack([torch.randperm(T, generator=g) for _ in range(B)]).int() if lists == "keys" else None
    kv = f_start = f_list = None
    if fresh != "none":
        nf = [rows[b] if fresh == "rows" else (b * 13 + 5) % 90 for b in range(B)]
        f_start = np.concatenate([[0], np.cumsum(nf)]).tolist()
        kv = _rows(g, (max(f_start[-1], 1) if fresh == "rows" else 150, 2, H, hd), dtype)
        if fresh == "list":
            f_list = torch.randint(0, 150, (max(f_start[-1], 1),), generator=g).int()
    if edit is not None:
        edit(codes, scales, q, kv, keys)
    out = torch.full_like(q, 7.0)
    t_start, t_fs, t_of, t_sr = _tensors(start, f_start, of, seg_req)
    t_nk = _tensors(counts)[0] if lists != "all" else None
    t_keys = keys.to(DEV) if keys is not None else None
    t_fl = f_list.to(DEV) if f_list is not None else None
    work = None
    if ws == "need":
        n = MS.ms_kv8_attention_workspace_bytes(q, codes, t_start, keys=t_keys, fresh=kv, fresh_list=t_fl)
        work = torch.full((n // 4 + 4,), float("nan"), device=DEV)
    elif ws:
        work = torch.full((ws // 4,), float("nan"), device=DEV)
    sc = hd ** -0.5 if scale is None else scale

    def call(stream=None):
        MS.ms_kv8_attention(q, codes, scales, out, t_start, block=block, seg_req=t_sr, cache_of=t_of, keys=t_keys, n_keys=t_nk,
                            fresh=kv, fresh_list=t_fl, fresh_start=t_fs, scale=scale, workspace=work, stream=stream)
    call()
    torch.cuda.synchronize()
    worst = 0.0
    refs = []
    for s in range(n_seg):
        b = s if seg_req is None else seg_req[s]
        c = b if of is None else of[b]
        k = np.zeros((0, 2, H, hd))
        if 0 <= c < S:
            k = kv8.values(codes[c].cpu().numpy(), scales[c].cpu().numpy(), block)
            at = keys[b, :counts[b]].numpy() if keys is not None else np.arange(counts[b])
            k = k[at[(at >= 0) & (at < T)]]
        if kv is not None:
            at = np.arange(f_start[b], f_start[b + 1])
            k = np.concatenate([k, _np(kv)[f_list.numpy()[at] if f_list is not None else at]])
        rs = slice(start[s], start[s + 1])
        ref, spread = kv8.attention(_np(q[rs]), k[:, 0], k[:, 1], sc)
        got = _np(out[rs])
        tol = _bound(q[rs], k, ref, spread, sc, dtype)
        assert np.array_equal(np.isnan(got), np.isnan(ref)), f"segment {s}: NaN in other places"
        off = np.abs(got - ref)
        fine = ~np.isnan(ref)
        assert np.all(off[fine] <= tol[fine]), f"segment {s}: {(off - tol)[fine].max():.3e} beyond, {len(k)} keys"
        if fine.any() and off[fine].size:
            worst = max(worst, float((off[fine] / np.maximum(tol[fine], 1e-30)).max()))
        refs.append(ref)
    assert bool((out[start[-1]:] == 7.0).all())      # rows behind the last segment
    print(f"[parity] {dtype} {H}x{G} hd {hd} T {T} rows {rows[:6]}: {worst:.2f} of the bound", flush=True)
    return out, call, refs


@pytest.mark.parametrize("dtype,hd", [("bf16", h) for h in range(8, 129, 8)] + [("fp32", h) for h in range(8, 65, 8)])
def test_attention_head_dims(dtype, hd):
    """Few and many rows, lists with and without, fresh rows, at every head_dim."""
    g = torch.Generator().manual_seed(hd)
    _check(g, dtype, 2, 1, hd, 32, 2, 150, [3, 140], lists="keys")
    _check(g, dtype, 1, 2, hd, 64, 1, 70, [9], lists="counts", fresh="none")
    _check(g, dtype, 3, 1, hd, 16, 3, 200, [1, 17, 300], lists="counts", fresh="list")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 1000])
@pytest.mark.parametrize("rows", [1, 2, 16, 17, 33, 65, 129])
def test_attention_lengths(dtype, T, rows):
    """Keys and rows at and beside tile edges; without fresh rows, and with them."""
    g = torch.Generator().manual_seed(T * 1000 + rows)
    _check(g, dtype, 1, 1, 64, 64, 1, T, [rows], fresh="none")
    _check(g, dtype, 2, 1, 40, 16, 1, T, [rows], lists="keys")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H,G", [(1, 8), (2, 3), (4, 4), (1, 32), (3, 16), (2, 64)])
@pytest.mark.parametrize("rows", [[1], [5, 0, 2], [40, 7]])
def test_attention_shared_heads(dtype, H, G, rows):
    g = torch.Generator().manual_seed(H * G + len(rows))
    _check(g, dtype, H, G, 64, 32, len(rows), 190, rows, lists="keys" if len(rows) > 1 else "all")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block", [1, 2, 4, 8, 16, 32, 64, 128])
def test_attention_blocks(dtype, block):
    g = torch.Generator().manual_seed(block)
    _check(g, dtype, 2, 1, 64, block, 2, 333, [7, 150], lists="keys")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_attention_batches(dtype):
    """Requests with no rows, no keys, neither; shared caches; a cache number outside (fresh rows still count); segments
    in another order than requests, two of one request; rows behind the last segment; 128 requests."""
    g = torch.Generator().manual_seed(3)
    _check(g, dtype, 2, 1, 64, 32, 2, 100, [0, 3, 0, 20, 1], of=[1, 0, 1, 0, 1], lists="keys", pad=5)
    _check(g, dtype, 2, 1, 64, 32, 2, 100, [4, 3, 2], of=[2, -1, 1], lists="all", fresh="none", pad=1)
    _check(g, dtype, 2, 1, 64, 32, 3, 100, [4, 30, 2, 70], seg_req=[2, 0, 2, 1], lists="keys", fresh="list", pad=3)
    _check(g, dtype, 1, 1, 32, 16, 1, 50, [0, 0], of=[0, 0], lists="counts", fresh="none", pad=2)
    _check(g, dtype, 1, 2, 16, 16, 128, 20, [b % 4 for b in range(128)], lists="counts", fresh="list")
    _check(g, dtype, 1, 1, 64, 32, 2, 64, [70, 80], lists="keys", fresh="none")      # the second request: no key at all


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[1], [3, 1, 16], [200]])
def test_attention_workspaces(dtype, rows):
    """No workspace, less than wanted, as wanted and more, all filled with NaN before."""
    for ws in (0, 4096, 70000, "need", 1 << 26):
        g = torch.Generator().manual_seed(8)
        _check(g, dtype, 2, 1, 64, 64, len(rows), 3000, rows, ws=ws, lists="keys" if len(rows) > 1 else "all")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[2], [150]])
def test_attention_long_list(dtype, rows):
    """20000 keys: softmax over many tiles, many key ranges."""
    g = torch.Generator().manual_seed(9)
    _check(g, dtype, 1, 1, 64, 128, 1, 20000, rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[3], [100]])
def test_attention_unlisted_tokens_have_no_effect(dtype, rows):
    """NaN codes and NaN scales of unlisted tokens, list entries outside the cache."""
    g = torch.Generator().manual_seed(10)

    def edit(codes, scales, q, kv, keys):
        listed = keys[0, :64].long().clone()
        keys[0, :128] = torch.cat([listed.int(), torch.full((64,), -1, dtype=torch.int32)])[torch.randperm(128, generator=g)]
        keys[0, 5], keys[0, 77] = 300, 1 << 30
        left = torch.ones(300, dtype=torch.bool)
        left[listed] = False
        codes[0, left.to(DEV)] = 0x7f
        scales[0, left.to(DEV)] = 255       # block 1: a scale per token
    _check(g, dtype, 2, 1, 64, 1, 1, 300, rows, lists="keys", fresh="rows", edit=lambda *a: edit(*a))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[3], [100]])
@pytest.mark.parametrize("where", ["k", "v", "scale", "fresh", "q"])
def test_attention_nan_of_a_listed_key_shows(dtype, rows, where):
    g = torch.Generator().manual_seed(12)

    def edit(codes, scales, q, kv, keys):
        if where == "k":
            codes[0, 100, 0, 1, 3] = 0xff
        elif where == "v":
            codes[0, 100, 1, 1, 3] = 0x7f
        elif where == "scale":
            scales[0, 2, 0, 0] = 255
        elif where == "fresh":
            kv[1, 0, 1, 7] = math.nan
        else:
            q[1, 0, 5] = math.nan
    _check(g, dtype, 2, 1, 64, 32, 1, 180, rows, edit=edit)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[4], [130]])
def test_attention_large_and_rising_scores(dtype, rows):
    """Scores of some hundreds whose largest comes last, first and in the middle (the running maximum moves), equal
    scores, scores far below the others, scales of 2^60 and 2^-60."""
    def rising(codes, scales, q, kv, keys):
        q[:, :, 1:] = 0
        codes[0, :, 0] = 0
        codes[0, :, 0, :, 0] = torch.arange(300, device=DEV).div(3, rounding_mode="floor").clamp(max=126).to(torch.uint8)[:, None]
        q[1::2] *= -1
        scales[0, :, 0] = 127 + 4
    def equal(codes, scales, q, kv, keys):
        q.zero_()
    def big(codes, scales, q, kv, keys):
        scales[:, :, 0] += 60
        q.mul_(2.0 ** -60)
        scales[:, :, 1] -= 60
        kv[:, 0] *= 2.0 ** 60
        kv[:, 1] *= 2.0 ** -60
    for e in (rising, equal, big):
        g = torch.Generator().manual_seed(13)
        _check(g, dtype, 2, 1, 64, 32, 1, 300, rows, edit=e)
    for scale in (1.0, -0.5, 1e-6):
        g = torch.Generator().manual_seed(14)
        _check(g, dtype, 2, 1, 64, 32, 1, 300, rows, scale=scale)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [[3, 2], [100, 140]])
def test_attention_in_place_other_stream_and_again(dtype, rows):
    """out = q; a side stream; the same call twice: the same bits."""
    g = torch.Generator().manual_seed(15)
    out, call, _ = _check(g, dtype, 2, 1, 64, 32, 2, 500, rows, lists="all")
    first = out.clone()
    out.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    call(side)
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    codes, scales = _cache(g, 2, 500, 2, 64, 32, dtype)
    q = torch.randn(sum(rows), 2, 64, generator=g).to(DT[dtype]).to(DEV)
    start = torch.tensor([0, rows[0], sum(rows)], dtype=torch.int32, device=DEV)
    n = MS.ms_kv8_attention_workspace_bytes(q, codes, start)
    ws = torch.empty(n + 16, dtype=torch.uint8, device=DEV)
    sep = torch.empty_like(q)
    MS.ms_kv8_attention(q, codes, scales, sep, start, block=32, workspace=ws)
    MS.ms_kv8_attention(q, codes, scales, q, start, block=32, workspace=ws)
    assert torch.equal(q, sep)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_captured_calls_replay(dtype):
    """Key list, rewrite, read back and attention in one graph, replayed with eager work and new inputs between."""
    g = torch.Generator().manual_seed(16)
    S, T, H, hd, block = 2, 300, 2, 64, 32
    codes, scales = _cache(g, S, T, H, hd, block, dtype)
    mask = torch.zeros(S, T, dtype=torch.uint8, device=DEV)
    keys, n = torch.zeros(S, T, dtype=torch.int32, device=DEV), torch.zeros(S, dtype=torch.int32, device=DEV)
    new, src = _rows(g, (40, 2, H, hd), dtype), torch.full((S, T), -1, dtype=torch.int32, device=DEV)
    kv = torch.zeros(S, T, 2, H, hd, dtype=DT[dtype], device=DEV)
    q = torch.randn(90, H, hd, generator=g).to(DT[dtype]).to(DEV)
    start = torch.tensor([0, 2, 90], dtype=torch.int32, device=DEV)
    fresh, fs = _rows(g, (90, 2, H, hd), dtype), start
    ws = torch.empty(MS.ms_kv8_attention_workspace_bytes(q, codes, start, keys=keys, fresh=fresh) + 16, dtype=torch.uint8, device=DEV)

    def step(codes, scales, kv, out):
        MS.ms_kv8_keys(mask, keys, n)
        MS.ms_kv8_quantize(new, codes, scales, block=block, src_row=src)
        MS.ms_kv8_dequantize(codes, scales, kv, block=block, keys=keys, n_keys=n)
        MS.ms_kv8_attention(q, codes, scales, out, start, block=block, keys=keys, n_keys=n, fresh=fresh, fresh_start=fs,
                            workspace=ws)
    out = torch.zeros_like(q)
    step(codes.clone(), scales.clone(), kv.clone(), out.clone())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(codes, scales, kv, out)
    for i in range(4):
        mask.copy_((torch.rand(S, T, generator=g) < 0.3 * i).to(torch.uint8))
        src.copy_(torch.where(torch.rand(S, T, generator=g) < 0.1, torch.randint(0, 40, (S, T), generator=g).int(), -1))
        new.copy_(_rows(g, (40, 2, H, hd), dtype))
        q.copy_(torch.randn(90, H, hd, generator=g).to(DT[dtype]))
        c2, s2, kv2, out2 = codes.clone(), scales.clone(), kv.clone(), torch.zeros_like(q)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        step(c2, s2, kv2, out2)
        torch.cuda.synchronize()
        for a, b in ((codes, c2), (scales, s2), (kv, kv2), (out, out2)):
            assert torch.equal(a, b)


def test_two_calls_at_once():
    """Two streams, each with its own workspace and output: the bits of each alone."""
    g = torch.Generator().manual_seed(17)
    S, T, H, hd, block = 2, 4000, 4, 64, 64
    codes, scales = _cache(g, S, T, H, hd, block, "bf16")
    calls = []
    for rows in (4, 300):
        q = torch.randn(2 * rows, H, hd, generator=g).bfloat16().to(DEV)
        start = torch.tensor([0, rows, 2 * rows], dtype=torch.int32, device=DEV)
        ws = torch.empty(MS.ms_kv8_attention_workspace_bytes(q, codes, start) + 16, dtype=torch.uint8, device=DEV)
        calls.append((q, start, ws, torch.zeros_like(q)))
    alone = []
    for q, start, ws, out in calls:
        MS.ms_kv8_attention(q, codes, scales, out, start, block=block, workspace=ws)
        torch.cuda.synchronize()
        alone.append(out.clone())
        out.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for st, (q, start, ws, out) in zip(streams, calls):
            MS.ms_kv8_attention(q, codes, scales, out, start, block=block, workspace=ws, stream=st)
    torch.cuda.synchronize()
    for (_, _, _, out), want in zip(calls, alone):
        assert torch.equal(out, want)


def test_round_trip_as_used():
    """A template written, an edit's rows attending over its unmasked tokens and themselves, the rows written into the
    cache, and the result read back: each against the oracle on the outputs of the one before."""
    g = torch.Generator().manual_seed(18)
    T, H, hd, block = 200, 3, 72, 64
    template = _rows(g, (1, T, 2, H, hd), "bf16")
    codes, scales = _empty_cache(1, T, H, hd, block)
    MS.ms_kv8_quantize(template, codes, scales, block=block)
    mask = torch.zeros(1, T, dtype=torch.uint8)
    mask[0, 40:75] = 1
    keys, n = torch.zeros(1, T, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    MS.ms_kv8_keys(mask.to(DEV), keys, n)
    fresh = _rows(g, (35, 2, H, hd), "bf16")
    q = torch.randn(35, H, hd, generator=g).bfloat16().to(DEV)
    out, start = torch.zeros_like(q), torch.tensor([0, 35], dtype=torch.int32, device=DEV)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=block, keys=keys, n_keys=n, fresh=fresh, fresh_start=start)
    c, e = _oracle_cache(template, block)
    k = np.concatenate([kv8.values(c[0], e[0], block)[mask[0].numpy() == 0], _np(fresh)])
    ref, spread = kv8.attention(_np(q), k[:, 0], k[:, 1], hd ** -0.5)
    assert np.all(np.abs(_np(out) - ref) <= _bound(q, k, ref, spread, hd ** -0.5, "bf16"))
    src = torch.full((1, T), -1, dtype=torch.int32)
    src[0, 40:75] = torch.arange(35, dtype=torch.int32)
    MS.ms_kv8_quantize(fresh, codes, scales, block=block, src_row=src.to(DEV))
    c, e = kv8.rewrite(c[0], e[0], block, _np(fresh), src[0].numpy())
    back = torch.zeros(1, T, 2, H, hd, dtype=torch.bfloat16, device=DEV)
    MS.ms_kv8_dequantize(codes, scales, back, block=block)
    assert np.array_equal(_np(back[0]), kv8.values(c, e, block))


def test_binding_refusals_on_the_gpu():
    """What the binding refuses with tensors on the GPU."""
    codes, scales = _empty_cache(2, 40, 4, 64, 16)
    kv, q = torch.zeros(2, 40, 2, 4, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(10, 8, 64, dtype=torch.bfloat16, device=DEV)
    start = torch.tensor([0, 4, 10], dtype=torch.int32, device=DEV)
    bad = [lambda: MS.ms_kv8_quantize(kv[:, :30], codes, scales, block=16), lambda: MS.ms_kv8_quantize(kv[:1], codes, scales, block=16),
           lambda: MS.ms_kv8_quantize(kv.transpose(0, 1), codes, scales, block=16),
           lambda: MS.ms_kv8_quantize(kv, codes, scales, block=16, src_row=torch.zeros(2, 40, dtype=torch.int32, device=DEV)),
           lambda: MS.ms_kv8_quantize(kv[0], codes, scales, block=16, src_row=torch.zeros(2, 40, dtype=torch.int64, device=DEV)),
           lambda: MS.ms_kv8_quantize(kv, codes[:, :, :, :, :32], scales, block=16),
           lambda: MS.ms_kv8_dequantize(codes, scales, kv, block=16, keys=start),
           lambda: MS.ms_kv8_dequantize(codes, scales, kv, block=16, n_keys=start),
           lambda: MS.ms_kv8_attention(q[:, :, :32], codes, scales, q, start, block=16),
           lambda: MS.ms_kv8_attention(q, codes, scales, q[:5], start, block=16),
           lambda: MS.ms_kv8_attention(q[:, :6].contiguous(), codes, scales, q[:, :6].contiguous(), start, block=16),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start, block=16, fresh=kv[0]),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start, block=16, fresh=kv[0].float(), fresh_start=start),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start.long(), block=16),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start.cpu(), block=16),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start, block=16, cache_of=start.long()),
           lambda: MS.ms_kv8_attention(q, codes, scales, torch.zeros_like(q), start, block=16, cache_of=start[:1])]
    for f in bad:
        with pytest.raises(MS.MaskStepError):
            f()
    torch.cuda.synchronize()
    assert bool((codes == 0x55).all()) and bool((scales == 0x55).all())


@pytest.mark.parametrize("dtype,H,hd", [("bf16", 31, 128), ("fp32", 62, 64)])
@pytest.mark.parametrize("rows", [2, 300])
def test_attention_at_the_end_of_the_largest_cache(dtype, H, hd, rows):
    """One cache of 3968 MiB of codes: row offsets just below 2^32."""
    T, block, n = 1 << 19, 64, 200
    codes = torch.zeros(1, T, 2, H, hd, dtype=torch.uint8, device=DEV)
    scales = torch.full((1, T // block, 2, H), 127, dtype=torch.uint8, device=DEV)
    g = torch.Generator().manual_seed(19)
    kv = _rows(g, (1, 256, 2, H, hd), dtype)
    MS.ms_kv8_quantize(kv, codes[:, T - 256:], scales[:, -256 // block:], block=block)
    c, e = _oracle_cache(kv, block)
    k = kv8.values(c[0], e[0], block)[256 - n:]
    q = torch.randn(rows, H, hd, generator=g).to(DT[dtype]).to(DEV)
    keys = torch.arange(T - n, T, dtype=torch.int32, device=DEV)[None]
    out, start = torch.zeros_like(q), torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=block, keys=keys)
    ref, spread = kv8.attention(_np(q), k[:, 0], k[:, 1], hd ** -0.5)
    assert np.all(np.abs(_np(out) - ref) <= _bound(q, k, ref, spread, hd ** -0.5, dtype))


def test_two_graphs_share_a_workspace():
    """Two captured calls with one workspace, replayed in turn on one stream: the bits of each alone."""
    g = torch.Generator().manual_seed(20)
    codes, scales = _cache(g, 2, 3000, 4, 64, 64, "bf16")
    calls, need = [], 0
    for rows in (3, 40):
        q = torch.randn(2 * rows, 4, 64, generator=g).bfloat16().to(DEV)
        start = torch.tensor([0, rows, 2 * rows], dtype=torch.int32, device=DEV)
        need = max(need, MS.ms_kv8_attention_workspace_bytes(q, codes, start))
        calls.append((q, start, torch.zeros_like(q)))
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    graphs, alone = [], []
    for q, start, out in calls:
        MS.ms_kv8_attention(q, codes, scales, out, start, block=64, workspace=ws)
        torch.cuda.synchronize()
        alone.append(out.clone())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            MS.ms_kv8_attention(q, codes, scales, out, start, block=64, workspace=ws)
        graphs.append(graph)
    for _ in range(3):
        for _, _, out in calls:
            out.zero_()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for (_, _, out), want in zip(calls, alone):
            assert torch.equal(out, want)
        ws.fill_(0xFF)

"""The 8-bit K/V cache where it could go wrong unseen."""
import numpy as np
import pytest
import torch

from oracle import kv8
from paper_2505_20600_amd import maskstep as MS
from tests import gpu_helpers as G
from tests import test_gpu_kv8 as K
from tests import test_gpu_kv8_step as S

pytestmark = pytest.mark.gpu
DEV = K.DEV


# ------------------------------------------------------------------ absent keys

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 25, 200])
@pytest.mark.parametrize("block", [1, 32])
@pytest.mark.parametrize("T", [45, 180])
@pytest.mark.parametrize("fresh", ["none", "rows"])
def test_unlisted_first_block_of_nan_scales_has_no_effect(dtype, rows, block, T, fresh):
    """Token 0's block holds NaN codes and NaN scales and is not listed: neither the lanes past the list's end (45 and 180
    keys end inside every tile) nor list entries outside the cache may take them."""
    for bad in (False, True):
        g = torch.Generator().manual_seed(T + rows)

        def edit(codes, scales, q, kv, keys):
            keys[0] = torch.randint(block, T, (T,), generator=g).int()
            if bad:
                keys[0, 3::7] = -1
                keys[0, T // 2] = 1 << 30
            codes[0, :block] = 0x7f
            scales[0, 0] = 255
        _, _, refs = K._check(g, dtype, 2, 1, 64, block, 1, T, [rows], lists="keys", fresh=fresh, edit=edit)
        assert np.isfinite(refs[0]).all()


@pytest.mark.parametrize("dtype,hd", [("bf16", h) for h in range(8, 129, 8)] + [("fp32", h) for h in range(8, 65, 8)])
def test_unlisted_first_block_at_every_head_dim(dtype, hd):
    for rows in (3, 40, 130):
        g = torch.Generator().manual_seed(hd + rows)

        def edit(codes, scales, q, kv, keys):
            keys[0] = torch.randint(16, 77, (77,), generator=g).int()
            codes[0, :16] = 0xff
            scales[0, 0] = 255
        _, _, refs = K._check(g, dtype, 1, 2, hd, 16, 1, 77, [rows], lists="keys", fresh="none", edit=edit)
        assert np.isfinite(refs[0]).all()


@pytest.mark.parametrize("shape", S.SHAPES, ids=lambda s: s.name)
@pytest.mark.parametrize("pinned", [False, True], ids=["resident", "streamed"])
def test_step_does_not_read_scales_of_masked_blocks(shape, pinned):
    """A mask over the first 40 tokens: their block's NaN scales and codes change no bit of the step."""
    ws, xt, codes, scales, kv, yc = S._inputs(shape, 92)
    mask = np.zeros((shape.batch, shape.n_image), np.uint8)
    mask[:, :40] = 1
    x = S.W.edited_hidden(shape, 92, xt, mask)
    want = S.Run(shape, mask, x, codes, scales, yc, ws, pinned=pinned).out()
    assert np.isfinite(want).all()
    codes, scales = [c.copy() for c in codes], [s.copy() for s in scales]
    for c, s in zip(codes, scales):
        c[:, :40] = 0x7f
        s[:, 0] = 255                                   # tokens 0 to 31, all masked
    np.testing.assert_array_equal(S.Run(shape, mask, x, codes, scales, yc, ws, pinned=pinned).out(), want)


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("bf16", 72), ("bf16", 40), ("fp32", 64), ("fp32", 24)])
@pytest.mark.parametrize("rows", [2, 30, 150])
def test_unlisted_fresh_rows_have_no_effect(dtype, hd, rows):
    """NaN in every fresh row that the list does not name, row 0 among them; list entries outside the rows; ranges that end
    inside a tile; a request without fresh rows."""
    g = torch.Generator().manual_seed(hd + rows)
    codes, scales = K._cache(g, 2, 50, 2, hd, 16, dtype)
    q = torch.randn(2 * rows, 2, hd, generator=g).to(K.DT[dtype]).to(DEV)
    kv = K._rows(g, (120, 2, 2, hd), dtype)
    rest = torch.randperm(119, generator=g)[:77] + 1
    left = torch.ones(120, dtype=torch.bool)
    left[rest] = False
    kv[left.to(DEV)] = float("nan")
    named = rest.int()
    named[5], named[40] = -1, 120
    start, fs = (torch.tensor(t, dtype=torch.int32, device=DEV) for t in ([0, rows, 2 * rows], [0, 77, 77]))
    out = torch.empty_like(q)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=16, fresh=kv, fresh_list=named.to(DEV), fresh_start=fs)
    for b in range(2):
        k = kv8.values(codes[b].cpu().numpy(), scales[b].cpu().numpy(), 16)
        if b == 0:
            k = np.concatenate([k, K._np(kv)[named[(named >= 0) & (named < 120)].numpy()]])
        rs = slice(b * rows, (b + 1) * rows)
        ref, spread = kv8.attention(K._np(q[rs]), k[:, 0], k[:, 1], hd ** -0.5)
        assert np.isfinite(ref).all()
        assert np.all(np.abs(K._np(out[rs]) - ref) <= K._bound(q[rs], k, ref, spread, hd ** -0.5, dtype))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block", [1, 8, 32, 64, 128])
@pytest.mark.parametrize("fill", [0xff, 0x7f])
def test_cache_filled_in_part(dtype, block, fill):
    """Codes and scales of NaN all over, some tokens written through src_row: they read back and are attended over as if
    the cache held nothing else; the rest stays NaN."""
    g = torch.Generator().manual_seed(block)
    T, H, hd = 300, 2, 64
    codes, scales = K._empty_cache(1, T, H, hd, block, fill)
    scales.fill_(255)
    kv = K._rows(g, (90, 2, H, hd), dtype)
    src = torch.full((1, T), -1, dtype=torch.int32)
    src[0, 130:220] = torch.arange(90, dtype=torch.int32)
    c, e = kv8.rewrite(codes[0].cpu().numpy(), scales[0].cpu().numpy(), block, K._np(kv), src[0].numpy())
    MS.ms_kv8_quantize(kv, codes, scales, block=block, src_row=src.to(DEV))
    assert np.array_equal(scales[0].cpu().numpy(), e) and K._same_codes(codes[0].cpu().numpy(), c)
    vals = kv8.values(c, e, block)
    assert np.isfinite(vals[130:220]).all() and np.isnan(vals[:130]).all() and np.isnan(vals[220:]).all()
    keys = (130 + torch.randperm(90, generator=g)).int()[None].to(DEV)
    for rows in (1, 30, 150):
        q = torch.randn(rows, H, hd, generator=g).to(K.DT[dtype]).to(DEV)
        out, start = torch.empty_like(q), torch.tensor([0, rows], dtype=torch.int32, device=DEV)
        MS.ms_kv8_attention(q, codes, scales, out, start, block=block, keys=keys)
        k = vals[keys[0].cpu().numpy()]
        ref, spread = kv8.attention(K._np(q), k[:, 0], k[:, 1], 0.125)
        assert np.all(np.abs(K._np(out) - ref) <= K._bound(q, k, ref, spread, 0.125, dtype))


# ------------------------------------------------------------------ rewriting

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block,T", [(1, 17), (8, 31), (32, 33), (64, 65), (64, 127), (128, 129), (128, 200)])
def test_rewrite_of_a_ragged_last_group(dtype, block, T):
    """The last workgroup of tokens holds 1 to 72 of its 16 to 128 rows; the rewritten rows are in it."""
    g = torch.Generator().manual_seed(T)
    codes, scales = K._cache(g, 2, T, 3, 40, block, dtype)
    kv = K._rows(g, (T, 2, 3, 40), dtype, width=5.0)
    src = torch.full((2, T), -1, dtype=torch.int32)
    src[:, T - 1], src[1, T - 5] = 0, 3
    want = [kv8.rewrite(codes[s].cpu().numpy(), scales[s].cpu().numpy(), block, K._np(kv), src[s].numpy()) for s in range(2)]
    MS.ms_kv8_quantize(kv, codes, scales, block=block, src_row=src.to(DEV))
    assert np.array_equal(scales.cpu().numpy(), np.stack([e for _, e in want]))
    assert K._same_codes(codes.cpu().numpy(), np.stack([c for c, _ in want]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("width", [-1, 1])
def test_rewrite_beside_the_largest_value(dtype, width):
    """The type's largest value is written as code 256 at the scale 2^120, a value of 2^128 that no float32 holds: it keeps
    its code when a neighbour is rewritten."""
    big = torch.finfo(K.DT[dtype]).max
    kv = torch.ones(1, 16, 2, 1, 8)
    kv[0, 3], kv[0, 4, 0, 0, 1] = big, -big
    kv = kv.to(K.DT[dtype]).to(DEV)
    codes, scales = K._empty_cache(1, 16, 1, 8, 16)
    MS.ms_kv8_quantize(kv, codes, scales, block=16)
    assert bool((scales == 247).all()) and int(codes[0, 3, 0, 0, 0]) == 120
    new = torch.full((1, 2, 1, 8), 2.0 ** (100 * width), dtype=K.DT[dtype], device=DEV)
    src = torch.full((1, 16), -1, dtype=torch.int32, device=DEV)
    src[0, 7] = 0
    c, e = kv8.rewrite(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 16, K._np(new), src[0].cpu().numpy())
    MS.ms_kv8_quantize(new, codes, scales, block=16, src_row=src)
    assert np.array_equal(scales[0].cpu().numpy(), e) and K._same_codes(codes[0].cpu().numpy(), c)
    assert int(codes[0, 3, 0, 0, 0]) == 120


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_kept_zeros_of_a_large_scale_stay_zeros(dtype):
    """One row of large values in every block is replaced by small ones of 1 to 2^-150 times their size (from every scale
    to every smaller one, those more than 2^127 apart included); the zeros beside it, of both signs, keep their codes."""
    scales = torch.arange(120, 255).view(1, -1, 1, 1).expand(1, -1, 2, 1)
    n = scales.shape[1]
    codes = torch.zeros(1, n, 4, 2, 1, 8, dtype=torch.uint8)
    codes[..., 1::2] = 0x80
    codes[:, :, 2] = 126
    for less in range(0, 151):
        kv = torch.ldexp(torch.ones(n, 2, 1, 8, dtype=torch.float64), (scales[0, :, :1].view(n, 1, 1, 1) - 127 - less).int())
        kv = kv.to(torch.float32).to(K.DT[dtype])
        src = torch.full((1, n, 4), -1, dtype=torch.int32)
        src[0, :, 2] = torch.arange(n, dtype=torch.int32)
        dc, ds = codes.view(1, 4 * n, 2, 1, 8).to(DEV), scales.to(torch.uint8).to(DEV).contiguous()
        MS.ms_kv8_quantize(kv.to(DEV), dc, ds, block=4, src_row=src.view(1, -1).to(DEV))
        assert torch.equal(dc.view(1, n, 4, 2, 1, 8)[:, :, [0, 1, 3]].cpu(), codes[:, :, [0, 1, 3]]), f"2^-{less}"
        if less % 25 == 0:
            c, e = kv8.rewrite(codes.view(4 * n, 2, 1, 8).numpy(), scales[0].to(torch.uint8).numpy(), 4, K._np(kv),
                               src.view(-1).numpy())
            assert np.array_equal(ds[0].cpu().numpy(), e) and K._same_codes(dc[0].cpu().numpy(), c)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("block,T", [(1, 40), (4, 70), (32, 100), (64, 200), (128, 300)])
@pytest.mark.parametrize("special", [False, True], ids=["finite", "nan"])
def test_rewrite_of_every_scale_is_exact(dtype, block, T, special):
    """Caches of random codes at every exponent byte (foreign ones too: quantize itself writes 1..247), new rows of every
    magnitude down to zero and the subnormals, with and without NaN and infinities in both; ragged last groups."""
    g = torch.Generator().manual_seed(T + block)
    H, hd = 2, 16
    codes = torch.randint(0, 127, (3, T, 2, H, hd), generator=g) + 128 * torch.randint(0, 2, (3, T, 2, H, hd), generator=g)
    scales = torch.randint(0, 255, (3, -(-T // block), 2, H), generator=g)
    codes[2] = codes[2] & 0x87                                      # magnitudes of the subnormal codes only
    kv = torch.randn(50, 2, H, hd, generator=g, dtype=torch.float64)
    kv *= torch.exp2(torch.randint(-140, 126, (50, 1, H, 1), generator=g).double())
    kv[::9] = 0
    kv = kv.to(torch.float32).to(K.DT[dtype])
    kv[4] = torch.finfo(K.DT[dtype]).max
    if special:
        scales[torch.rand(scales.shape, generator=g) < 0.1] = 255
        codes[torch.rand(codes.shape, generator=g) < 0.003] = 0x7f
        kv[torch.rand(kv.shape, generator=g) < 0.003] = float("inf")
        kv[torch.rand(kv.shape, generator=g) < 0.003] = float("nan")
    src = torch.where(torch.rand(3, T, generator=g) < 0.2, torch.randint(0, 50, (3, T), generator=g), -1).int()
    codes, scales = codes.to(torch.uint8), scales.to(torch.uint8)
    want = [kv8.rewrite(codes[s].numpy(), scales[s].numpy(), block, K._np(kv), src[s].numpy()) for s in range(3)]
    dc, ds = codes.to(DEV), scales.to(DEV)
    MS.ms_kv8_quantize(kv.to(DEV), dc, ds, block=block, src_row=src.to(DEV))
    assert np.array_equal(ds.cpu().numpy(), np.stack([e for _, e in want]))
    assert K._same_codes(dc.cpu().numpy(), np.stack([c for c, _ in want]))


# ------------------------------------------------------------------ the step's tensors

def test_step_refuses_tables_and_caches_of_another_kind():
    """int64, short and host cache_of; scales for another block; caches of another count; codes on the host, pinned ones
    on the GPU. Addresses given as int and stacked tensors are taken."""
    shape = S.SHAPES[1]
    ws, xt, codes, scales, kv, yc = S._inputs(shape, 94)
    mask = S._masks(shape, (0.3, 0.1), 15)
    x = S.W.edited_hidden(shape, 94, xt, mask)
    run, streamed = (S.Run(shape, mask, x, codes, scales, yc, ws, pinned=p) for p in (False, True))
    want = run.out()
    of = torch.tensor([0, 1], dtype=torch.int32, device=DEV)
    run.y.fill_(3.0)
    held, host = run.codes, [c.cpu() for c in run.codes]
    for change in (dict(cache_of=of.long()), dict(cache_of=of[:1]), dict(cache_of=of.cpu()), dict(block=16), dict(block=64)):
        with pytest.raises(MS.MaskStepError):
            run.step.stack_forward_kv8(run.wc, run.x, run.yc, run.codes, run.scales, run.y, **{**run.kw, **change})
    for codes_, scales_ in ((host, run.scales), ([c[:1].contiguous() for c in held], run.scales),
                            (held, [s[:1].contiguous() for s in run.scales]), (held, [s.cpu() for s in run.scales])):
        with pytest.raises(MS.MaskStepError):
            run.step.stack_forward_kv8(run.wc, run.x, run.yc, codes_, scales_, run.y, **run.kw)
    with pytest.raises(MS.MaskStepError):
        streamed.step.stack_forward_kv8(run.wc, run.x, run.yc, held, run.scales, run.y, **streamed.kw)
    torch.cuda.synchronize()
    assert bool((run.y == 3.0).all())
    for codes_, kw in ((torch.stack(held), dict(cache_of=of)), ([c.data_ptr() for c in held], dict(cache_of=of.data_ptr()))):
        run.y.fill_(3.0)
        run.step.stack_forward_kv8(run.wc, run.x, run.yc, codes_, run.scales, run.y, **{**run.kw, **kw})
        torch.cuda.synchronize()
        np.testing.assert_array_equal(K._np(run.y), want)


# ------------------------------------------------------------------ empty tables

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [2, 140])
def test_tables_without_entries_name_nothing(dtype, rows):
    """keys of no columns: no cached token is read; a fresh_list of no entries: no fresh row."""
    g = torch.Generator().manual_seed(21)
    codes, scales = K._cache(g, 1, 60, 2, 64, 32, dtype)
    q = torch.randn(rows, 2, 64, generator=g).to(K.DT[dtype]).to(DEV)
    start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    none = torch.zeros(1, 0, dtype=torch.int32, device=DEV)
    fresh = K._rows(g, (rows, 2, 2, 64), dtype)
    out = torch.full_like(q, 7.0)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=32, keys=none)
    assert bool((out == 0).all())
    MS.ms_kv8_attention(q, codes, scales, out, start, block=32, keys=none, fresh=fresh, fresh_start=start)
    k = K._np(fresh)
    ref, spread = kv8.attention(K._np(q), k[:, 0], k[:, 1], 0.125)
    assert np.all(np.abs(K._np(out) - ref) <= K._bound(q, k, ref, spread, 0.125, dtype))
    want = torch.empty_like(q)
    MS.ms_kv8_attention(q, codes, scales, want, start, block=32)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=32, fresh=fresh, fresh_list=none[0], fresh_start=start)
    k = kv8.values(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 32)
    ref, spread = kv8.attention(K._np(q), k[:, 0], k[:, 1], 0.125)
    for t in (want, out):
        assert np.all(np.abs(K._np(t) - ref) <= K._bound(q, k, ref, spread, 0.125, dtype))
    kv = torch.full((1, 60, 2, 2, 64), 7.0, dtype=K.DT[dtype], device=DEV)
    MS.ms_kv8_dequantize(codes, scales, kv, block=32, keys=none)
    assert bool((kv == 7.0).all())


# ------------------------------------------------------------------ the step's timing classes

def test_step_books_the_join_of_key_ranges_as_such():
    """attention and attn_combine of a step over an 8-bit cache, one each per block, as over a K/V cache."""
    shape = S.W.ModelShape("k8_join", 3, 256, 4, 4, 32, 32, dtype="bf16", batch=1)
    ws, xt, codes, scales, kv, yc = S._inputs(shape, 93)
    mask = np.zeros((1, shape.n_image), np.uint8)
    mask[0, 100:104] = 1
    run = S.Run(shape, mask, S.W.edited_hidden(shape, 93, xt, mask), codes, scales, yc, ws)
    run.out()
    MS.profiler_start(("attention", "attn_combine"), capacity=64)
    y = run.out()
    tot = MS.profiler_stop()
    assert tot["attention"][1] == 3 and tot["attn_combine"][1] == 3
    G.assert_close(y, S.oracle.masked_stack(S.W.edited_hidden(shape, 93, xt, mask), mask, kv, yc, ws, shape, round_p=True),
                   "bf16", "joined ranges", blocks=3, inp=S.W.edited_hidden(shape, 93, xt, mask))


# ------------------------------------------------------------------ scores beyond float32

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 25, 200])
@pytest.mark.parametrize("ws", [0, "need"])
def test_scores_of_minus_infinity_weigh_nothing(dtype, rows, ws):
    """Scores that overflow float32 downwards: beside finite ones they weigh nothing, and a row of nothing else is 0.
    Query column 0 is -2^100; a key's column 0 is 2^100 or 0."""
    g = torch.Generator().manual_seed(22)
    T = 1500
    codes, scales = K._cache(g, 1, T, 2, 64, 1, dtype)
    far = torch.rand(T, generator=g) < 0.5
    codes[0, :, 0, :, 0] = 0
    q = torch.randn(rows, 2, 64, generator=g).to(K.DT[dtype])
    q[:, :, 0] = -2.0 ** 100
    q = q.to(DEV)
    start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    work = None
    if ws:
        work = torch.full((MS.ms_kv8_attention_workspace_bytes(q, codes, start) // 4 + 4,), float("nan"), device=DEV)
    k = kv8.values(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 1)
    k = k[~far.numpy()]
    codes[0, far.to(DEV), 0] = 0
    codes[0, far.to(DEV), 0, :, 0] = 0x38               # 1.0
    scales[0, far.to(DEV), 0] = 227                     # 2^100
    out = torch.empty_like(q)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=1, workspace=work)
    q0 = q.clone()
    q0[:, :, 0] = 0                                     # the finite keys' column 0 is 0
    ref, spread = kv8.attention(K._np(q0), k[:, 0], k[:, 1], 0.125)
    assert np.all(np.abs(K._np(out) - ref) <= K._bound(q0, k, ref, spread, 0.125, dtype))
    only = far.nonzero().flatten().int()[None].to(DEV)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=1, keys=only, workspace=work)
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [3, 25, 200])
@pytest.mark.parametrize("ws", [0, "need"])
@pytest.mark.parametrize("where", [0, 700, 1499])
def test_a_score_of_infinity_makes_its_row_nan(dtype, rows, ws, where):
    """One key's score overflows float32 upwards for every other row; the rows between are as without that key's."""
    g = torch.Generator().manual_seed(23)
    T = 1500
    codes, scales = K._cache(g, 1, T, 1, 64, 1, dtype)
    codes[0, :, 0, :, 0] = 0
    codes[0, where, 0] = 0
    codes[0, where, 0, :, 0] = 0x38
    scales[0, where, 0] = 227
    q = torch.randn(rows, 1, 64, generator=g).to(K.DT[dtype])
    q[:, :, 0] = 0
    q[::2, :, 0] = 2.0 ** 100
    q = q.to(DEV)
    start = torch.tensor([0, rows], dtype=torch.int32, device=DEV)
    work = None
    if ws:
        work = torch.full((MS.ms_kv8_attention_workspace_bytes(q, codes, start) // 4 + 4,), float("nan"), device=DEV)
    out = torch.empty_like(q)
    MS.ms_kv8_attention(q, codes, scales, out, start, block=1, workspace=work)
    assert bool(out[::2].isnan().all())
    k = kv8.values(codes[0].cpu().numpy(), scales[0].cpu().numpy(), 1)
    ref, spread = kv8.attention(K._np(q[1::2]), k[:, 0], k[:, 1], 0.125)
    k[where, 0] = 0                                     # its score in these rows is 0
    assert np.all(np.abs(K._np(out[1::2]) - ref) <= K._bound(q[1::2], k, ref, spread, 0.125, dtype))

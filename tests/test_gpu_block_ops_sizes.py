"""The block operators on the GPU at the largest sizes that they take, as replayed graphs whose tables change, and in flight together, against
the float64 oracle."""
import math

import numpy as np
import pytest
import torch

from oracle import mx4, qk_norm_rope, shared
from paper_2505_20600_amd import maskstep as MS
from tests.test_gpu_block_ops import (DEV, DT, _attend, _attend_bound, _batch, _bits, _check, _int, _np, _qk_case, _qk_check, _randn,
                                      _within)
from tests.test_gpu_block_ops_product import _values

pytestmark = pytest.mark.gpu


def _rows_check(q, out, rows, kv, seen, own, what):
    """Rows ``rows`` of out against the oracle over the prefix rows ``seen`` (None: all) and the own rows ``own``."""
    hd, dtype = q.shape[2], "bf16" if q.dtype == torch.bfloat16 else "fp32"
    kv = kv if seen is None else kv[seen.to(DEV)]
    qs, n = _np(q[rows]), len(rows)
    fresh, start = (None, None) if own is None else (_np(own), [0, len(own)])
    want, spread, size, reach = shared.attention(qs, _np(kv), None, [0, n], fresh, start, 1 / math.sqrt(hd))
    keys = len(kv) + (0 if own is None else len(own))
    _within(_np(out[rows]), want, _attend_bound(want, spread, size, reach, keys, hd, dtype), what)


@pytest.mark.parametrize("dtype,hd", [("bf16", 128), ("fp32", 64)])
@pytest.mark.parametrize("rows", [3, 60, 500])
def test_prefix_and_own_rows_of_almost_4_gib(dtype, hd, rows):
    """Offsets past 31 bits and up to the limit: a few tokens seen, at both ends and between; own rows at the end of their buffer."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    T, G = 1_040_000, 8
    kv = torch.randn(T, 2, G, hd, generator=g, device=DEV, dtype=DT[dtype])
    fresh = torch.randn(T, 2, G, hd, generator=g, device=DEV, dtype=DT[dtype])
    q = torch.randn(2 * rows, G, hd, generator=g, device=DEV).to(DT[dtype])
    seen = torch.cat([torch.arange(0, 70), torch.arange(523_990, 524_400), torch.randint(0, T, (200,), generator=torch.Generator().manual_seed(rows)), torch.arange(T - 100, T)]).unique()
    hidden = torch.ones(2, T, dtype=torch.bool)
    hidden[:, seen] = False
    own = [T - 900, T - 800, T]
    need = MS.ms_shared_attention_workspace_bytes(q, kv, fresh=fresh)
    for ws in (None, torch.empty(need + 16, dtype=torch.uint8, device=DEV)):
        out = torch.full_like(q, 7.0)
        MS.ms_shared_attention(q, kv, out, seg_start=_int([0, rows, 2 * rows]), bits=_bits(hidden), fresh=fresh, fresh_start=_int(own), workspace=ws)
        for b in range(2):
            _rows_check(q, out, torch.arange(b * rows, (b + 1) * rows)[::max(1, rows // 40)], kv, seen, fresh[own[b]:own[b + 1]], f"request {b}")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [2, 1000])
def test_prefix_of_most_tokens(dtype, rows):
    g = torch.Generator(device=DEV).manual_seed(rows)
    T = 1 << 20
    kv, q = torch.randn(T, 2, 1, 8, generator=g, device=DEV).to(DT[dtype]), (3 * torch.randn(rows, 1, 8, generator=g, device=DEV)).to(DT[dtype])
    need = MS.ms_shared_attention_workspace_bytes(q, kv)
    for ws in (None, torch.empty(need + 16, dtype=torch.uint8, device=DEV)):
        out = torch.full_like(q, 7.0)
        MS.ms_shared_attention(q, kv, out, workspace=ws)
        _rows_check(q, out, torch.tensor([0, rows // 2, rows - 1]).unique(), kv, None, None, f"{rows} rows")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_most_query_rows(dtype):
    """2^26 rows of two heads: offsets of queries and results past 32 bits."""
    g = torch.Generator(device=DEV).manual_seed(1)
    M, T, hd = 1 << 26, 70, 16
    kv = torch.randn(T, 2, 1, hd, generator=g, device=DEV).to(DT[dtype])
    q = torch.randn(M, 2, hd, generator=g, device=DEV, dtype=DT[dtype])
    out = torch.empty_like(q)
    out[-1000:] = 7.0
    MS.ms_shared_attention(q, kv, out, seg_start=_int([0, M - 500]))
    rows = torch.cat([torch.arange(200), torch.arange(M // 2 - 100, M // 2 + 100), torch.arange(M - 700, M - 500)])
    _rows_check(q, out, rows, kv, None, None, "rows")
    assert bool((out[M - 500:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("M,N,K", [(5, 12, 1 << 20), (300, 100, 1 << 20), (3, 1 << 20, 32), (70, 1 << 20, 64)])
def test_longest_sums_and_widest_outputs(dtype, M, N, K):
    """Codes under one scale: products are quarters and their sums stay below 2^22, so every order of summation is exact."""
    g = torch.Generator(device=DEV).manual_seed(K)
    a, w = ((torch.randint(0, 256, (n, K // 2), generator=g, device=DEV, dtype=torch.uint8),
             torch.full((n, K // 32), 127, dtype=torch.uint8, device=DEV)) for n in (M, N))
    av, wv = _values(*a), _values(*w)
    want = av @ wv.t().contiguous()
    assert float(want.abs().max()) < 2.0 ** 20
    bias = torch.zeros(N, dtype=DT[dtype], device=DEV)
    need = MS.ms_mx4_linear_workspace_bytes(a[0], w[0])
    for ws in (None, torch.empty(need + 16, dtype=torch.uint8, device=DEV)):
        out = torch.full((M, N), 7.0, dtype=DT[dtype], device=DEV)
        MS.ms_mx4_linear(*a, *w, bias, out, workspace=ws)
        assert torch.equal(out, want.to(DT[dtype]))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_most_rows_of_codes(dtype):
    """2^26 rows of 96 columns: three sweeps of the largest launch, offsets past 32 bits."""
    M = 1 << 26
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randn(M, 96, generator=g, device=DEV, dtype=DT[dtype])
    codes, scales = torch.empty(M, 48, dtype=torch.uint8, device=DEV), torch.empty(M, 3, dtype=torch.uint8, device=DEV)
    MS.ms_mx4_quantize(x, codes, scales)
    at = torch.cat([torch.arange(200), torch.arange(M // 2 - 100, M // 2 + 100), torch.randint(0, M, (500,), generator=torch.Generator().manual_seed(3)), torch.arange(M - 200, M)])
    c, s = mx4.quantize(_np(x[at.to(DEV)]))
    assert np.array_equal(codes[at.to(DEV)].cpu().numpy(), c) and np.array_equal(scales[at.to(DEV)].cpu().numpy(), s)
    x.fill_(7.0)
    MS.ms_mx4_dequantize(codes, scales, x)
    assert np.array_equal(_np(x[at.to(DEV)]), mx4.values(c, s))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_norms_of_many_rows_and_heads(dtype):
    """1024 heads of either kind; rows whose offsets pass 32 bits, without K/V rows to write."""
    g = torch.Generator().manual_seed(3)
    for H, G in ((1024, 3), (3, 1024)):
        _qk_check(_qk_case(g, dtype, 5, H, G, 8, 8, 0, 60, 9), dtype, H, G, 8, False)
    M, H, G, hd = 1 << 23, 4, 1, 64
    qkv = torch.randn(M, (H + 2 * G) * hd, generator=torch.Generator(device=DEV).manual_seed(4), device=DEV, dtype=DT[dtype])
    q, kv = torch.empty(M, H, hd, dtype=DT[dtype], device=DEV), torch.empty(0, 2, G, hd, dtype=DT[dtype], device=DEV)
    gain = 1 + _randn(g, (hd,), dtype, 0.3)
    MS.ms_qk_norm_rope(qkv, q, kv, q_gain=gain, k_gain=gain)
    at = torch.cat([torch.arange(100), torch.arange(M // 2 - 50, M // 2 + 50), torch.arange(M - 100, M)])
    (want, size), _, _ = qk_norm_rope.qk_norm_rope(_np(qkv[at.to(DEV)]), H, G, hd, _np(gain), _np(gain), 1e-6, None, None, False)
    e = (hd / 2 + 12) * 2.0 ** -24
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    _within(_np(q[at.to(DEV)]), want, e * size + half * (np.abs(want) + e * size) + 1e-38, "q")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [4, 300, 900])
def test_one_request_without_starts(dtype, rows):
    """No row table: every row is the one request's, with hidden tokens and own rows."""
    g = torch.Generator().manual_seed(rows)
    s = _batch(g, dtype, (rows,), 300, 2, 40, 1)
    want, spread, size, reach = shared.attention(_np(s["q"]), _np(s["kv"]), s["hidden"].numpy(), s["seg"], _np(s["fresh"]), s["own"], 1 / math.sqrt(40))
    MS.ms_shared_attention(s["q"], s["kv"], s["out"], bits=_bits(s["hidden"]), fresh=s["fresh"], fresh_start=_int(s["own"]))
    _within(_np(s["out"]), want, _attend_bound(want, spread, size, reach, 300 + rows, 40, dtype), "one request")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("total", [40, 1000])
def test_a_replayed_graph_reads_the_tables_anew(dtype, total):
    """Captured once for a padded batch; starts, own rows and hidden tokens change between replays, as requests join and leave."""
    g = torch.Generator().manual_seed(total)
    T = 700
    s = _batch(g, dtype, (total // 2, total // 4, total - total // 2 - total // 4), T, 2, 64, 1)
    seg, own, bits = _int(s["seg"]), _int(s["own"]), _bits(s["hidden"])
    need = MS.ms_shared_attention_workspace_bytes(s["q"], s["kv"], fresh=s["fresh"])
    ws = torch.empty(need + 16, dtype=torch.uint8, device=DEV)

    def call(out):
        MS.ms_shared_attention(s["q"], s["kv"], out, seg_start=seg, bits=bits, fresh=s["fresh"], fresh_start=own, workspace=ws)

    call(s["out"])
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), torch.full_like(s["out"], 7.0)
    with torch.cuda.graph(graph):
        call(out)
    for cut in ([0, total // 3, total // 3, total - 3], [5, 6, 7, 8], [0, 0, 0, 0], [0, total, total, total], [1, 2, total // 2, total]):
        hidden = torch.rand(3, T, generator=g) < 0.3
        seg.copy_(_int(cut))
        own.copy_(_int(cut))
        bits.copy_(_bits(hidden))
        s["q"].copy_(torch.randn(s["q"].shape, generator=g))
        eager = torch.full_like(out, 7.0)
        call(eager)
        torch.cuda.synchronize()
        for _ in range(2):
            out.fill_(7.0)
            ws.fill_(0xff)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
        _check(dict(s, seg=cut, own=cut, hidden=hidden), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_calls_in_flight_together(dtype):
    """Two streams, each with buffers of its own: the same bits as one after the other."""
    g = torch.Generator().manual_seed(5)
    sides = [_batch(g, dtype, rows, 900, 4, 64, 1) for rows in ((300, 20, 90), (5, 700, 200))]
    works = []
    for s in sides:
        need = MS.ms_shared_attention_workspace_bytes(s["q"], s["kv"], fresh=s["fresh"])
        works.append(dict(seg_start=_int(s["seg"]), bits=_bits(s["hidden"]), fresh=s["fresh"], fresh_start=_int(s["own"]),
                          workspace=torch.empty(need + 16, dtype=torch.uint8, device=DEV)))
    for s, k in zip(sides, works):
        MS.ms_shared_attention(s["q"], s["kv"], s["out"], **k)
    torch.cuda.synchronize()
    outs, streams = [torch.full_like(s["out"], 7.0) for s in sides], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(20):
        for s, k, o, stream in zip(sides, works, outs, streams):
            MS.ms_shared_attention(s["q"], s["kv"], o, stream=stream, **k)
    torch.cuda.synchronize()
    assert all(torch.equal(o, s["out"]) for o, s in zip(outs, sides))

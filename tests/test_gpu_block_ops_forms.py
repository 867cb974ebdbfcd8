"""Attention over a shared prefix on the GPU in each of its forms, against the float64 oracle: every width, key ranges, prefix
tiles that whole workgroups skip."""
import math

import pytest
import torch

from oracle import shared
from paper_2505_20600_amd import maskstep as MS
from tests import block_ops_forms as F
from tests.test_gpu_block_ops import DT, DEV, _attend, _attend_bound, _batch, _check, _check_rows, _np, _within

pytestmark = pytest.mark.gpu


def _form(s, ws):
    need = MS.ms_shared_attention_workspace_bytes(s["q"], s["kv"], fresh=s["fresh"])
    return MS.ms_shared_attention_plan(s["q"], s["kv"], fresh=s["fresh"], workspace_bytes={None: 0, "some": need // 2, "need": need}[ws])


def _parts(rows, n):
    """rows packed rows of n requests, one of them empty, ragged."""
    cut = sorted({0, rows, *(rows * i // n + i for i in range(1, n))}) if rows > 4 * n else [0, rows]
    cut = [min(c, rows) for c in cut]
    return [b - a for a, b in zip(cut, cut[1:])][:1] + [0] + [b - a for a, b in zip(cut, cut[1:])][1:]


@pytest.mark.parametrize("dtype,hd,tile,split", [(d, hd, *f) for d in F.HEAD_DIMS for hd in F.HEAD_DIMS[d] for f in F.ATTENTION_FORMS[d]])
def test_every_form_at_every_head_dim(dtype, hd, tile, split):
    rows, G, group, T = F.attention_of(dtype, hd, tile, split)
    g = torch.Generator().manual_seed(hd + tile)
    s = _batch(g, dtype, _parts(rows - 1 if rows > 20 else rows, 7), T, G, hd, group, tail=1 if rows > 20 else 0)
    t, r = _form(s, "need")
    assert t == tile and (r > 1) == split
    _check(s, dtype, *([None, "need", "some"] if split else [None]))


@pytest.mark.parametrize("group", [1, 3, 8])
@pytest.mark.parametrize("own", ["none", "more", "fewer"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_many_slots_with_own_rows_of_any_number(dtype, group, own):
    """Workgroups of 128 slots (in float32 of 16) over requests with no own rows, without query rows, of one row."""
    g = torch.Generator().manual_seed(group)
    rows = [n * 8 // group for n in (30, 0, 1, 64, 17, 12)]
    n = {"none": [0] * 6, "more": [70, 33, 5, 129, 0, 200], "fewer": [0, 0, 1, 3, 2, 0]}[own]
    s = _batch(g, dtype, rows, 260, 2, 40, group, own=n, hide=0.4, lead=3, tail=5)
    assert dtype != "bf16" or _form(s, None)[0] == 128
    _check(s, dtype, None, "need")


def _hidden(kind, B, T, g):
    """Whole runs of 64 tokens hidden, from some requests or all, beside single tokens."""
    h = torch.rand(B, T, generator=g) < 0.1
    if kind == "ends and middle":
        h[:, :320] = h[:, 20 * 64:40 * 64] = h[:, T - T % 64 - 192:] = True
    elif kind == "one tile for one request":
        h[0, 64:128] = True
    elif kind == "all":
        h[:] = True
    elif kind == "all but the last token":
        h[:] = True
        h[:, T - 1] = False
    elif kind == "all but the first token":
        h[:] = True
        h[:, 0] = False
    elif kind == "all but one far in":
        h[:] = True
        h[B - 1, 77 * 64 + 5] = False
    elif kind == "in turn":
        tiles = torch.arange(T) // 64
        for b in range(B):
            h[b] |= tiles % 2 == b % 2
    elif kind == "all from one request":
        h[0] = True
    elif kind == "more than 64 tiles":
        h[:, 64:130 * 64] = True
    return h


KINDS = ["ends and middle", "one tile for one request", "all", "all but the last token", "all but the first token", "all but one far in", "in turn",
         "all from one request", "more than 64 tiles"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [(530, 290), (100,) * 8, (60, 0, 1, 700, 3, 100)], ids=lambda r: f"{len(r)}")
@pytest.mark.parametrize("ws", [None, "some"])
def test_hidden_runs_of_tiles(kind, rows, ws):
    """Prefix tiles that no request of a workgroup sees are left out: first, last, all, one window of 64 tiles and more; with NaN in
    what nobody sees, and the output over the queries."""
    g = torch.Generator().manual_seed(len(rows))
    s = _batch(g, "bf16", rows, 8500, 1, 16, 1)
    t, r = _form(s, ws)
    assert t == 128 and (r > 1) == (ws is not None) and 8500 // 64 // r >= 8
    s["hidden"] = _hidden(kind, len(rows), 8500, g)
    _check(s, "bf16", ws)
    nobody = s["hidden"].all(dim=0)
    bad = dict(s, kv=s["kv"].clone(), q=s["q"].clone())
    bad["kv"][nobody.to(DEV)] = math.nan
    got = _attend(bad, ws).clone()
    _check_rows(bad, "bf16", got, slice(0, sum(rows)))
    onto = _attend(bad, ws, out=bad["q"])
    assert torch.equal(onto, got)


@pytest.mark.parametrize("hd", [64, 72, 128])
def test_hidden_runs_of_tiles_at_other_widths(hd):
    g = torch.Generator().manual_seed(hd)
    s = _batch(g, "bf16", (500, 310), 2000, 1, hd, 1)
    for kind in ("ends and middle", "in turn", "all but the last token"):
        s["hidden"] = _hidden(kind, 2, 2000, g)
        assert _form(s, None)[0] == 128
        _check(s, "bf16", None, "need")


def test_hidden_tiles_of_many_requests():
    """A workgroup's 128 slots go across more requests than tiles are looked up for."""
    g = torch.Generator().manual_seed(1)
    s = _batch(g, "bf16", (8,) * 110, 1300, 1, 32, 1)
    s["hidden"][:, 256:640] = True
    assert _form(s, None)[0] == 128
    _check(s, "bf16", None, "need")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tables_of_many_rows_out_of_range_are_bounded(dtype):
    """Starts that do not ascend or lie outside the rows, in the forms for many slots."""
    g = torch.Generator().manual_seed(2)
    n = 1000
    s = _batch(g, dtype, (300, 400, 300), 900, 8, 64, 1)
    assert dtype != "bf16" or _form(s, None)[0] == 128
    for seg, own in [([0, 700, 300, 1000], s["own"]), ([-5, 100, 1 << 30, 2000], [-7, 400, 1 << 30, 5000]), (s["seg"], [900, 200, 700, 0]),
                     ([500] * 4, s["own"]), ([1000, 600, 200, 0], s["own"])]:
        for ws in (None, "need"):
            s["out"].fill_(7.0)
            got = _attend(dict(s, seg=seg, own=own), ws)
            lo, hi = min(max(seg[0], 0), n), min(max(seg[-1], 0), n)
            assert bool(torch.isfinite(got).all())
            assert bool((got[:lo] == 7.0).all()) and (hi < lo or bool((got[hi:] == 7.0).all()))


@pytest.mark.parametrize("dtype,tile,split", [(d, *f) for d in F.HEAD_DIMS for f in F.ATTENTION_FORMS[d]])
def test_other_requests_nan_in_every_form(dtype, tile, split):
    """NaN in another request's own rows and in tokens that all hide: results are computed again, also onto the queries."""
    g = torch.Generator().manual_seed(3)
    n, G, group, T = F.attention_of(dtype, 64, tile, split)
    a = n // 2
    s = _batch(g, dtype, (a, 1, n - a - 1), T, G, 64, group, hide=0.3)
    s["hidden"][1:] = s["hidden"][0]
    s["kv"][s["hidden"][0].to(DEV)] = math.nan
    s["fresh"][a] = math.nan
    for ws in [None] + ["need"] * split:
        assert _form(s, ws)[0] == tile
        got = _attend(s, ws).clone()
        assert bool(torch.isnan(got[a]).all())
        for rows in (slice(0, a), slice(a + 1, n)):
            _check_rows(s, dtype, got, rows)
        bad = dict(s, q=s["q"].clone())
        onto = _attend(bad, ws, out=bad["q"])
        assert torch.equal(onto[:a], got[:a]) and torch.equal(onto[a + 1:], got[a + 1:]) and bool(torch.isnan(onto[a]).all())

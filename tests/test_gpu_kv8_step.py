"""The denoising step over a K/V cache in 8 bits: resident (shared by requests or not) and streamed, against the oracle's
step over the values that the codes stand for, in the same bounds as the step over a K/V cache of the model's type."""
import ctypes as C

import numpy as np
import pytest
import torch

import oracle
from oracle import kv8
from paper_2505_20600_amd import maskstep as MS
from paper_2505_20600_amd import workloads as W
from tests import gpu_helpers as G

pytestmark = pytest.mark.gpu

SHAPES = [W.ModelShape("k8_fp32", 2, 128, 4, 4, 9, 11, dtype="fp32", batch=2),
          W.ModelShape("k8_hd72", 3, 576, 8, 4, 16, 16, dtype="bf16", batch=2),
          W.ModelShape("k8_text", 2, 256, 4, 4, 13, 16, n_text=9, dtype="bf16", batch=2),
          W.ModelShape("k8_dual", 3, 256, 2, 4, 8, 16, n_text=16, dual_stream=True, dtype="bf16", batch=2)]
BLOCK = 32


def _inputs(shape, cfg):
    """Weights, template, codes and scales per layer ([L][B][N]...), the oracle's K/V of them, final state."""
    ws = W.stack_weights(shape, cfg, random_ln=True, std=0.03)
    xt = W.template_hidden(shape, cfg)
    yc = W.synthetic_y_cache(shape, cfg)
    H, hd, N = shape.n_heads, shape.head_dim, shape.n_image
    codes, scales, kv = [], [], []
    for l in range(shape.n_layers):
        full = np.asarray(W.synthetic_kv_cache(shape, cfg, l), np.float64)
        both = [kv8.quantize(full[b, shape.n_text:].reshape(N, 2, H, hd), BLOCK) for b in range(shape.batch)]
        full[:, :shape.n_text] = np.nan                # text rows are always fresh
        for b, (c, e) in enumerate(both):
            full[b, shape.n_text:] = kv8.values(c, e, BLOCK).reshape(N, 2, shape.d_model)
        codes.append(np.stack([c for c, _ in both]))
        scales.append(np.stack([e for _, e in both]))
        kv.append(full)
    return ws, xt, codes, scales, np.stack(kv), yc


def _masks(shape, ratios, seed):
    return np.stack([W.ellipse_mask(shape.grid_h, shape.grid_w, r, W.rng(seed, 6, b)) if 0 < r < 1 else
                     np.full(shape.n_image, int(r), np.uint8) for b, r in enumerate(ratios)])


class Run:
    """One step context with its device inputs; call() runs the step."""

    def __init__(self, shape, mask, x, codes, scales, yc, ws, *, cache_of=None, pinned=False, n_slots=2, per_request=False,
                 serialize=False, prefix=0):
        self.wc = MS.weights_array(G.dev_weights(ws, shape))
        self.x, self.yc = G.to_dev(x, shape), G.to_dev(yc, shape) if yc is not None else None
        self.step = G.new_step(shape, mask)
        if prefix:
            self.step.set_dense_prefix(prefix)
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(G.DEV)
        pin = lambda a: torch.from_numpy(np.ascontiguousarray(a)).pin_memory()
        self.scales = [dev(s) for s in scales]
        self.kw = dict(block=BLOCK, cache_of=None if cache_of is None else torch.tensor(cache_of, dtype=torch.int32, device=G.DEV))
        self.codes = None
        if pinned:
            of = cache_of or range(shape.batch)
            if per_request:
                self.kw["per_request"] = [[pin(c[s]) if mask[b].any() or shape.n_text else None for b, s in enumerate(of)] for c in codes]
            else:
                self.codes = [pin(np.stack([c[s] for s in of])) for c in codes]
            slot = (shape.batch, shape.n_image, 2, shape.n_heads, shape.head_dim)
            self.slots = [torch.full(slot, 0x7f, dtype=torch.uint8, device=G.DEV) for _ in range(n_slots)]
            self.kw.update(pinned=True, slots=self.slots, copy_stream=None if serialize else torch.cuda.Stream())
        else:
            self.codes = [dev(c) for c in codes]
        self.y = torch.empty((shape.batch, shape.n_tokens, shape.d_model), dtype=G.tdtype(shape), device=G.DEV)

    def call(self, y=None, **kw):
        y = self.y if y is None else y
        self.step.stack_forward_kv8(self.wc, self.x, self.yc, self.codes, self.scales, y, **self.kw, **kw)
        return y

    def out(self):
        self.call()
        torch.cuda.synchronize()
        return G.to_np(self.y)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.name)
def test_step_matches_oracle_resident_and_streamed(shape):
    """Resident, streamed through 1, 2 and n_layers slots, serialized and with per-request buffers: the same bits; the
    unmasked rows of the output are the cached ones, and the caches are as before."""
    ws, xt, codes, scales, kv, yc = _inputs(shape, 81)
    mask = _masks(shape, (0.3, 0.1), 3)
    x = W.edited_hidden(shape, 81, xt, mask)
    ref = oracle.masked_stack(x, mask, kv, yc, ws, shape, round_p=True)
    run = Run(shape, mask, x, codes, scales, yc, ws)
    y = run.out()
    G.assert_close(y, ref, shape.dtype, f"{shape.name} 8-bit cache", blocks=shape.n_layers, inp=x)
    for l in range(shape.n_layers):
        assert np.array_equal(run.codes[l].cpu().numpy(), codes[l]) and np.array_equal(run.scales[l].cpu().numpy(), scales[l])
    yc_b = G.to_np(G.to_dev(yc, shape))
    for b in range(shape.batch):
        keep = np.concatenate([np.zeros(shape.n_text, bool), mask[b] == 0])
        np.testing.assert_array_equal(y[b, keep], yc_b[b, keep])
    for kw in (dict(n_slots=1), dict(n_slots=2), dict(n_slots=shape.n_layers), dict(serialize=True), dict(per_request=True)):
        np.testing.assert_array_equal(Run(shape, mask, x, codes, scales, yc, ws, pinned=True, **kw).out(), y, err_msg=str(kw))


@pytest.mark.parametrize("shape", SHAPES[1:], ids=lambda s: s.name)
def test_requests_share_and_swap_caches(shape):
    """cache_of: both requests on cache 1, and swapped; streamed with the scale tables so numbered."""
    ws, xt, codes, scales, kv, yc = _inputs(shape, 82)
    mask = _masks(shape, (0.2, 0.4), 4)
    x = W.edited_hidden(shape, 82, xt, mask)
    for of in ((1, 1), (1, 0)):
        ref = oracle.masked_stack(x, mask, kv[:, list(of)], yc, ws, shape, round_p=True)
        y = Run(shape, mask, x, codes, scales, yc, ws, cache_of=of).out()
        G.assert_close(y, ref, shape.dtype, f"{shape.name} caches {of}", blocks=shape.n_layers, inp=x)
        np.testing.assert_array_equal(Run(shape, mask, x, codes, scales, yc, ws, cache_of=of, pinned=True).out(), y)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: s.name)
def test_masks_that_leave_nothing(shape):
    """A request with no masked token (streamed: no buffer for it), one with all of them, and a whole batch of each."""
    ws, xt, codes, scales, kv, yc = _inputs(shape, 83)
    for ratios in ((0.0, 0.3), (1.0, 0.2), (0.0, 1.0), (1.0, 1.0), (0.0, 0.0)):
        mask = _masks(shape, ratios, 5)
        x = W.edited_hidden(shape, 83, xt, mask)
        ref = oracle.masked_stack(x, mask, kv, yc, ws, shape, round_p=True)
        y = Run(shape, mask, x, codes, scales, yc, ws).out()
        G.assert_close(y, ref, shape.dtype, f"{shape.name} masks {ratios}", blocks=shape.n_layers, inp=x)
        for kw in (dict(), dict(per_request=True)):
            np.testing.assert_array_equal(Run(shape, mask, x, codes, scales, yc, ws, pinned=True, **kw).out(), y)


@pytest.mark.parametrize("shape", SHAPES[1:], ids=lambda s: s.name)
def test_dense_prefix_and_poisoned_slots(shape, monkeypatch):
    ws, xt, codes, scales, kv, yc = _inputs(shape, 84)
    mask = _masks(shape, (0.3, 0.15), 6)
    x = W.edited_hidden(shape, 84, xt, mask)
    for k in (1, shape.n_layers):
        ref = oracle.masked_stack(x, mask, np.nan_to_num(kv), yc, ws, shape, dense_prefix=k, round_p=True)
        y = Run(shape, mask, x, codes, scales, yc, ws, prefix=k).out()
        G.assert_close(y, ref, shape.dtype, f"{shape.name} prefix {k}", blocks=shape.n_layers, inp=x)
        monkeypatch.setenv("MS_POISON", "1")
        for n in (1, 2):
            np.testing.assert_array_equal(Run(shape, mask, x, codes, scales, yc, ws, prefix=k, pinned=True, n_slots=n).out(), y)
        monkeypatch.delenv("MS_POISON")


@pytest.mark.parametrize("pinned", [False, True], ids=["resident", "streamed"])
def test_step_replays_as_a_graph(pinned):
    """Captured and replayed with eager steps of another context (K/V caching too) between the replays."""
    shape = SHAPES[3]
    ws, xt, codes, scales, kv, yc = _inputs(shape, 85)
    masks = [_masks(shape, r, 7 + i) for i, r in enumerate(((0.3, 0.1), (0.2, 0.5)))]
    runs = [Run(shape, m, W.edited_hidden(shape, 85, xt, m), codes, scales, yc, ws, pinned=pinned) for m in masks]
    want = [r.out() for r in runs]
    graph = torch.cuda.CUDAGraph()
    y = torch.empty_like(runs[0].y)
    with torch.cuda.graph(graph):
        runs[0].call(y)
    torch.cuda.synchronize()
    for i in range(3):
        y.fill_(float("nan"))
        graph.replay()
        np.testing.assert_array_equal(runs[1].out(), want[1])
        G.run_stack(shape, masks[1], W.edited_hidden(shape, 85, xt, masks[1]), np.nan_to_num(kv), yc, ws)
        np.testing.assert_array_equal(G.to_np(y), want[0], err_msg=f"replay {i}")


def test_back_to_back_streamed_steps_with_loads_ahead():
    """Two contexts through the same slots, loads of a step under the one before."""
    shape = SHAPES[1]
    ws, xt, codes, scales, kv, yc = _inputs(shape, 86)
    runs = [Run(shape, m, W.edited_hidden(shape, 86, xt, m), codes, scales, yc, ws, pinned=True, n_slots=3)
            for m in (_masks(shape, (0.3, 0.1), 8), _masks(shape, (0.1, 0.6), 9))]
    want = [r.out() for r in runs]
    runs[1].kw.update(slots=runs[0].slots, copy_stream=runs[0].kw["copy_stream"])
    ys = [torch.empty_like(runs[0].y) for _ in range(6)]
    for i, y in enumerate(ys):
        runs[i % 2].call(y, loads_ahead=i > 0)
    torch.cuda.synchronize()
    for i, y in enumerate(ys):
        np.testing.assert_array_equal(G.to_np(y), want[i % 2], err_msg=f"step {i}")


def test_template_filled_by_the_cache_calls_and_edited():
    """As a program uses it: a dense pass's K/V written into 8-bit caches by ms_kv8_quantize, then the step over them."""
    shape = SHAPES[2]
    ws = W.stack_weights(shape, 87, random_ln=True, std=0.03)
    xt = W.template_hidden(shape, 87)
    yc, kv = oracle.dense_stack(xt, ws, shape, round_p=True)
    H, hd, N = shape.n_heads, shape.head_dim, shape.n_image
    codes, scales, vals = [], [], np.array(kv)
    for l in range(shape.n_layers):
        full = G.to_dev(kv[l], shape).view(shape.batch, shape.n_tokens, 2, H, hd)
        c = torch.empty(shape.batch, N, 2, H, hd, dtype=torch.uint8, device=G.DEV)
        s = torch.empty(shape.batch, -(-N // BLOCK), 2, H, dtype=torch.uint8, device=G.DEV)
        MS.ms_kv8_quantize(full[:, shape.n_text:], c, s, block=BLOCK)
        codes.append(c.cpu().numpy())
        scales.append(s.cpu().numpy())
        for b in range(shape.batch):
            vals[l][b, shape.n_text:] = kv8.values(codes[-1][b], scales[-1][b], BLOCK).reshape(N, 2, shape.d_model)
    mask = _masks(shape, (0.25, 0.1), 10)
    x = W.edited_hidden(shape, 87, xt, mask)
    y = Run(shape, mask, x, codes, scales, yc, ws).out()
    G.assert_close(y, oracle.masked_stack(x, mask, vals, yc, ws, shape, round_p=True), "bf16", "template and edit",
                   blocks=shape.n_layers, inp=x)


def test_refusals():
    shape = SHAPES[1]
    ws, xt, codes, scales, kv, yc = _inputs(shape, 88)
    mask = _masks(shape, (0.3, 0.1), 11)
    run = Run(shape, mask, xt, codes, scales, yc, ws)
    lib = MS.load()
    L = shape.n_layers
    p = (C.c_void_p * L)(*[t.data_ptr() for t in run.codes])
    q = (C.c_void_p * L)(*[t.data_ptr() for t in run.scales])
    pp = lambda a: C.cast(a, C.POINTER(C.c_void_p))
    none = C.POINTER(C.c_void_p)()

    def status(handle=run.step.handle, **kw):
        src = MS.Kv8Source(MS.MS_KV_DEVICE, BLOCK, shape.batch, pp(p), pp(q), None, 0, none, none, 0)
        for k, v in kw.items():
            setattr(src, k, v)
        return lib.mask_stack_forward_kv8(handle, run.wc, run.x.data_ptr(), run.yc.data_ptr(), C.byref(src), run.y.data_ptr(), None, None)
    run.y.fill_(3.0)
    assert status(handle=None) == MS.MS_ESTATE
    for kw, st in ((dict(kind=MS.MS_Y_DEVICE), MS.MS_EINVAL), (dict(kind=9), MS.MS_EINVAL), (dict(scales=none), MS.MS_EINVAL),
                   (dict(scales=pp((C.c_void_p * L)())), MS.MS_EINVAL), (dict(layer=none), MS.MS_EINVAL),
                   (dict(block=0), MS.MS_ESHAPE), (dict(block=48), MS.MS_ESHAPE), (dict(block=256), MS.MS_ESHAPE),
                   (dict(n_caches=0), MS.MS_ESHAPE), (dict(n_caches=1), MS.MS_ESHAPE), (dict(cache_of=run.scales[0].data_ptr() + 2), MS.MS_EALIGN),
                   (dict(kind=MS.MS_KV_HOST_PINNED), MS.MS_EINVAL)):
        assert status(**kw) == st, kw
    assert lib.mask_stack_forward_kv8(run.step.handle, run.wc, run.x.data_ptr(), run.yc.data_ptr(), None, run.y.data_ptr(), None,
                                      None) == MS.MS_EINVAL
    torch.cuda.synchronize()
    assert bool((run.y == 3.0).all())


@pytest.mark.parametrize("block", [1, 32, 128])
def test_more_tokens_than_one_pass_of_the_lists(block, monkeypatch):
    """1600 image tokens and 9 of text: the lists of cached and fresh tokens take several passes; every size of block."""
    monkeypatch.setattr(f"{__name__}.BLOCK", block)
    shape = W.ModelShape("k8_1600", 2, 128, 2, 4, 40, 40, n_text=9, dtype="bf16", batch=2)
    ws, xt, codes, scales, kv, yc = _inputs(shape, 89)
    mask = _masks(shape, (0.5, 0.05), 12)
    x = W.edited_hidden(shape, 89, xt, mask)
    y = Run(shape, mask, x, codes, scales, yc, ws).out()
    G.assert_close(y, oracle.masked_stack(x, mask, kv, yc, ws, shape, round_p=True), "bf16", f"1600 tokens, block {block}",
                   blocks=shape.n_layers, inp=x)
    np.testing.assert_array_equal(Run(shape, mask, x, codes, scales, yc, ws, pinned=True).out(), y)


def test_largest_batch():
    """64 requests with two streams, 128 packed segments, masks of 0 to 100% in turn."""
    shape = W.ModelShape("k8_b64", 1, 128, 2, 4, 8, 8, n_text=5, dual_stream=True, dtype="bf16", batch=64)
    ws, xt, codes, scales, kv, yc = _inputs(shape, 90)
    mask = _masks(shape, [(0.0, 0.1, 0.5, 1.0)[b % 4] for b in range(64)], 13)
    x = W.edited_hidden(shape, 90, xt, mask)
    y = Run(shape, mask, x, codes, scales, yc, ws).out()
    G.assert_close(y, oracle.masked_stack(x, mask, kv, yc, ws, shape, round_p=True), "bf16", "64 requests", blocks=1, inp=x)


def test_a_cache_number_out_of_range_is_no_cache():
    """Its request attends over its own fresh rows; the other one is as it was."""
    shape = SHAPES[2]
    ws, xt, codes, scales, kv, yc = _inputs(shape, 91)
    mask = _masks(shape, (0.3, 0.2), 14)
    x = W.edited_hidden(shape, 91, xt, mask)
    want = Run(shape, mask, x, codes, scales, yc, ws).out()
    for bad in (2, -1, 2 ** 31 - 1):
        y = Run(shape, mask, x, codes, scales, yc, ws, cache_of=(bad, 1)).out()
        np.testing.assert_array_equal(y[1], want[1])
        assert np.isfinite(y[0]).all() and not np.array_equal(y[0], want[0])

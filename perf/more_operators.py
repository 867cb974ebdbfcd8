"""Performance cases of a block's first half over 4-bit weights and a shared template.

Three operators around the attention of a batch of edits of one image template: row products whose operands are
microscaled 4-bit floating point (codes of two bits of exponent and one of mantissa, one power-of-two scale per 32 columns),
the norms of queries and keys for each head with the position rotation and the K/V scatter in the same pass, and attention
of packed query rows over the template's K/V, read once for all requests, less the tokens each request hides, and over the
request's own K/V rows. A case is a dict of sizes; every value is drawn from the seed.

The plain forms below are elementary torch operations in float32; ``exact`` is the definition in float64.
"""
import math

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------


def _codes(name, rows, cols, dtype="bf16"):
    return {"name": name, "op": "codes", "dtype": dtype, "rows": rows, "cols": cols}


def _linear(name, rows, n, k, *, epilogue="bias", dtype="bf16"):
    return {"name": name, "op": "linear", "dtype": dtype, "rows": rows, "n": n, "k": k, "epilogue": epilogue}


def _qk(name, rows, tokens, heads, kv_heads, head_dim, *, rot=0, halves=False, text=0, extra=0, dtype="bf16"):
    """``rows`` image rows at as many of the ``tokens`` positions, after ``text`` rows without a position; ``extra``: columns
    of the projection behind Q, K and V."""
    return {"name": name, "op": "qk", "dtype": dtype, "rows": rows, "tokens": tokens, "heads": heads, "kv_heads": kv_heads,
            "head_dim": head_dim, "rot": rot or head_dim, "halves": halves, "text": text, "extra": extra}


def _attend(name, batch, tokens, kv_heads, head_dim, *, group=1, lo=1, hi=1, text=0, hide=True, dtype="bf16"):
    """lo, hi: edited tokens of the first and the last request, the others spread evenly over their logarithm: rows that are
    queries and own keys, and, with ``hide``, template tokens that the request does not see. ``text`` rows per request are
    queries and own keys too. ``group`` query heads share a K/V head."""
    return {"name": name, "op": "attend", "dtype": dtype, "batch": batch, "tokens": tokens, "kv_heads": kv_heads,
            "head_dim": head_dim, "group": group, "lo": lo, "hi": hi, "text": text, "hide": hide}


def listed():
    return [
        # a weight matrix laid out once: four columns of a width for one, and read back
        _codes("codes_16384x4096", 16384, 4096),
        # one edited token through Q, K and V of a 1152-wide model
        _linear("linear_1x3456x1152", 1, 3456, 1152),
        # the ragged last rows of a batch, a small float32 model
        _linear("linear_77x1000x1056_fp32", 77, 1000, 1056, dtype="fp32"),
        # an ordinary edit of one request, up projection
        _linear("linear_410x4608x1152_gelu", 410, 4608, 1152, epilogue="gelu"),
        # a full batch at the largest width, down projection onto the residual stream
        _linear("linear_8192x4096x16384_resid", 8192, 4096, 16384, epilogue="resid"),
        # a fifth of a 32 x 32 latent, float32, halves rotated
        _qk("qk_205_4x64_fp32", 205, 1024, 4, 4, 64, halves=True, dtype="fp32"),
        # every token of eight templates of a 16 x 72 model
        _qk("qk_32768_16x72", 32768, 32768, 16, 16, 72),
        # a single token in each of eight edits of one template
        _attend("attend_8x1row_12x64", 8, 4096, 12, 64),
        # retouching: 32 requests of a few tokens each
        _attend("attend_32x16rows_16x72", 32, 4096, 16, 72, lo=4, hi=48),
        # eight query heads per K/V head, a template with an odd number of tokens as context that stays whole
        _attend("attend_6x8x128_3001", 6, 3001, 4, 128, group=8, lo=1, hi=33, hide=False),
        # float32: four edits of a 32 x 32 latent
        _attend("attend_4x205rows_4x64_fp32", 4, 1024, 4, 64, lo=103, hi=410, dtype="fp32"),
        # a full serving batch on one template, text rows always recomputed
        _attend("attend_8x4608_16x128", 8, 4096, 16, 128, lo=123, hi=2458, text=512),
    ]


_HEAD_DIMS = (64, 64, 64, 72, 72, 128, 128, 128, 96, 80, 48, 40, 32, 104, 16, 8)


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    most = {}
    for c in listed():
        w = work(c)
        most[c["op"]] = tuple(max(a, b) for a, b in zip(most.get(c["op"], (0, 0)), (w["flops"], w["bytes"])))
    while True:
        op = rng.choice(("codes", "linear", "linear", "linear", "qk", "qk", "attend", "attend", "attend", "attend"))
        dtype = "fp32" if rng.random() < 0.15 else "bf16"
        hd = rng.choice((16, 32, 40, 64, 64)) if dtype == "fp32" else rng.choice(_HEAD_DIMS)
        heads = int(_log_uniform(rng, 2, 33))
        if op == "codes":
            c = _codes("", int(_log_uniform(rng, 1, 16385)), 32 * int(_log_uniform(rng, 1, 257)), dtype)
        elif op == "linear":
            c = _linear("", int(_log_uniform(rng, 1, 8193)), 4 * int(_log_uniform(rng, 16, 4097)), 32 * int(_log_uniform(rng, 2, 513)),
                        epilogue=rng.choice(("bias", "resid", "gelu")), dtype=dtype)
        elif op == "qk":
            tokens = int(_log_uniform(rng, 16, 32769))
            rot = hd if rng.random() < 0.6 else 2 * rng.randint(1, hd // 2)
            c = _qk("", max(1, int(tokens * _log_uniform(rng, 0.01, 1.0))), tokens, heads, heads if rng.random() < 0.7 else 1, hd,
                    rot=rot, halves=rng.random() < 0.5, text=rng.choice((0, 0, rng.randint(1, 512))),
                    extra=rng.choice((0, 0, 8 * rng.randint(1, 512))), dtype=dtype)
        else:
            group = rng.choice((1, 1, 1, 1, 2, 4, 8))
            tokens = int(_log_uniform(rng, 64, 5000))
            batch = int(_log_uniform(rng, 1, 41))
            few = rng.random() < 0.5
            hi = max(1, min(tokens, int(_log_uniform(rng, 1, 64) if few else tokens * _log_uniform(rng, 0.02, 1.0))))
            lo = hi if batch == 1 else max(1, int(hi / _log_uniform(rng, 1, 8)))
            c = _attend("", batch, tokens, max(1, heads // group), hd, group=group, lo=lo, hi=hi,
                        text=rng.choice((0, 0, rng.randint(1, 512))) if not few else 0, hide=rng.random() < 0.8, dtype=dtype)
        del c["name"]
        w = work(c)
        if "head_dim" in c and max(c.get("heads", 0), c["kv_heads"] * c.get("group", 1)) * hd > 4096:
            continue
        if w["flops"] > most[op][0] or w["bytes"] > most[op][1] or (dtype == "fp32" and op == "attend" and w["flops"] > most[op][0] / 16):
            continue
        return c


def _edited(case):
    """Edited tokens of each request."""
    B = case["batch"]
    return [min(case["tokens"], max(1, round(case["lo"] * (case["hi"] / case["lo"]) ** (b / (B - 1) if B > 1 else 0.0)))) for b in range(B)]


def work(case):
    """Every input and every result once. Attention: the template's K/V once for all requests, the two products over every
    (query row, key that its request sees)."""
    e = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "codes":
        n = case["rows"] * case["cols"]
        return {"bytes": n * 2 * e + 2 * (n // 2 + n // 32), "flops": 4 * n}
    if case["op"] == "linear":
        m, n, k = case["rows"], case["n"], case["k"]
        return {"bytes": m * k * e + n * (k // 2 + k // 32) + n * e + m * n * e * (2 if case["epilogue"] == "resid" else 1), "flops": 2 * m * n * k}
    if case["op"] == "qk":
        rows, hd = case["rows"] + case["text"], case["head_dim"]
        cols = (case["heads"] + 2 * case["kv_heads"]) * hd
        return {"bytes": rows * (2 * cols * e + 8) + case["rows"] * case["rot"] * 4 + 2 * hd * e, "flops": rows * cols * 7}
    dkv, T = case["kv_heads"] * case["head_dim"], case["tokens"]
    d, n = dkv * case["group"], _edited(case)
    rows = [x + case["text"] for x in n]
    keys = [T - (n[b] if case["hide"] else 0) + rows[b] for b in range(len(n))]
    return {"bytes": 2 * sum(rows) * d * e + (T + sum(rows)) * 2 * dkv * e + (len(n) * T // 8 if case["hide"] else 0),
            "flops": 4 * d * sum(r * k for r, k in zip(rows, keys))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------


def _runs(tokens, n, g):
    """n token numbers, ascending: one to four runs of neighbours, as an edited region's rows are, at random places."""
    pieces = min(4, n)
    at = torch.randint(0, tokens, (pieces,), generator=g, device=DEV)
    near = (torch.arange(tokens, device=DEV)[None] - at[:, None]).abs().min(0).values
    return near.argsort(stable=True)[:n].sort().values


def _acts(rows, cols, dt, g):
    """Normalised activations: columns of different widths, a few of them far wider than the others."""
    x = torch.randn(rows, cols, generator=g, device=DEV)
    x *= torch.exp(0.4 * torch.randn(cols, generator=g, device=DEV))
    x *= torch.where(torch.rand(cols, generator=g, device=DEV) < 0.01, 8.0, 1.0)
    return x.to(dt)


def _kv(rows, heads, hd, dt, g):
    """K/V rows [rows][2][heads][hd] as a projection of normalised activations gives them: channels of different widths."""
    x = torch.randn(rows, 2, heads, hd, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(2, heads, hd, generator=g, device=DEV))
    return x.to(dt)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 29)
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    s = {"case": case}
    if case["op"] == "codes":
        s["x"] = _acts(case["rows"], case["cols"], dt, g) * (0.02 if case["rows"] > case["cols"] else 1.0)
        s["codes"] = torch.zeros(case["rows"], case["cols"] // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.zeros(case["rows"], case["cols"] // 32, dtype=torch.uint8, device=DEV)
        s["values"] = torch.zeros_like(s["x"])
        return s
    if case["op"] == "linear":
        m, n, k = case["rows"], case["n"], case["k"]
        s["x"] = _acts(m, k, dt, g)
        w = torch.randn(n, k, generator=g, device=DEV) / math.sqrt(k)
        y, ex = _mx4(w)
        s["w_codes"], s["w_scales"] = _pack(y), (ex + 127).to(torch.uint8)
        s["bias"] = (0.1 * torch.randn(n, generator=g, device=DEV)).to(dt)
        s["resid"] = torch.randn(m, n, generator=g, device=DEV).to(dt) if case["epilogue"] == "resid" else None
        s["codes"] = torch.zeros(m, k // 2, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.zeros(m, k // 32, dtype=torch.uint8, device=DEV)
        s["out"] = torch.zeros(m, n, dtype=dt, device=DEV)
        if own:
            from paper_2505_20600_amd import maskstep as MS
            s["workspace"] = torch.empty(max(16, MS.ms_mx4_linear_workspace_bytes(s["codes"], s["w_codes"])), dtype=torch.uint8, device=DEV)
        return s
    if case["op"] == "qk":
        M, T, H, G, hd = case["rows"] + case["text"], case["tokens"], case["heads"], case["kv_heads"], case["head_dim"]
        cols = (H + 2 * G) * hd
        wide = _acts(M, cols + case["extra"], dt, g)
        s["qkv"] = wide[:, :cols]
        s["q_gain"] = (1.0 + 0.2 * torch.randn(hd, generator=g, device=DEV)).to(dt)
        s["k_gain"] = (1.0 + 0.2 * torch.randn(hd, generator=g, device=DEV)).to(dt)
        # one angle per pair: the frequencies of a base of 10000 over the rotated columns
        freq = torch.exp(torch.arange(case["rot"] // 2, dtype=torch.float64, device=DEV) * (-2.0 * math.log(1e4) / case["rot"]))
        angle = torch.arange(T, dtype=torch.float64, device=DEV)[:, None] * freq
        s["table"] = torch.stack([angle.cos(), angle.sin()], dim=2).float().contiguous()
        at = _runs(T, case["rows"], g)
        s["pos"] = torch.cat([torch.full((case["text"],), -1, device=DEV), at]).int()
        s["rows"] = torch.cat([torch.arange(case["text"], device=DEV), case["text"] + at]).int()
        s["kv"] = _kv(case["text"] + T, G, hd, dt, g)
        s["q"] = torch.zeros(M, H, hd, dtype=dt, device=DEV)
        return s
    B, T, G, hd = case["batch"], case["tokens"], case["kv_heads"], case["head_dim"]
    n = _edited(case)
    rows = [x + case["text"] for x in n]
    s["starts"] = [sum(rows[:b]) for b in range(B + 1)]
    s["seg_start"] = torch.tensor(s["starts"], dtype=torch.int32, device=DEV)
    s["template"] = _kv(T, G, hd, dt, g)
    s["fresh"] = _kv(sum(rows), G, hd, dt, g)
    s["q"] = (1.5 * torch.randn(sum(rows), G * case["group"], hd, generator=g, device=DEV)).to(dt)
    s["out"] = torch.zeros_like(s["q"])
    s["hidden"] = None
    if case["hide"]:
        s["hidden"] = torch.zeros(B, T, dtype=torch.uint8, device=DEV)
        for b in range(B):
            s["hidden"][b, _runs(T, n[b], g)] = 1
    if own:
        from paper_2505_20600_amd import maskstep as MS
        # constant over a request's steps and layers, as its mask is
        s["bits"] = None
        if case["hide"]:
            s["bits"] = torch.empty(B, -(-T // 64), dtype=torch.int64, device=DEV)
            MS.ms_shared_bits(s["hidden"], s["bits"])
        need = MS.ms_shared_attention_workspace_bytes(s["q"], s["template"], fresh=s["fresh"])
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------


def _mx4(x):
    """(codes' values [rows][cols] before scaling, exponents [rows][cols / 32] of the scales) of x [rows][cols]."""
    v = x.float().view(x.shape[0], -1, 32)
    a = v.abs().amax(dim=2)
    m, x2 = torch.frexp(a)                                  # a = m 2^x2, 1/2 <= m < 1
    ex = torch.where(m > 0.875, x2 - 2, x2 - 3)             # smallest with a <= 7 2^ex
    ex = torch.where(a == 0, torch.zeros_like(ex), ex.clamp(-126, 125))
    y = torch.ldexp(v, -ex[:, :, None])
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y)[1].clamp(min=1) - 2)    # one bit below the leading one
    y = (torch.round(y / step) * step).clamp(-6.0, 6.0)
    return y.view(x.shape), ex


def _pack(y):
    """Codes of values 0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives, two per byte, the first in the low half."""
    a = y.abs()
    c = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    c = torch.where(torch.signbit(y), c + 8, c)
    return c[:, 0::2] | (c[:, 1::2] << 4)


def _unpack(codes, exps):
    """float32 values of codes [rows][cols / 2] with exponent bytes [rows][cols / 32]."""
    c = torch.stack([codes & 15, codes >> 4], dim=2).view(codes.shape[0], -1).long()
    grid = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=DEV)
    y = torch.cat([grid, -grid])[c].view(codes.shape[0], -1, 32)
    return torch.ldexp(y, exps.int()[:, :, None] - 127).view(codes.shape[0], -1)


def _gelu(x):
    return x * 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _rotate(x, gain, s):
    """x [rows][heads][hd], normalised by its head's root mean square and rotated by its row's position."""
    case = s["case"]
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(dim=2, keepdim=True) + EPS) * gain.float()
    there = (s["pos"] >= 0) & (s["pos"] < case["tokens"])
    cs = s["table"][s["pos"].clamp(0, case["tokens"] - 1).long()]
    cos = torch.where(there[:, None], cs[:, :, 0], torch.ones_like(cs[:, :, 0]))[:, None]
    sin = torch.where(there[:, None], cs[:, :, 1], torch.zeros_like(cs[:, :, 1]))[:, None]
    rot = case["rot"]
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if case["halves"] else (x[..., 0:rot:2], x[..., 1:rot:2])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.cat(y, dim=2) if case["halves"] else torch.stack(y, dim=3).flatten(2)
    return torch.cat([y, x[..., rot:]], dim=2)


def _plain(s):
    case = s["case"]
    if case["op"] == "codes":
        y, ex = _mx4(s["x"])
        v = torch.ldexp(y.view(y.shape[0], -1, 32), ex[:, :, None]).view(y.shape)
        return v.to(s["x"].dtype), (ex + 127).to(torch.uint8)
    if case["op"] == "linear":
        y, ex = _mx4(s["x"])
        x = torch.ldexp(y.view(y.shape[0], -1, 32), ex[:, :, None]).view(y.shape)
        z = x @ _unpack(s["w_codes"], s["w_scales"]).t() + s["bias"].float()
        if case["epilogue"] == "gelu":
            z = _gelu(z)
        if case["epilogue"] == "resid":
            z = z + s["resid"].float()
        return z.to(s["out"].dtype)
    if case["op"] == "qk":
        H, G, hd = case["heads"], case["kv_heads"], case["head_dim"]
        x = s["qkv"].view(s["qkv"].shape[0], H + 2 * G, hd)
        s["q"] = _rotate(x[:, :H], s["q_gain"], s).to(s["q"].dtype)
        k = _rotate(x[:, H:H + G], s["k_gain"], s).to(s["q"].dtype)
        s["kv"][s["rows"].long()] = torch.stack([k, x[:, H + G:]], dim=1)
        return s["q"], s["kv"]
    # requests padded to the longest one's rows: [request and K/V head][query row and head of its group][key]
    B, T, G, hd, group = (case[k] for k in ("batch", "tokens", "kv_heads", "head_dim", "group"))
    start = s["seg_start"].long()
    count = start[1:] - start[:-1]
    R = max(b - a for a, b in zip(s["starts"], s["starts"][1:]))
    at = torch.arange(R, device=DEV)[None]
    there = at < count[:, None]
    row = torch.where(there, start[:-1, None] + at, torch.zeros_like(at))
    q = s["q"].float()[row].view(B, R, G, group, hd).permute(0, 2, 1, 3, 4).reshape(B * G, R * group, hd)
    own_kv = s["fresh"].float()[row].permute(0, 2, 3, 1, 4)                       # [B][2][G][R][hd]
    kv = s["template"].float().permute(1, 2, 0, 3)[None].expand(B, 2, G, T, hd)
    kv = torch.cat([kv, own_kv], dim=3)
    k, v = (kv[:, i].reshape(B * G, T + R, hd).contiguous() for i in range(2))
    p = torch.bmm(q.contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(hd)
    sees = torch.ones(B, T, dtype=torch.bool, device=DEV) if s["hidden"] is None else s["hidden"] == 0
    sees = torch.cat([sees, there], dim=1).repeat_interleave(G, 0)[:, None]
    p = torch.where(sees, p, torch.full_like(p, -math.inf))
    p = torch.exp(p - p.amax(2, keepdim=True))
    o = torch.bmm(p, v) / p.sum(2, keepdim=True)
    o = o.view(B, G, R, group, hd).permute(0, 2, 1, 3, 4).reshape(B, R, G * group, hd)
    s["out"][row[there]] = o[there].to(s["out"].dtype)
    return s["out"]


def _own(s):
    from paper_2505_20600_amd import maskstep as MS
    case = s["case"]
    if case["op"] == "codes":
        MS.ms_mx4_quantize(s["x"], s["codes"], s["scales"])
        MS.ms_mx4_dequantize(s["codes"], s["scales"], s["values"])
        return s["values"], s["scales"]
    if case["op"] == "linear":
        MS.ms_mx4_quantize(s["x"], s["codes"], s["scales"])
        MS.ms_mx4_linear(s["codes"], s["scales"], s["w_codes"], s["w_scales"], s["bias"], s["out"], resid=s["resid"],
                         gelu=case["epilogue"] == "gelu", workspace=s["workspace"])
        return s["out"]
    if case["op"] == "qk":
        MS.ms_qk_norm_rope(s["qkv"], s["q"], s["kv"], q_gain=s["q_gain"], k_gain=s["k_gain"], eps=EPS, table=s["table"], pos=s["pos"],
                           halves=case["halves"], rows=s["rows"])
        return s["q"], s["kv"]
    MS.ms_shared_attention(s["q"], s["template"], s["out"], seg_start=s["seg_start"], bits=s["bits"], fresh=s["fresh"],
                           fresh_start=s["seg_start"], workspace=s["workspace"])
    return s["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------

_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact_mx4(x):
    """Nearest code's value of every element by search, ties to the even code, at the smallest power of two that a block's
    largest is at most seven times of (2^-126 to 2^125; 1 for a block of zeros), and that power's exponent byte."""
    grid = torch.tensor(_GRID, dtype=torch.float64, device=DEV)
    mid = (grid[1:] + grid[:-1]) / 2
    out, exps = torch.empty(x.shape, dtype=torch.float64, device=DEV), []
    for r in range(0, x.shape[0], 2048):
        v = x[r:r + 2048].double().view(-1, x.shape[1] // 32, 32)
        a = v.abs().amax(dim=2)
        ex = torch.where(a > 0, torch.ceil(torch.log2(a / 7.0)), torch.zeros_like(a))
        ex = torch.where(a > 7.0 * torch.exp2(ex), ex + 1, ex)                  # the logarithm's own rounding
        ex = torch.where((a > 0) & (a <= 7.0 * torch.exp2(ex - 1)), ex - 1, ex).clamp(-126.0, 125.0)
        y = v / torch.exp2(ex)[:, :, None]
        down = torch.searchsorted(mid, y.abs().contiguous())                     # a midpoint goes down here
        up = torch.searchsorted(mid, y.abs().contiguous(), right=True)
        at = torch.where(down % 2 == 0, down, up)
        out[r:r + 2048] = (grid[at] * y.sign() * torch.exp2(ex)[:, :, None]).view(-1, x.shape[1])
        exps.append((ex + 127).to(torch.uint8))
    return out, torch.cat(exps)


def _exact_rotate(x, gain, s):
    case = s["case"]
    rot, x = case["rot"], x.double()
    x = x / torch.sqrt(x.square().mean(dim=2, keepdim=True) + EPS) * gain.double()
    out = x.clone()
    half = rot // 2
    first = torch.arange(half, device=DEV) if case["halves"] else 2 * torch.arange(half, device=DEV)
    second = first + (half if case["halves"] else 1)
    hit = (s["pos"] >= 0).nonzero().flatten()
    turn = torch.view_as_complex(s["table"][s["pos"][hit].long()].double())[:, None]
    z = torch.complex(x[hit][:, :, first], x[hit][:, :, second]) * turn
    part = out[hit]
    part[:, :, first], part[:, :, second] = z.real, z.imag
    out[hit] = part
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "codes":
        return _exact_mx4(s["x"])
    if case["op"] == "linear":
        x = _exact_mx4(s["x"])[0]
        out = torch.empty(case["rows"], case["n"], dtype=torch.float64, device=DEV)
        grid = torch.tensor(_GRID, dtype=torch.float64, device=DEV)
        for n in range(0, case["n"], 1024):
            c = s["w_codes"][n:n + 1024].long()
            w = torch.empty(c.shape[0], case["k"], dtype=torch.float64, device=DEV)
            w[:, 0::2], w[:, 1::2] = (grid[h % 8] * (1 - 2 * (h // 8)) for h in (c % 16, c // 16))
            w *= torch.exp2(s["w_scales"][n:n + 1024].double() - 127.0).repeat_interleave(32, 1)
            z = x @ w.t().contiguous() + s["bias"][n:n + 1024].double()
            if case["epilogue"] == "gelu":
                z = z * torch.special.ndtr(z)
            out[:, n:n + 1024] = z
        return out + s["resid"].double() if s["resid"] is not None else out
    if case["op"] == "qk":
        H, G, hd = case["heads"], case["kv_heads"], case["head_dim"]
        x = s["qkv"].reshape(-1, H + 2 * G, hd)
        kv = s["kv"].double()
        kv[s["rows"].long(), 0] = _exact_rotate(x[:, H:H + G], s["k_gain"], s)
        kv[s["rows"].long(), 1] = x[:, H + G:].double()
        return _exact_rotate(x[:, :H], s["q_gain"], s), kv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        r0, r1 = s["starts"][b], s["starts"][b + 1]
        seen = torch.arange(case["tokens"], device=DEV) if s["hidden"] is None else (s["hidden"][b] == 0).nonzero().flatten()
        kv = torch.cat([s["template"][seen], s["fresh"][r0:r1]]).double()
        for h in range(case["kv_heads"] * case["group"]):
            g = h // case["group"]
            z = s["q"][r0:r1, h].double() @ kv[:, 0, g].t().contiguous() / math.sqrt(case["head_dim"])
            out[r0:r1, h] = torch.softmax(z, dim=1) @ kv[:, 1, g].contiguous()
    return out

"""Performance cases of the 8-bit K/V cache operators.

The cached keys and values of an image template, held as e4m3 codes with one power-of-two scale per block of tokens, K or
V, and head: writing K/V rows into such a cache (a whole template, or only the rows that an edit recomputed), reading the
rows of listed tokens back, and attention of a batch's packed query rows over the listed cached tokens and the fresh K/V
rows. A case is a dict of sizes; every value is drawn from the seed.

The plain forms below are elementary torch operations in float32; ``exact`` is the definition in float64.
"""
import math

import torch

own = False

DEV = "cuda:0"


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------


def _case(name, op, caches, tokens, kv_heads, head_dim, *, dtype="bf16", block=64, group=1, batch=0, lo=0, hi=0, text=0,
          fresh=True):
    """lo, hi: edited tokens of the first and the last request, the others spread evenly over their logarithm. ``group``
    query heads share a K/V head; ``text`` rows per request are queries and fresh keys that no cache holds; without
    ``fresh`` the queries read cached tokens only."""
    return {"name": name, "op": op, "dtype": dtype, "caches": caches, "tokens": tokens, "kv_heads": kv_heads,
            "head_dim": head_dim, "block": block, "group": group, "batch": batch or caches, "lo": lo, "hi": hi, "text": text,
            "fresh": fresh}


def listed():
    return [
        # a float32 model's template on a 32 x 32 latent: the smallest cache, bound by latency
        _case("write_1024_4x64_fp32", "write", 1, 1024, 4, 64, dtype="fp32", block=32),
        # one layer of eight templates of a 16 x 72 model: what filling the cache costs beside the template's own pass
        _case("write_8x4096_16x72", "write", 8, 4096, 16, 72),
        # an edit becomes the next template: a tenth of the tokens rewritten in place
        _case("rewrite_4096_16x72", "rewrite", 1, 4096, 16, 72, lo=410, hi=410),
        # one request's unmasked tokens back into its working K/V
        _case("read_4096_12x64", "read", 1, 4096, 12, 64, lo=819, hi=819),
        # a serving batch of the largest model, four requests
        _case("read_4x4096_24x128", "read", 4, 4096, 24, 128, lo=410, hi=1638),
        # a single token: one query row over a whole template
        _case("attend_1row_12x64", "attention", 1, 4096, 12, 64, lo=1, hi=1),
        # retouching: eight requests of a few tokens each
        _case("attend_8x16rows_16x72", "attention", 8, 4096, 16, 72, lo=4, hi=48),
        # eight query heads per K/V head, six requests on two shared templates with an odd number of tokens
        _case("attend_shared_4x8x128", "attention", 2, 3001, 4, 128, group=8, batch=6, lo=1, hi=33, block=32),
        # float32: a fifth of a 32 x 32 latent
        _case("attend_205rows_4x64_fp32", "attention", 1, 1024, 4, 64, dtype="fp32", lo=205, hi=205, block=32),
        # an ordinary edit of one request
        _case("attend_410rows_16x72", "attention", 1, 4096, 16, 72, lo=410, hi=410),
        # a full serving batch, masks as different as traffic brings
        _case("attend_8x4096_16x72", "attention", 8, 4096, 16, 72, lo=123, hi=2458),
        # the largest model, text rows always recomputed
        _case("attend_4x4608_24x128", "attention", 4, 4096, 24, 128, lo=410, hi=1638, text=512),
    ]


_HEAD_DIMS = (64, 64, 64, 72, 72, 128, 128, 128, 96, 80, 48, 40, 32, 104, 16, 8)


def _log_uniform(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    every = [work(c) for c in listed()]
    most_flops, most_bytes = max(w["flops"] for w in every), max(w["bytes"] for w in every)
    while True:
        op = rng.choice(("write", "rewrite", "read", "attention", "attention", "attention", "attention"))
        dtype = "fp32" if rng.random() < 0.15 else "bf16"
        hd = rng.choice((16, 32, 40, 64, 64)) if dtype == "fp32" else rng.choice(_HEAD_DIMS)
        group = rng.choice((1, 1, 1, 1, 2, 4, 8)) if op == "attention" else 1
        kv_heads = max(1, int(_log_uniform(rng, 2, 33)) // (group if group < 8 else 4))
        tokens = int(_log_uniform(rng, 64, 5000))
        caches = int(_log_uniform(rng, 1, 9))
        batch = caches if rng.random() < 0.7 else max(1, int(_log_uniform(rng, 1, 17)))
        few = rng.random() < 0.4
        hi = max(1, min(tokens, int(_log_uniform(rng, 1, 64) if few else tokens * _log_uniform(rng, 0.02, 1.0))))
        lo = hi if batch == 1 else max(1, int(hi / _log_uniform(rng, 1, 8)))
        if op != "attention":
            batch = caches
        text = rng.choice((0, 0, 0, rng.randint(1, 512))) if op == "attention" and not few else 0
        c = _case("", op, caches, tokens, kv_heads, hd, dtype=dtype, block=rng.choice((1, 16, 32, 64, 64, 128)), group=group,
                  batch=batch, lo=lo, hi=hi, text=text, fresh=text > 0 or rng.random() < 0.85)
        del c["name"]
        w = work(c)
        if kv_heads * hd * group > 4096 or w["flops"] > most_flops or w["bytes"] > most_bytes:
            continue
        return c


def _edited(case):
    """Edited tokens of each request."""
    B = case["batch"]
    return [min(case["tokens"], max(0, round(case["lo"] * (case["hi"] / case["lo"]) ** (b / (B - 1) if B > 1 else 0.0))))
            if case["hi"] else 0 for b in range(B)]


def work(case):
    """K/V rows, codes and scales that the path reads or writes, once each; a template that several requests share is read
    once. Attention: the two products over every (query row, key)."""
    e = 4 if case["dtype"] == "fp32" else 2
    dkv, T, S, B = case["kv_heads"] * case["head_dim"], case["tokens"], case["caches"], case["batch"]
    n = _edited(case)
    scales = 2 * case["kv_heads"] * -(-T // case["block"])
    if case["op"] == "write":
        return {"bytes": S * (T * 2 * dkv * (e + 1) + scales), "flops": 4 * S * T * 2 * dkv}
    if case["op"] == "rewrite":
        touched = min(T, 2 * case["block"] + n[0] * 2)   # at least the rewritten rows' blocks, which lie in runs
        return {"bytes": S * (n[0] * 2 * dkv * (e + 1) + touched * 2 * dkv), "flops": 4 * S * touched * 2 * dkv}
    if case["op"] == "read":
        return {"bytes": sum((T - n[b]) * 2 * dkv * (e + 1) for b in range(B)) + S * scales, "flops": sum((T - n[b]) * 2 * dkv for b in range(B))}
    d = dkv * case["group"]
    cached = min(S, B) * T if S != B else sum(T - n[b] for b in range(B))
    rows = [n[b] + case["text"] for b in range(B)]
    keys = [T - n[b] + (rows[b] if case["fresh"] else 0) for b in range(B)]
    return {"bytes": 2 * sum(rows) * d * e + cached * 2 * dkv + min(S, B) * scales + (sum(rows) * 2 * dkv * e if case["fresh"] else 0),
            "flops": 4 * d * sum(r * k for r, k in zip(rows, keys))}


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------


def _runs(tokens, n, g):
    """n token numbers, ascending: one to four runs of neighbours, as an edited region's rows are, at random places."""
    if n == 0:
        return torch.zeros(0, dtype=torch.int64, device=DEV)
    pieces = min(4, n)
    at = torch.randint(0, tokens, (pieces,), generator=g, device=DEV)
    score = torch.arange(tokens, device=DEV)
    near = torch.stack([(score - a).abs() for a in at]).min(0).values
    return near.argsort(stable=True)[:n].sort().values


def _kv(rows, case, g):
    """K/V rows [rows][2][heads][hd] as a projection of normalised activations gives them: channels of different widths."""
    H, hd = case["kv_heads"], case["head_dim"]
    x = torch.randn(rows, 2, H, hd, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(2, H, hd, generator=g, device=DEV))
    return x.to(torch.float32 if case["dtype"] == "fp32" else torch.bfloat16)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 7919 + 13)
    S, T, H, hd, B = (case[k] for k in ("caches", "tokens", "kv_heads", "head_dim", "batch"))
    dt = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    s = {"case": case}
    template = _kv(S * T, case, g).view(S, T, 2, H, hd)
    n = _edited(case)
    if case["op"] == "write":
        s["kv"] = template
        s["codes"] = torch.zeros(S, T, 2, H, hd, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.zeros(S, -(-T // case["block"]), 2, H, dtype=torch.uint8, device=DEV)
        return s
    codes, exps = _quantize(template, case["block"])
    s["codes"], s["scales"] = codes.view(torch.uint8), exps
    del template
    if case["op"] == "rewrite":
        # the edit's K/V rows, packed, and for every token its row or -1
        tokens = [_runs(T, n[b], g) for b in range(S)]
        s["kv"] = 1.2 * _kv(sum(n), case, g)
        s["src_row"] = torch.full((S, T), -1, dtype=torch.int32, device=DEV)
        at = 0
        for b in range(S):
            s["src_row"][b, tokens[b]] = torch.arange(at, at + n[b], dtype=torch.int32, device=DEV)
            at += n[b]
        return s
    # the unmasked tokens of each request
    edited = [_runs(T, n[b], g) for b in range(B)]
    s["keys"] = torch.zeros(B, T, dtype=torch.int32, device=DEV)
    for b in range(B):
        left = torch.ones(T, dtype=torch.bool, device=DEV)
        left[edited[b]] = False
        s["keys"][b, :T - n[b]] = left.nonzero().flatten().int()
    s["counts"] = [T - n[b] for b in range(B)]
    s["n_keys"] = torch.tensor(s["counts"], dtype=torch.int32, device=DEV)
    if case["op"] == "read":
        s["kv"] = _kv(B * T, case, g).view(B, T, 2, H, hd)
        return s
    rows = [n[b] + case["text"] for b in range(B)]
    s["starts"] = [sum(rows[:b]) for b in range(B + 1)]
    s["seg_start"] = torch.tensor(s["starts"], dtype=torch.int32, device=DEV)
    s["q"] = (1.5 * torch.randn(sum(rows), H * case["group"], hd, generator=g, device=DEV)).to(dt)
    s["fresh"] = _kv(sum(rows), case, g) if case["fresh"] else None
    s["of"] = [b % S for b in range(B)]
    s["cache_of"] = torch.tensor(s["of"], dtype=torch.int32, device=DEV) if S != B else None
    s["out"] = torch.zeros_like(s["q"])
    if own:
        from paper_2505_20600_amd import maskstep as MS
        need = MS.ms_kv8_attention_workspace_bytes(s["q"], s["codes"], s["seg_start"], fresh=s["fresh"])
        s["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------


def _quantize(x, block):
    """(codes [S][T][2][H][hd] as float8_e4m3fn, exponent bytes [S][blocks][2][H]) of x [S][T][2][H][hd]."""
    S, T, _, H, hd = x.shape
    nb = -(-T // block)
    v = torch.zeros(S, nb * block, 2, H, hd, dtype=torch.float32, device=x.device)
    v[:, :T] = x
    v = v.view(S, nb, block, 2, H, hd)
    a = v.abs().amax(dim=(2, 5))
    m, x2 = torch.frexp(a)                                  # a = m 2^x2, 1/2 <= m < 1
    ex = torch.where(m > 0.875, x2 - 8, x2 - 9)             # smallest with a <= 448 2^ex
    ex = torch.where(a == 0, torch.zeros_like(ex), ex.clamp(min=-126))
    y = torch.ldexp(v, -ex[:, :, None, :, :, None])
    step = torch.ldexp(torch.ones_like(y), torch.frexp(y)[1].clamp(min=-5) - 4)    # 3 bits below the leading one
    y = torch.round(y / step) * step
    return y.view(S, nb * block, 2, H, hd)[:, :T].to(torch.float8_e4m3fn), (ex + 127).to(torch.uint8)


def _values(codes, exps, block):
    """float32 values of codes [T][2][H][hd] (uint8) with exponent bytes [blocks][2][H]."""
    T = codes.shape[0]
    s = torch.exp2(exps.float() - 127.0).repeat_interleave(block, 0)[:T]
    return codes.view(torch.float8_e4m3fn).float() * s[..., None]


def _touched(src, block):
    """Blocks of tokens with a rewritten one, from the tokens' rows (-1: kept)."""
    pad = torch.full((-src.numel() % block,), -1, dtype=src.dtype, device=src.device)
    return (torch.cat([src, pad]).view(-1, block) >= 0).any(1)


def _plain(s):
    case = s["case"]
    block = case["block"]
    if case["op"] == "write":
        return _quantize(s["kv"], block)
    if case["op"] == "rewrite":
        out = []
        for b in range(case["caches"]):
            v = _values(s["codes"][b], s["scales"][b], block)
            src = s["src_row"][b].long()
            v = torch.where((src >= 0)[:, None, None, None], s["kv"].float()[src.clamp(min=0)], v)
            codes, exps = _quantize(v[None], block)
            hit = _touched(src, block)          # the other blocks keep their codes and scales
            exps = torch.where(hit[:, None, None], exps[0], s["scales"][b])
            hit = hit.repeat_interleave(block)[:src.numel(), None, None, None]
            out.append((torch.where(hit, codes[0].view(torch.uint8), s["codes"][b]), exps))
        return torch.stack([c for c, _ in out]).view(torch.float8_e4m3fn), torch.stack([e for _, e in out])
    if case["op"] == "read":
        for b in range(case["batch"]):
            k = s["keys"][b, :s["counts"][b]].long()
            s["kv"][b, k] = _values(s["codes"][b], s["scales"][b], block)[k].to(s["kv"].dtype)
        return s["kv"]
    scale = 1.0 / math.sqrt(case["head_dim"])
    for b in range(case["batch"]):
        r0, r1 = s["starts"][b], s["starts"][b + 1]
        k = s["keys"][b, :s["counts"][b]].long()
        kv = _values(s["codes"][s["of"][b]], s["scales"][s["of"][b]], block)[k]
        if s["fresh"] is not None:
            kv = torch.cat([kv, s["fresh"][r0:r1].float()])
        if r1 == r0:
            continue
        if kv.shape[0] == 0:
            s["out"][r0:r1] = 0
            continue
        # [K/V head][query row and head of its group][hd] against [K/V head][key][hd]
        q = s["q"][r0:r1].float().view(r1 - r0, case["kv_heads"], case["group"], case["head_dim"])
        q = q.permute(1, 0, 2, 3).reshape(case["kv_heads"], -1, case["head_dim"]).contiguous()
        p = torch.bmm(q, kv[:, 0].permute(1, 2, 0).contiguous()) * scale
        p = torch.exp(p - p.amax(2, keepdim=True))
        o = torch.bmm(p, kv[:, 1].permute(1, 0, 2).contiguous()) / p.sum(2, keepdim=True)
        o = o.view(case["kv_heads"], r1 - r0, case["group"], case["head_dim"]).permute(1, 0, 2, 3)
        s["out"][r0:r1] = o.reshape(r1 - r0, -1, case["head_dim"]).to(s["out"].dtype)
    return s["out"]


def _own(s):
    from paper_2505_20600_amd import maskstep as MS
    op, block = s["case"]["op"], s["case"]["block"]
    if op in ("write", "rewrite"):
        MS.ms_kv8_quantize(s["kv"], s["codes"], s["scales"], block=block, src_row=s.get("src_row"))
        return s["codes"].view(torch.float8_e4m3fn), s["scales"]
    if op == "read":
        MS.ms_kv8_dequantize(s["codes"], s["scales"], s["kv"], block=block, keys=s["keys"], n_keys=s["n_keys"])
        return s["kv"]
    MS.ms_kv8_attention(s["q"], s["codes"], s["scales"], s["out"], s["seg_start"], block=block, cache_of=s["cache_of"],
                        keys=s["keys"], n_keys=s["n_keys"], fresh=s["fresh"], fresh_start=s["seg_start"],
                        workspace=s["workspace"])
    return s["out"]


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------


def _codes64():
    """The 256 codes' values: sign, four exponent bits (bias 7), three mantissa bits; no infinities, NaN at 127 and 255."""
    v = []
    for c in range(128):
        e, m = c >> 3, c & 7
        v.append(math.ldexp(m, -9) if e == 0 else math.ldexp(8 + m, e - 10))
    v[127] = math.nan
    return torch.tensor(v + [-x for x in v], dtype=torch.float64, device=DEV)


def _exact_quantize(v, block):
    """Nearest code of every value by search, ties to the even code, at the smallest power of two that holds the block."""
    grid = _codes64()[:127]
    mid = (grid[1:] + grid[:-1]) / 2
    T = v.shape[0]
    codes = torch.empty(v.shape, dtype=torch.float64, device=DEV)
    for t in range(0, T, block):
        x = v[t:t + block].double()
        a = x.abs().amax(dim=(0, 3))
        ex = torch.where(a > 0, torch.ceil(torch.log2(a / 448.0)), torch.zeros_like(a))
        ex = torch.where((a > 448.0 * torch.exp2(ex)), ex + 1, ex)          # the logarithm's own rounding
        ex = torch.where((a > 0) & (a <= 448.0 * torch.exp2(ex - 1)), ex - 1, ex).clamp(min=-126.0)
        y = x / torch.exp2(ex)[None, :, :, None]
        down = torch.searchsorted(mid, y.abs().contiguous())                 # a midpoint goes down here
        up = torch.searchsorted(mid, y.abs().contiguous(), right=True)
        at = torch.where(down % 2 == 0, down, up)
        codes[t:t + block] = grid[at] * y.sign()
    return codes


def _values64(codes, exps, block):
    s = torch.exp2(exps.double() - 127.0).repeat_interleave(block, 0)[:codes.shape[0]]
    return _codes64()[codes.long()] * s[..., None]


def exact(case, seed):
    s = prepare(case, seed)
    block = case["block"]
    if case["op"] == "write":
        return torch.stack([_exact_quantize(s["kv"][b], block) for b in range(case["caches"])]), None
    if case["op"] == "rewrite":
        out = []
        for b in range(case["caches"]):
            v = _values64(s["codes"][b], s["scales"][b], block)
            hit = (s["src_row"][b] >= 0).nonzero().flatten()
            v[hit] = s["kv"][s["src_row"][b, hit].long()].double()
            new = _exact_quantize(v, block)
            for t in range(0, v.shape[0], block):
                if not bool((s["src_row"][b, t:t + block] >= 0).any()):
                    new[t:t + block] = _codes64()[s["codes"][b, t:t + block].long()]
            out.append(new)
        return torch.stack(out), None
    if case["op"] == "read":
        kv = s["kv"].double()
        for b in range(case["batch"]):
            k = s["keys"][b, :s["counts"][b]].long()
            kv[b, k] = _values64(s["codes"][b][k], s["scales"][b].repeat_interleave(block, 0)[k], 1)
        return kv
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        r0, r1 = s["starts"][b], s["starts"][b + 1]
        k = s["keys"][b, :s["counts"][b]].long()
        kv = _values64(s["codes"][s["of"][b]][k], s["scales"][s["of"][b]].repeat_interleave(block, 0)[k], 1)
        if s["fresh"] is not None:
            kv = torch.cat([kv, s["fresh"][r0:r1].double()])
        if kv.shape[0] == 0:
            continue
        for h in range(case["kv_heads"] * case["group"]):
            g = h // case["group"]
            z = s["q"][r0:r1, h].double() @ kv[:, 0, g].t().contiguous() / math.sqrt(case["head_dim"])
            out[r0:r1, h] = torch.softmax(z, dim=1) @ kv[:, 1, g].contiguous()
    return out

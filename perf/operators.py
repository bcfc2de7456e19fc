"""Cases of the operators of an encoded decoder block, with their plain forms.

Four operators: the root-mean-square norm whose output is 8-bit level indices with one range per row
(``norm``), the product of level bytes with bias, activation and residual in its epilogue (``linear``),
writing keys and values into a paged cache of 8- or 4-bit levels and reading them back (``cache``), and
the attention of new tokens over such a cache (``attention``).

A value on levels of ``bits`` bits with range s is q s / L with q = 2u - L, L = 2^bits - 1 and u the level
index: u = floor((x (1/s)) ((L+1)/2 - 1/2)) + (L+1)/2, clamped to 0..L.
"""
import math
import random

import torch

own = False  # True: run() calls the framework's operators; False: the plain forms below

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
EPS = 1e-6


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a single token of one user between two layers: latency only
        dict(name="norm_token", op="norm", rows=1, k=4096, dtype="bf16", residual=True),
        # a long prompt's chunk between two layers
        dict(name="norm_chunk", op="norm", rows=4096, k=4096, dtype="bf16", residual=True),
        # one token through a projection back onto the residual stream: the weights are read once
        dict(name="linear_token", op="linear", m=1, n=4096, k=4096, out="bf16", act="none", bias=False, residual=True),
        # the benchmark's fully connected layer, 64 inputs, bias and ReLU, 32-bit output
        dict(name="linear_fc64", op="linear", m=64, n=4096, k=9216, out="f32", act="relu", bias=True, residual=False),
        # sizes that no tile divides: 777 tokens of several prompts, an odd number of outputs
        dict(name="linear_ragged", op="linear", m=777, n=5001, k=4100, out="f16", act="silu", bias=True, residual=True),
        # the square product of the benchmark's sweep, as the first half of a feed-forward layer
        dict(name="linear_4096", op="linear", m=4096, n=4096, k=4096, out="bf16", act="gelu_tanh", bias=True, residual=False),
        # one decode step of 64 users: one token each, 8 bits
        dict(name="cache_step", op="cache", tokens=64, heads=8, dim=128, bits=8, page=16, pages=4096, dtype="bf16", skip=0),
        # a long chunk written in 4 bits and read back for a layer that wants 16-bit keys; some padding tokens
        dict(name="cache_chunk4", op="cache", tokens=8192, heads=8, dim=128, bits=4, page=64, pages=512, dtype="f16", skip=37),
        # one user's next token, a short context: latency only
        dict(name="attn_token", op="attention", batch=1, q=1, kv=1000, spread=0, heads=32, kv_heads=8, dim=128, bits=8,
             page=16, dtype="bf16", causal=True, window=0, lse=False),
        # a decode step of 32 users with contexts of up to 16384 tokens
        dict(name="attn_step", op="attention", batch=32, q=1, kv=16384, spread=1, heads=32, kv_heads=8, dim=128, bits=8,
             page=16, dtype="bf16", causal=True, window=0, lse=False),
        # prompts and single tokens in one batch over 4-bit pages of 24 tokens, a sliding window, and an idle sequence
        dict(name="attn_ragged4", op="attention", batch=7, q=511, kv=5000, spread=2, heads=12, kv_heads=4, dim=64, bits=4,
             page=24, dtype="f16", causal=True, window=1500, lse=True),
        # the last chunk of a long prompt
        dict(name="attn_chunk", op="attention", batch=1, q=2048, kv=10240, spread=0, heads=32, kv_heads=8, dim=128, bits=8,
             page=64, dtype="bf16", causal=True, window=0, lse=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["norm", "linear", "cache", "attention"])
    if op == "norm":
        return dict(op=op, rows=_log(rng, 1, 4096), k=_log(rng, 64, 9216), dtype=rng.choice(["f32", "f16", "bf16"]),
                    residual=rng.random() < 0.7)
    if op == "linear":
        m, n, k = _log(rng, 1, 4096), _log(rng, 64, 9216), _log(rng, 64, 9216)
        m = max(1, min(m, 4096 ** 3 // (n * k)))
        return dict(op=op, m=m, n=n, k=k, out=rng.choice(["f32", "f16", "bf16"]),
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    if op == "cache":
        tokens, page = _log(rng, 1, 8192), rng.choice([8, 16, 24, 32, 64, 128])
        return dict(op=op, tokens=tokens, heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128]), bits=rng.choice([4, 8]), page=page,
                    pages=2 * tokens // page + 2, dtype=rng.choice(["f32", "f16", "bf16"]), skip=rng.randrange(0, 1 + tokens // 8))
    kv_heads = rng.choice([1, 2, 4, 8])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 8])
    dim, bits, page = rng.choice([64, 128]), rng.choice([4, 8]), rng.choice([8, 16, 24, 32, 64, 128])
    batch, q, kv = _log(rng, 1, 32), rng.choice([1, 1, _log(rng, 1, 2048)]), _log(rng, 1, 16384)
    q = min(q, kv)
    while batch * q * kv * heads > 32 * 2048 * 10240:      # pairs of the largest listed case
        batch, q = max(1, batch // 2), (max(1, q // 2) if batch == 1 else q)
    while batch * kv * kv_heads > 32 * 16384 * 8:
        kv //= 2
    return dict(op=op, batch=batch, q=min(q, kv), kv=kv, spread=rng.choice([0, 1, 2]) if batch > 1 else 0, heads=heads, kv_heads=kv_heads,
                dim=dim, bits=bits, page=page, dtype=rng.choice(["f16", "bf16"]), causal=rng.random() < 0.85,
                window=rng.choice([0, 0, _log(rng, 1, 4096)]), lse=rng.random() < 0.3)


def _lens(case):
    """New tokens and context lengths (new tokens included) of each sequence. spread 0: all alike;
    1: contexts from an eighth of the largest up; 2: chunks and single tokens mixed, one sequence idle."""
    batch, q, kv, rng = case["batch"], case["q"], case["kv"], random.Random(case["kv"] * 31 + case["q"])
    if case["spread"] == 0:
        return [q] * batch, [kv] * batch
    kvs = [kv] + [rng.randint(max(1, kv // 8), kv) for _ in range(batch - 1)]
    if case["spread"] == 1:
        return [min(q, n) for n in kvs], kvs
    qs = [q] + [min(kvs[i], 1 if i % 2 else rng.randint(1, q)) for i in range(1, batch)]
    if batch > 2:
        qs[2] = 0
    return qs, kvs


def _pairs(case):
    """(query, key) pairs that the masks leave, over all sequences and one head, and the keys that are read."""
    pairs = keys = 0
    for nq, nk in zip(*_lens(case)):
        lo = nk if nq else 0
        for i in range(nq):
            last = nk - nq + i if case["causal"] else nk - 1
            first = max(0, nk - nq + i - case["window"] + 1) if case["window"] else 0
            pairs += max(0, last - first + 1)
            lo = min(lo, first)
        keys += nk - lo if nq else 0
    return pairs, keys


def work(case):
    size = {"f32": 4, "f16": 2, "bf16": 2}
    if case["op"] == "norm":
        rows, k, e = case["rows"], case["k"], size[case["dtype"]]
        # x, residual, gain in; the new residual, level bytes, decoded values, range and level sum out
        return {"bytes": rows * k * (e * (3 if case["residual"] else 1) + 1 + 2) + 4 * k + 8 * rows, "flops": 8 * rows * k}
    if case["op"] == "linear":
        m, n, k, e = case["m"], case["n"], case["k"], size[case["out"]]
        return {"bytes": m * k + n * k + 8 * (m + n) + m * n * e * (2 if case["residual"] else 1) + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    if case["op"] == "cache":
        t, h, d = case["tokens"], case["heads"], case["dim"]
        e, row = size[case["dtype"]], d * case["bits"] // 8 + 4
        # keys and values in, levels and ranges out; the same back
        return {"bytes": 2 * t * h * (d * e + row) * 2 + 8 * t * 2, "flops": 8 * t * h * d}
    pairs, keys = _pairs(case)
    d, e, total = case["dim"], size[case["dtype"]], sum(_lens(case)[0])
    row = d * case["bits"] // 8 + 4
    return {"bytes": 2 * total * case["heads"] * d * e + 2 * keys * case["kv_heads"] * row + 4 * keys // case["page"],
            "flops": 4 * d * case["heads"] * pairs}


# ------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _index(y, s, bits):
    """Level index of y with range s (broadcast), in 32 bits: reciprocal, two products, floor."""
    half = 1 << (bits - 1)
    inv = torch.where((s > 0) & torch.isfinite(s), 1.0 / s, torch.zeros_like(s))
    t = torch.nan_to_num((y * inv) * (((1 << bits) - 1) / 2), nan=0.0)
    return torch.floor(torch.clamp(t, -half, half - 0.5)) + half


def _level_rows(x):
    """An operand of the product as it is kept: level bytes in rows of a multiple of 16 (zeros behind), range and level sum of each row."""
    rows, k = x.shape
    s = x.abs().amax(1)
    u = _index(x, s[:, None], 8).to(torch.uint8)
    held = torch.zeros((rows, -(-k // 16) * 16), dtype=torch.uint8, device="cuda")
    held[:, :k] = u
    return {"bytes": held, "scale": s, "sums": u.sum(1, dtype=torch.int32)}


def _pack(u, bits):
    u = u.to(torch.uint8)
    return u if bits == 8 else u[..., 0::2] | (u[..., 1::2] << 4)


def prepare(case, seed):
    g, s = _gen(seed), {"case": dict(case)}
    if case["op"] == "norm":
        dt, shape = DTYPES[case["dtype"]], (case["rows"], case["k"])
        channel = torch.exp(0.5 * _randn(g, case["k"]))          # channels of a residual stream differ in size
        s["x"] = (_randn(g, *shape) * channel).to(dt)
        s["r"] = (2.0 * _randn(g, *shape) * channel).to(dt) if case["residual"] else None
        s["gain"] = 1.0 + 0.2 * _randn(g, case["k"])
        s["values_type"] = torch.bfloat16 if case["dtype"] != "f16" else torch.float16
    elif case["op"] == "linear":
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _level_rows(_randn(g, m, k) * torch.exp(0.3 * _randn(g, m, 1)))
        s["w"] = _level_rows(_randn(g, n, k) / math.sqrt(k))
        s["bias"] = 0.2 * _randn(g, n) if case["bias"] else None
        s["res"] = _randn(g, m, n).to(DTYPES[case["out"]]) if case["residual"] else None
    elif case["op"] == "cache":
        t, h, d, dt = case["tokens"], case["heads"], case["dim"], DTYPES[case["dtype"]]
        kv = torch.exp(0.4 * _randn(g, 2, t, h, 1)) * _randn(g, 2, t, h, d)
        s["k"], s["v"] = kv[0].to(dt), kv[1].to(dt)
        slots = torch.randperm(case["pages"] * case["page"], generator=g, device="cuda")[:t]
        slots[t - case["skip"]:] = -1                             # padding of the batch: written nowhere
        s["slots"] = slots
        s["cache"] = _empty_cache(case["pages"], h, case["page"], d, case["bits"])
    else:
        s.update(_attention_inputs(case, g))
    return s


def _empty_cache(pages, heads, page, dim, bits):
    rows = lambda: torch.zeros((pages, heads, page, dim * bits // 8), dtype=torch.uint8, device="cuda")     # noqa: E731
    ranges = lambda: torch.zeros((pages, heads, page), dtype=torch.float32, device="cuda")                   # noqa: E731
    return {"k": rows(), "k_scale": ranges(), "v": rows(), "v_scale": ranges()}


def _attention_inputs(case, g):
    qs, kvs = _lens(case)
    batch, page, d, bits = case["batch"], case["page"], case["dim"], case["bits"]
    per = -(-max(kvs) // page)
    need = sum(-(-n // page) for n in kvs)
    pages = need + need // 8 + 1
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros((batch, per), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(kvs):
        used = -(-n // page)
        table[b, :used] = order[at:at + used]
        at += used
    cache = {}
    for name in ("k", "v"):
        x = _randn(g, pages, case["kv_heads"], page, d)
        if name == "v":
            x *= torch.exp(0.5 * _randn(g, pages, case["kv_heads"], page, 1))
        r = x.abs().amax(-1)
        cache[name], cache[name + "_scale"] = _pack(_index(x, r[..., None], bits), bits), r
    starts = [0]
    for n in qs:
        starts.append(starts[-1] + n)
    return {"q": (1.5 * _randn(g, starts[-1], case["heads"], d)).to(DTYPES[case["dtype"]]), "cache": cache, "table": table,
            "starts": torch.tensor(starts, dtype=torch.int32, device="cuda"), "lens": torch.tensor(kvs, dtype=torch.int32, device="cuda"),
            "max_q": max(qs), "max_kv": max(kvs), "scale": 1.0 / math.sqrt(d)}


# -------------------------------------------------------------------------------------------- runs
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_1905_13389_b200 import binding as mpq
    case = s["case"]
    if case["op"] == "norm":
        values = torch.empty(s["x"].shape, dtype=s["values_type"], device="cuda")
        h = torch.empty_like(s["x"]) if s["r"] is not None else None
        y = mpq.rmsnorm_levels(s["x"], s["gain"], EPS, 8, residual=s["r"], residual_out=h, values=values)
        return {"h": h, "values": values, "scale": y.scale}
    if case["op"] == "linear":
        a, w = (mpq.Levels(o["bytes"], o["scale"], o["sums"], 8, case["k"]) for o in (s["a"], s["w"]))
        return mpq.linear_levels(a, w, bias=s["bias"], act=case["act"], residual=s["res"], dtype=DTYPES[case["out"]])
    cache = mpq.LevelCache(s["cache"]["k"], s["cache"]["k_scale"], s["cache"]["v"], s["cache"]["v_scale"], case["bits"])
    if case["op"] == "cache":
        mpq.cache_write(cache, s["k"], s["v"], s["slots"])
        k, v = mpq.cache_read(cache, s["slots"], DTYPES[case["dtype"]])
        return {"k": k, "v": v}
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device="cuda") if case["lse"] else None
    out = mpq.cache_attention(s["q"], cache, s["starts"], s["lens"], s["table"], s["max_q"], s["max_kv"],
                              causal=case["causal"], window=case["window"], scale=s["scale"], lse=lse)
    return {"out": out, "lse": lse}


def _activate(y, act):
    if act == "relu":
        return torch.clamp(y, min=0)
    if act == "silu":
        return y / (1 + torch.exp(-y))
    if act == "gelu_tanh":
        return 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    if act == "gelu":
        return 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return y


def _decode(held, scale, bits):
    """Level bytes [..., d * bits / 8] with ranges [...] -> 32-bit values."""
    u = held if bits == 8 else torch.stack((held & 15, held >> 4), -1).flatten(-2)
    top = (1 << bits) - 1
    return (2 * u.float() - top) * (scale / top)[..., None]


def _run_plain(s):
    case = s["case"]
    if case["op"] == "norm":
        h = s["x"].float() + s["r"].float() if s["r"] is not None else s["x"].float()
        y = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["gain"]
        scale = y.abs().amax(1)
        values = (2 * _index(y, scale[:, None], 8) - 255) * (scale / 255)[:, None]
        return {"h": h.to(s["x"].dtype) if s["r"] is not None else None, "values": values.to(s["values_type"]), "scale": scale}
    if case["op"] == "linear":
        k = case["k"]
        a, w = (2 * s[o]["bytes"][:, :k].float() - 255 for o in ("a", "w"))
        y = (a @ w.T) * (s["a"]["scale"] / 255)[:, None] * (s["w"]["scale"] / 255)
        y = _activate(y + s["bias"] if case["bias"] else y, case["act"])
        return (y + s["res"].float() if case["residual"] else y).to(DTYPES[case["out"]])
    if case["op"] == "cache":
        return _cache_plain(s)
    return _attention_plain(s)


def _cache_plain(s):
    case, page, out = s["case"], s["case"]["page"], {}
    kept = case["tokens"] - case["skip"]
    p, o = s["slots"][:kept] // page, s["slots"][:kept] % page
    for name in ("k", "v"):
        x = s[name].float()
        r = x[:kept].abs().amax(-1)
        s["cache"][name][p, :, o] = _pack(_index(x[:kept], r[..., None], case["bits"]), case["bits"])
        s["cache"][name + "_scale"][p, :, o] = r
        back = torch.zeros_like(x)
        back[:kept] = _decode(s["cache"][name][p, :, o], s["cache"][name + "_scale"][p, :, o], case["bits"])
        out[name] = back.to(s[name].dtype)
    return out


def _attention_plain(s):
    case, q, c = s["case"], s["q"], s["cache"]
    page, groups, most_q, most_k = case["page"], case["heads"] // case["kv_heads"], s["max_q"], s["max_kv"]
    starts, lens = s["starts"].long(), s["lens"].long()
    nq = starts[1:] - starts[:-1]
    j = torch.arange(most_k, device="cuda")
    p, o = s["table"].long()[:, j // page], j % page                                           # [B, S]
    keys, vals = (_decode(c[n][p, :, o], c[n + "_scale"][p, :, o], case["bits"]) for n in ("k", "v"))   # [B, S, Hkv, D]
    i = torch.arange(most_q, device="cuda")
    rows = torch.clamp(starts[:-1, None] + i, max=max(0, q.shape[0] - 1))                      # [B, Q]
    qb = q[rows].float().unflatten(2, (case["kv_heads"], groups))                              # [B, Q, Hkv, G, D]
    pos = lens[:, None] - nq[:, None] + i                                                      # [B, Q]
    seen = j < lens[:, None, None]
    if case["causal"]:
        seen = seen & (j <= pos[:, :, None])
    if case["window"]:
        seen = seen & (j > pos[:, :, None] - case["window"])
    x = qb.permute(0, 2, 3, 1, 4).flatten(2, 3) @ keys.permute(0, 2, 3, 1)                     # [B, Hkv, G*Q, S]
    x = x.unflatten(2, (groups, most_q)).mul_(s["scale"]).masked_fill_(~seen[:, None, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    x = x.sub_(top).exp_()
    total = x.sum(-1)
    out = (x.flatten(2, 3) @ vals.permute(0, 2, 1, 3)).unflatten(2, (groups, most_q))
    out = out / torch.where(total > 0, total, torch.ones_like(total))[..., None]
    lse = torch.log(total) + top[..., 0]
    live = i < nq[:, None]                                                                     # [B, Q]
    out = out.permute(0, 3, 1, 2, 4).flatten(2, 3)[live].to(q.dtype)
    return {"out": out, "lse": lse.permute(0, 3, 1, 2).flatten(2, 3)[live] if case["lse"] else None}


# ------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The operators' definitions in 64 bits. Level indices of the cache are decided by the quantizer's own
    32-bit arithmetic, which is its definition; everything else is 64-bit."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "norm":
        h = s["x"].to(f64)
        if case["residual"]:
            h = h + s["r"].to(f64)
        y = s["gain"].to(f64) * h / (h.pow(2).sum(1, keepdim=True) / case["k"] + EPS).sqrt()
        top = y.abs().max(1, keepdim=True).values
        level = torch.floor(127.5 * y / top).clamp(-128, 127)
        return {"h": h if case["residual"] else None, "values": (2 * level + 1) / 255 * top, "scale": top[:, 0]}
    if case["op"] == "linear":
        k = case["k"]
        q = [s[o]["bytes"][:, :k].to(f64).mul_(2).sub_(255).mul_(s[o]["scale"].to(f64)[:, None] / 255) for o in ("a", "w")]
        y = torch.mm(q[0], q[1].t())
        if case["bias"]:
            y += s["bias"].to(f64)
        act = case["act"]
        if act == "relu":
            y = y.relu()
        elif act == "silu":
            y = y * torch.sigmoid(y)
        elif act == "gelu":
            y = y * 0.5 * torch.erfc(-y / math.sqrt(2.0))
        elif act == "gelu_tanh":
            y = y * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (y + 0.044715 * y ** 3))
        return y + s["res"].to(f64) if case["residual"] else y
    if case["op"] == "cache":
        out, kept = {}, case["tokens"] - case["skip"]
        top = (1 << case["bits"]) - 1
        for name in ("k", "v"):
            x = s[name].float()
            r = x.abs().max(-1, keepdim=True).values
            half = (top + 1) // 2
            level = torch.floor(((x * (1.0 / r)) * (top / 2)).clamp(-half, half - 0.5)).to(f64) * 2 + 1
            out[name] = level * r.to(f64) / top
            out[name][kept:] = 0
        return out
    return _attention_exact(case, s)


def _attention_exact(case, s):
    f64, top = torch.float64, (1 << case["bits"]) - 1
    groups, page = case["heads"] // case["kv_heads"], case["page"]
    out = torch.zeros(s["q"].shape, dtype=f64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=f64, device="cuda")
    starts, lens = s["starts"].tolist(), s["lens"].tolist()
    for b in range(case["batch"]):
        lo, hi, n = starts[b], starts[b + 1], lens[b]
        if hi == lo or n == 0:
            continue
        pos = n - (hi - lo) + torch.arange(hi - lo, device="cuda")
        j = torch.arange(n, device="cuda")
        hide = torch.zeros((hi - lo, n), dtype=torch.bool, device="cuda")
        if case["causal"]:
            hide |= j[None] > pos[:, None]
        if case["window"]:
            hide |= j[None] <= pos[:, None] - case["window"]
        used = s["table"][b, :-(-n // page)].long()
        for h in range(case["kv_heads"]):
            kv = []
            for name in ("k", "v"):
                raw = s["cache"][name][used, h].reshape(-1, case["dim"] * case["bits"] // 8)[:n].to(torch.int64)
                if case["bits"] == 4:
                    raw = torch.stack([raw % 16, raw // 16], dim=2).reshape(n, case["dim"])
                kv.append((raw.to(f64) * 2 - top) / top * s["cache"][name + "_scale"][used, h].reshape(-1, 1)[:n].to(f64))
            for head in range(h * groups, (h + 1) * groups):
                x = (s["q"][lo:hi, head].to(f64) @ kv[0].T) * s["scale"]
                x[hide] = -math.inf
                z = torch.logsumexp(x, dim=1)
                w = torch.exp(x - torch.where(torch.isinf(z), torch.zeros_like(z), z)[:, None])
                out[lo:hi, head], lse[lo:hi, head] = w @ kv[1], z
    return {"out": out, "lse": lse if case["lse"] else None}

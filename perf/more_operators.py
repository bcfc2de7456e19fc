"""Cases of the operators around a server's step over many requests, with their plain forms.

Three operators: page tables and slot maps made from request lengths on the device, with the way back
(``pages``), the product of level bytes with low-rank adapters chosen per request in its epilogue (``adapted``),
and drawing tokens from logits with temperature, top-k, top-p and min-p from given random numbers (``sample``).

A value on levels of ``bits`` bits with range s is q s / L with q = 2u - L, L = 2^bits - 1 and u the level index.
"""
import math
import random

import torch

own = False  # True: run() calls the framework's operators; False: the plain forms below

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}


# ---------------------------------------------------------------------------------------------- cases
def listed():
    return [
        # a decode step of 64 users, one token each, contexts of up to 4096 tokens; three entries are padding of a captured step
        dict(name="pages_step", op="pages", batch=64, idle=3, sequences=80, per=256, page=16, context=4096, new=1, pad=3, full=False),
        # a verification step of 200 users, up to five draft tokens each, pages that are no power of two
        dict(name="pages_draft", op="pages", batch=200, idle=0, sequences=333, per=171, page=24, context=4000, new=5, pad=0, full=False),
        # prompts of up to 4096 tokens admitted beside long contexts, and dropped again
        dict(name="pages_prompts", op="pages", batch=512, idle=17, sequences=512, per=1024, page=16, context=12000, new=4096, pad=1000, full=False),
        # one user's token through a projection with an adapter: latency
        dict(name="adapted_token", op="adapted", batch=1, m=1, n=4096, k=4096, rank=16, adapters=4, bare=0, weights="bf16",
             out="bf16", act="none", bias=False, residual=True),
        # a decode step of 64 users, each with one of 48 adapters or none, into the benchmark's fully connected layer
        dict(name="adapted_step", op="adapted", batch=64, m=64, n=4096, k=9216, rank=16, adapters=48, bare=5, weights="bf16",
             out="bf16", act="relu", bias=True, residual=False),
        # prompts and single tokens mixed, sizes that no tile divides, a rank that is no multiple of 16
        dict(name="adapted_ragged", op="adapted", batch=23, m=777, n=5001, k=4100, rank=24, adapters=9, bare=3, weights="f16",
             out="f16", act="silu", bias=True, residual=True),
        # the long chunks of six prompts through the first half of a feed-forward layer
        dict(name="adapted_prompts", op="adapted", batch=6, m=4096, n=4096, k=4096, rank=64, adapters=5, bare=1, weights="bf16",
             out="bf16", act="gelu_tanh", bias=True, residual=False),
        # one user's next token, every rule on: latency
        dict(name="sample_token", op="sample", rows=1, vocab=131072, dtype="f32", rules="all", masked=0.0, logprob=True),
        # a few users of a small vocabulary of odd size, some of its tokens forbidden by a grammar
        dict(name="sample_masked", op="sample", rows=7, vocab=50021, dtype="f16", rules="mixed", masked=0.7, logprob=True),
        # a decode step of 64 users, each with rules of their own, greedy ones among them
        dict(name="sample_step", op="sample", rows=64, vocab=131072, dtype="bf16", rules="mixed", masked=0.0, logprob=True),
        # a wide batch of rollouts, nucleus and temperature
        dict(name="sample_nucleus", op="sample", rows=256, vocab=151000, dtype="f32", rules="top_p", masked=0.0, logprob=False),
        # the same by temperature alone: the whole vocabulary stays
        dict(name="sample_all", op="sample", rows=256, vocab=131072, dtype="bf16", rules="none", masked=0.0, logprob=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["pages", "adapted", "sample"])
    if op == "pages":
        batch, page = _log(rng, 1, 512), rng.choice([8, 16, 24, 32, 64, 128])
        context = _log(rng, 1, 12000)
        new = rng.choice([1, 1, _log(rng, 1, 8), _log(rng, 8, 4096)])
        return dict(op=op, batch=batch, idle=rng.randrange(0, 1 + batch // 8), sequences=batch + rng.randrange(0, 100),
                    per=-(-(context + new) // page) + rng.randrange(0, 9), page=page, context=context, new=new, pad=rng.randrange(0, 64),
                    full=rng.random() < 0.1)
    if op == "adapted":
        m, n, k = _log(rng, 1, 4096), _log(rng, 64, 9216), _log(rng, 64, 9216)
        m = max(1, min(m, 4096 ** 3 // (n * k)))
        adapters = _log(rng, 1, 64)
        return dict(op=op, batch=min(m, _log(rng, 1, 128)), m=m, n=n, k=k, rank=rng.choice([4, 8, 16, 16, 24, 32, 64]), adapters=adapters,
                    bare=rng.randrange(0, 4), weights=rng.choice(["f16", "bf16"]), out=rng.choice(["f32", "f16", "bf16"]),
                    act=rng.choice(["none", "relu", "gelu", "gelu_tanh", "silu"]), bias=rng.random() < 0.5, residual=rng.random() < 0.5)
    vocab = _log(rng, 100, 151000)
    return dict(op=op, rows=_log(rng, 1, 256), vocab=vocab, dtype=rng.choice(["f32", "f16", "bf16"]),
                rules=rng.choice(["all", "mixed", "mixed", "top_k", "top_p", "min_p", "none"]),
                masked=rng.choice([0.0, 0.0, 0.5, 0.95]), logprob=rng.random() < 0.6)


def _lengths(case):
    """Tokens of each sequence of an adapted batch: `m` in all, single tokens and longer pieces mixed."""
    batch, m, rng = case["batch"], case["m"], random.Random(case["m"] * 131 + case["batch"])
    share = [1 if i % 3 == 1 else rng.random() ** 3 * m for i in range(batch)]
    left, out = m - batch, []
    total = sum(share)
    for x in share:
        out.append(1 + int(left * x / total))
    out[0] += m - sum(out)
    return out


def _chosen(case):
    """The adapter of each sequence, -1 for none."""
    rng = random.Random(case["batch"] * 7 + case["adapters"])
    return [-1 if case["batch"] > 1 and i < case["bare"] * case["batch"] // 16 else rng.randrange(case["adapters"]) for i in range(case["batch"])]


def _page_sizes(case):
    """Sequence, context and new tokens of each entry of a batch, and the contexts of all sequences."""
    rng = random.Random(case["batch"] * 977 + case["page"] + case["context"])
    lens = [rng.randint(0, case["context"]) for _ in range(case["sequences"])]
    seqs = rng.sample(range(case["sequences"]), case["batch"])
    for i in rng.sample(range(case["batch"]), case["idle"]):
        seqs[i] = -1
    new = [case["new"] if case["new"] == 1 else _log(rng, 1, case["new"]) for _ in seqs]
    return seqs, new, lens


def work(case):
    if case["op"] == "pages":
        seqs, new, lens = _page_sizes(case)
        total = sum(n for q, n in zip(seqs, new) if q >= 0)
        used = sum(-(-(lens[q] + n) // case["page"]) for q, n in zip(seqs, new) if q >= 0)
        added = sum(-(-(lens[q] + n) // case["page"]) - -(-lens[q] // case["page"]) for q, n in zip(seqs, new) if q >= 0)
        # slots and table rows out, the tables in, lengths, the pages taken and given back
        return {"bytes": 8 * (total + case["pad"]) + 4 * case["batch"] * (case["per"] + 8) + 4 * used + 16 * added, "flops": 4 * total}
    if case["op"] == "adapted":
        m, n, k, e, rank = case["m"], case["n"], case["k"], SIZE[case["out"]], case["rank"]
        ids = [(i, x) for i, x in zip(_chosen(case), _lengths(case)) if i >= 0]
        used, rows = len({i for i, _ in ids}), sum(x for _, x in ids)
        return {"bytes": m * k + n * k + 8 * (m + n) + m * n * e * (2 if case["residual"] else 1) + (4 * n if case["bias"] else 0) + 2 * used * rank * (n + k),
                "flops": 2 * m * n * k + 2 * rows * rank * (n + k)}
    return {"bytes": case["rows"] * (case["vocab"] * SIZE[case["dtype"]] + 32), "flops": 4 * case["rows"] * case["vocab"]}


# ------------------------------------------------------------------------------------------- inputs
def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 29)


def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _ints(v, dtype=torch.int32):
    return torch.tensor(v, dtype=dtype, device="cuda")


def _level_rows(x):
    """An operand of the product as it is kept: level bytes in rows of a multiple of 16 (zeros behind), range and level sum of each row."""
    rows, k = x.shape
    s = x.abs().amax(1)
    inv = torch.where((s > 0) & torch.isfinite(s), 1.0 / s, torch.zeros_like(s))[:, None]
    u = (torch.floor(torch.clamp((x * inv) * 127.5, -128, 127.5)) + 128).to(torch.uint8)
    held = torch.zeros((rows, -(-k // 16) * 16), dtype=torch.uint8, device="cuda")
    held[:, :k] = u
    return {"bytes": held, "scale": s, "sums": u.sum(1, dtype=torch.int32)}


def prepare(case, seed):
    g, s = _gen(seed), {"case": dict(case)}
    if case["op"] == "pages":
        seqs, new, lens = _page_sizes(case)
        page, per = case["page"], case["per"]
        held = [-(-n // page) for n in lens]
        spare = sum(-(-n // page) + 1 for n in new)
        pages = sum(held) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        s["lens"] = _ints(lens)
        firsts = torch.cumsum(_ints(held, torch.int64), 0) - _ints(held, torch.int64)
        i = torch.arange(per, device="cuda")
        at = torch.clamp(firsts[:, None] + i, max=pages - 1)
        s["table"] = torch.where(i < _ints(held, torch.int64)[:, None], order[at], torch.zeros_like(order[at]))
        s["free"] = torch.zeros(pages, dtype=torch.int32, device="cuda")
        left = spare // 8 if case["full"] else spare            # a full cache has too few pages for this batch
        s["free"][:left] = order[sum(held):sum(held) + left]
        s["count"] = _ints([left, 0])                            # pages that are free, and a word that the calls need
        s["seqs"], s["new"] = _ints(seqs), _ints(new)
        s["old"] = torch.where(s["seqs"] >= 0, s["lens"][s["seqs"].long().clamp(min=0)], 0)
        s["tokens"] = sum(n for q, n in zip(seqs, new) if q >= 0) + case["pad"]
        # a server's step keeps the buffers that its batch is described in
        s["out"] = [torch.empty(s["tokens"], dtype=torch.int64, device="cuda")] + [
            torch.empty(n, dtype=torch.int32, device="cuda") for n in (len(seqs) + 1, len(seqs), (len(seqs), per), 1)]
    elif case["op"] == "adapted":
        m, n, k, rank, dt = case["m"], case["n"], case["k"], case["rank"], DTYPES[case["weights"]]
        s["a"] = _level_rows(_randn(g, m, k) * torch.exp(0.3 * _randn(g, m, 1)))
        s["w"] = _level_rows(_randn(g, n, k) / math.sqrt(k))
        wide, row = -(-rank // 16) * 16, -(-k // 16) * 16         # adapters are kept padded with zeros to whole 16s
        s["down"] = torch.zeros((case["adapters"], wide, row), dtype=dt, device="cuda")
        s["down"][:, :rank, :k] = (_randn(g, case["adapters"], rank, k) / math.sqrt(k)).to(dt)
        s["up"] = torch.zeros((case["adapters"], n, wide), dtype=dt, device="cuda")
        s["up"][:, :, :rank] = (0.5 * _randn(g, case["adapters"], n, rank) / math.sqrt(rank)).to(dt)
        s["factor"] = 0.5 + torch.rand(case["adapters"], generator=g, device="cuda")
        starts = [0]
        for x in _lengths(case):
            starts.append(starts[-1] + x)
        s["starts"], s["ids"] = _ints(starts), _ints(_chosen(case))
        s["bias"] = 0.2 * _randn(g, n) if case["bias"] else None
        s["res"] = _randn(g, m, n).to(DTYPES[case["out"]]) if case["residual"] else None
    else:
        rows, vocab = case["rows"], case["vocab"]
        # a bell of unlikely tokens and a few likely ones, as the last layer gives them
        x = 2.0 * _randn(g, rows, vocab)
        likely = torch.randint(0, vocab, (rows, 20), generator=g, device="cuda")
        x.scatter_add_(1, likely, 4.0 + 5.0 * torch.rand((rows, 20), generator=g, device="cuda"))
        if case["masked"]:
            x[torch.rand((rows, vocab), generator=g, device="cuda") < case["masked"]] = -math.inf
            x[:, vocab // 2] = 1.0
        s["logits"] = x.to(DTYPES[case["dtype"]])
        u = lambda lo, hi: lo + (hi - lo) * torch.rand(rows, generator=g, device="cuda")          # noqa: E731
        on = lambda share: torch.rand(rows, generator=g, device="cuda") < share                   # noqa: E731
        s["uniform"], rules = u(0, 1), case["rules"]
        s["temperature"], s["top_k"], s["top_p"], s["min_p"] = u(0.6, 1.2), None, None, None
        if rules in ("all", "mixed", "top_k"):
            s["top_k"] = torch.randint(1, 200, (rows,), generator=g, device="cuda", dtype=torch.int32)
        if rules in ("all", "mixed", "top_p"):
            s["top_p"] = u(0.7, 0.98)
        if rules in ("all", "mixed", "min_p"):
            s["min_p"] = u(0.01, 0.1)
        if rules == "mixed":                                       # each request has some of the rules
            s["temperature"] = torch.where(on(0.2), 0.0, s["temperature"])
            s["top_k"] = torch.where(on(0.5), 0, s["top_k"])
            s["top_p"] = torch.where(on(0.5), 1.0, s["top_p"])
            s["min_p"] = torch.where(on(0.5), 0.0, s["min_p"])
    return s


# -------------------------------------------------------------------------------------------- runs
def run(s):
    return (_run_own if own else _run_plain)(s)


def _run_own(s):
    from paper_1905_13389_b200 import binding as mpq
    case = s["case"]
    if case["op"] == "pages":
        state = mpq.PageState(s["table"], s["lens"], s["free"], s["count"], case["page"])
        plan = mpq.pages_extend(state, s["seqs"], s["new"], s["tokens"], out=mpq.PagePlan(*s["out"]))
        mpq.pages_trim(state, s["seqs"], s["old"])                # the step's tokens are rejected, its requests dropped
        return {"slots": plan.slots, "starts": plan.q_starts, "lens": plan.kv_lens, "table": plan.table, "missing": plan.missing,
                "kept": s["lens"], "free": s["free"], "count": s["count"][:1]}
    if case["op"] == "adapted":
        k = case["k"]
        a, w = (mpq.Levels(o["bytes"], o["scale"], o["sums"], 8, k) for o in (s["a"], s["w"]))
        low = mpq.Adapters(s["down"], s["up"], s["factor"], k)
        return mpq.linear_adapted(a, w, low, s["starts"], s["ids"], bias=s["bias"], act=case["act"], residual=s["res"], dtype=DTYPES[case["out"]])
    logprob = torch.empty(case["rows"], dtype=torch.float32, device="cuda") if case["logprob"] else None
    tokens = mpq.sample(s["logits"], s["uniform"], s["temperature"], s["top_k"], s["top_p"], s["min_p"], logprob=logprob)
    return {"tokens": tokens, "logprob": logprob}


def _run_plain(s):
    return {"pages": _pages_plain, "adapted": _adapted_plain, "sample": _sample_plain}[s["case"]["op"]](s)


def _entries(s):
    """Which entries name a sequence, its row (0 for the others), and the entry of each sequence (-1: none)."""
    n = s["lens"].shape[0]
    named = (s["seqs"] >= 0) & (s["seqs"] < n)
    entry = torch.full((n + 1,), -1, dtype=torch.int64, device="cuda")
    entry[torch.where(named, s["seqs"], n).long()] = torch.arange(len(s["seqs"]), device="cuda")
    return named, torch.where(named, s["seqs"], 0).long(), entry[:n]


def _pages_plain(s):
    page, per, pages, tokens = s["case"]["page"], s["case"]["per"], s["free"].shape[0], s["tokens"]
    named, q, entry = _entries(s)
    # the batch's tokens and pages
    n, old = torch.where(named, s["new"], 0).long(), torch.where(named, s["lens"][q], 0).long()
    have, want = (old + page - 1) // page, (old + n + page - 1) // page
    need, count = want - have, s["count"][0].long()
    ends, upto = torch.cumsum(n, 0), torch.cumsum(need, 0)
    missing = torch.clamp(upto[-1] - count, min=0)
    missing = torch.where(ends[-1] > tokens, -2, missing)
    missing = torch.where((want > per).any(), -1, missing)
    fine = missing == 0
    i = torch.arange(per, device="cuda")
    popped = s["free"][torch.clamp(count - 1 - ((upto - need)[:, None] + i - have[:, None]), 0, pages - 1)]
    rows = torch.where(i < have[:, None], s["table"][q], torch.where(i < want[:, None], popped, 0))
    t = torch.arange(tokens, device="cuda")
    b = torch.clamp(torch.searchsorted(ends, t, right=True), max=len(n) - 1)
    j = torch.where(t < ends[-1], old[b] + t - (ends - n)[b], 0)
    slots = rows[b, torch.clamp(j // page, max=per - 1)].long() * page + j % page
    slots = torch.where(fine & (t < ends[-1]), slots, -1)
    at = torch.clamp(entry, min=0)
    new_here = (fine & (entry >= 0))[:, None] & (i >= have[at][:, None]) & (i < want[at][:, None])
    s["table"].copy_(torch.where(new_here, rows[at], s["table"]))
    s["lens"].copy_(torch.where(fine & (entry >= 0), (old + n)[at], s["lens"].long()))
    s["count"][0] -= torch.where(fine, upto[-1], 0).int()
    out = {"slots": slots, "starts": torch.where(fine, torch.cat([ends[:1] * 0, ends]), 0).int(), "lens": torch.where(fine, old + n, 0).int(),
           "table": torch.where(fine, rows, 0), "missing": missing.int()[None]}
    # and back to the lengths before
    keep = torch.minimum(torch.where(named, s["old"], 0).long(), s["lens"][q].long())
    first = (keep + page - 1) // page
    back = torch.where(named, (s["lens"][q].long() + page - 1) // page - first, 0)
    upto, count = torch.cumsum(back, 0), s["count"][0].long()
    spot = torch.arange(pages, device="cuda")
    k = upto[-1] - 1 - (spot - count)
    b = torch.clamp(torch.searchsorted(upto, k, right=True), max=len(n) - 1)
    page_at = s["table"][q[b], torch.clamp(first[b] + k - (upto - back)[b], 0, per - 1)]
    s["free"].copy_(torch.where((spot >= count) & (k >= 0), page_at, s["free"]))
    s["lens"].copy_(torch.where(entry >= 0, keep[at], s["lens"].long()))
    s["count"][0] += upto[-1].int()
    return dict(out, kept=s["lens"], free=s["free"], count=s["count"][:1])


def _adapted_plain(s):
    case, k = s["case"], s["case"]["k"]
    m, count, wide = case["m"], case["adapters"], s["down"].shape[1]
    x, w = ((2 * s[o]["bytes"][:, :k].float() - 255) * (s[o]["scale"] / 255)[:, None] for o in ("a", "w"))
    y = x @ w.T
    if case["bias"]:
        y = y + s["bias"]
    # every token through every adapter, all but its own one masked
    t = torch.arange(m, device="cuda")
    mine = s["ids"].long()[torch.searchsorted(s["starts"][1:].long(), t, right=True)]
    z = (x @ s["down"][:, :, :k].float().flatten(0, 1).T).unflatten(1, (count, wide)) * s["factor"][:, None]
    z = torch.where(mine[:, None, None] == torch.arange(count, device="cuda")[:, None], z, 0)
    y = y + z.flatten(1) @ s["up"].float().permute(0, 2, 1).flatten(0, 1)
    act = case["act"]
    if act == "relu":
        y = torch.clamp(y, min=0)
    elif act == "silu":
        y = y / (1 + torch.exp(-y))
    elif act == "gelu_tanh":
        y = 0.5 * y * (1 + torch.tanh(math.sqrt(2 / math.pi) * (y + 0.044715 * y * y * y)))
    elif act == "gelu":
        y = 0.5 * y * (1 + torch.erf(y * math.sqrt(0.5)))
    return (y + s["res"].float() if case["residual"] else y).to(DTYPES[case["out"]])


def _sample_plain(s):
    """64 bits throughout: a token is decided by where a running sum passes a border."""
    case, vocab = s["case"], s["case"]["vocab"]
    x = s["logits"].double()
    value, order = torch.sort(x, dim=1, descending=True, stable=True)                # ties: the lowest index first
    top, greedy = value[:, :1], s["temperature"] <= 0
    warm = torch.where(greedy, 1.0, s["temperature"]).double()[:, None]
    weight = torch.exp((value - top) / warm)
    if s["top_k"] is not None:
        k = torch.where(s["top_k"] > 0, s["top_k"], vocab)[:, None]
        weight = torch.where(torch.arange(vocab, device="cuda") < k, weight, 0)
    if s["top_p"] is not None:
        p = torch.where(s["top_p"] < 1, s["top_p"], math.inf).double()[:, None]
        upto = torch.cumsum(weight, 1)
        before = torch.cat([torch.zeros_like(upto[:, :1]), upto[:, :-1]], 1)
        weight = torch.where((before < p * upto[:, -1:]), weight, 0)
        weight[:, 0] = 1
    if s["min_p"] is not None:
        weight = torch.where(weight >= s["min_p"].double()[:, None], weight, 0)
        weight[:, 0] = 1
    upto = torch.cumsum(torch.zeros_like(x).scatter_(1, order, weight), 1)           # in the order of the vocabulary
    token = torch.searchsorted(upto, s["uniform"].double()[:, None] * upto[:, -1:], right=True)
    token = torch.where(greedy, order[:, 0], torch.clamp(token[:, 0], max=vocab - 1))
    logprob = None
    if case["logprob"]:
        total = torch.exp(value - top).sum(1)
        logprob = (x.gather(1, token[:, None])[:, 0] - top[:, 0] - torch.log(total)).float()
    return {"tokens": token, "logprob": logprob}


# ------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The operators' definitions in 64 bits, sequence by sequence and row by row."""
    s = prepare(case, seed)
    if case["op"] == "pages":
        return _pages_exact(case, s)
    return (_adapted_exact if case["op"] == "adapted" else _sample_exact)(case, s)


def _pages_exact(case, s):
    page, per = case["page"], case["per"]
    table, lens, count = s["table"].tolist(), s["lens"].tolist(), s["count"].tolist()[0]
    stack, starts, ends, rows, slots, taken = s["free"].tolist()[:count], [0], [], [], [], 0
    for q, n in zip(s["seqs"].tolist(), s["new"].tolist()):
        if q < 0:
            starts.append(starts[-1])
            ends.append(0)
            rows.append([0] * per)
            continue
        mine = table[q][:-(-lens[q] // page)]
        while len(mine) * page < lens[q] + n:
            taken += 1
            mine.append(stack.pop() if stack else 0)
        slots += [mine[j // page] * page + j % page for j in range(lens[q], lens[q] + n)]
        starts.append(len(slots))
        ends.append(lens[q] + n)
        rows.append(mine + [0] * (per - len(mine)))
    short = max(0, taken - count)
    if short:
        starts, ends, rows, slots = [0] * len(starts), [0] * len(ends), [[0] * per for _ in ends], []
    slots += [-1] * (s["tokens"] - len(slots))
    return {"slots": _ints(slots, torch.int64), "starts": _ints(starts), "lens": _ints(ends), "table": _ints(rows), "missing": _ints([short]),
            "kept": s["lens"], "free": s["free"], "count": s["count"][:1]}


def _adapted_exact(case, s):
    f64, k = torch.float64, case["k"]
    a, w = (s[o]["bytes"][:, :k].to(f64).mul_(2).sub_(255).mul_(s[o]["scale"].to(f64)[:, None] / 255) for o in ("a", "w"))
    y = torch.mm(a, w.t())
    if case["bias"]:
        y += s["bias"].to(f64)
    starts, ids = s["starts"].tolist(), s["ids"].tolist()
    for b, i in enumerate(ids):
        if i >= 0:
            rows = slice(starts[b], starts[b + 1])
            low = torch.mm(a[rows], s["down"][i, :, :k].to(f64).t())
            y[rows] += s["factor"][i].to(f64) * torch.mm(low, s["up"][i].to(f64).t())
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


def _sample_exact(case, s):
    if case["rows"] * case["vocab"] > 1 << 26:
        return None
    tokens, logprob = [], []
    settings = [None if s[n] is None else s[n].double().tolist() for n in ("temperature", "top_k", "top_p", "min_p", "uniform")]
    for r in range(case["rows"]):
        warm, k, p, least, u = (None if v is None else v[r] for v in settings)
        x = s["logits"][r].double()
        live = torch.nonzero(x > -math.inf)[:, 0]
        ranked = live[torch.argsort(x[live], descending=True, stable=True)]
        if warm <= 0:
            tokens.append(int(ranked[0]))
        else:
            if k is not None and k > 0:
                ranked = ranked[:int(k)]
            w = torch.exp(x[ranked] / warm - x[ranked[0]] / warm)
            if p is not None and p < 1:
                size = 1 + int((torch.cumsum(w, 0) < p * w.sum()).sum())
                ranked, w = ranked[:size], w[:size]
            if least is not None:
                few = max(1, int((w >= least).sum()))
                ranked, w = ranked[:few], w[:few]
            kept, at = torch.sort(ranked)
            upto = torch.cumsum(w[at], 0)
            tokens.append(int(kept[min(len(kept) - 1, int((upto <= u * upto[-1]).sum()))]))
        logprob.append(float(x[tokens[-1]] - torch.logsumexp(x, 0)))
    return {"tokens": _ints(tokens, torch.int64), "logprob": torch.tensor(logprob, dtype=torch.float64, device="cuda") if case["logprob"] else None}

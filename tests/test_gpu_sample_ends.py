"""Drawing tokens where a border lies next to a sum and where most of a row weighs nothing: the token is one of those that the stated
errors of the weights allow."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
LONG = np.longdouble


def upto_of(w, n):
    return w[:n].sum()


def allowed(x, warm, k, p, least, u):
    """One row: the tokens that may be drawn.  A weight is a whole multiple of 2^-shift of the largest one, which is exact: the nearest to a
    number that is off by 2^-42 of itself at most.  So it is off by that and by half a multiple, or by itself where it comes out as
    nothing; shares of sums are rounded to a multiple."""
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if warm <= 0:
        return {int(order[0])}
    bits = math.ceil(math.log2(len(x))) if len(x) > 1 else 0
    unit = LONG(2) ** -min(50, 62 - bits)
    if k > 0:
        order = order[:k]
    w = np.exp((x[order].astype(LONG) - LONG(x[order[0]])) / LONG(warm))
    off = np.minimum(w, unit / 2) + w * LONG(2) ** -42
    off[w == 1] = 0
    spare = LONG(0)
    sizes = [len(order)]
    if p < 1:
        upto, by = np.cumsum(w), np.cumsum(off) + LONG(p) * off.sum() + unit
        goal = LONG(max(p, 0.0)) * upto[-1]
        first = lambda reached: int(np.argmax(reached)) + 1 if reached.any() else len(order)      # noqa: E731
        sizes = range(first(upto >= goal - by), first(upto >= goal + by) + 1)
        if len(sizes) > 4:                                    # the shortest and the longest, and what they differ by as one more error
            spare = upto[sizes[-1] - 1] - upto[sizes[0] - 1]
            sizes = [sizes[0], sizes[-1]]
    found = set()
    for size in sizes:
        sure, maybe = size, size
        if least > 0:
            sure = max(1, int((w[:size] - off[:size] - unit >= least).sum()))
            maybe = max(1, int((w[:size] + off[:size] >= least).sum()))
        # (where weights differ by less than their errors any number of them may reach min-p: all numbers, or the ends as above)
        wide_min = upto_of(w, maybe) - upto_of(w, sure) if maybe - sure > 64 else LONG(0)
        for few in range(sure, maybe + 1) if maybe - sure <= 64 else (sure, maybe):
            at = np.argsort(order[:few])
            mine, err = w[:few][at], off[:few][at]
            upto, by = np.cumsum(mine), np.cumsum(err)
            share = LONG(min(max(u, 0.0), 1.0))
            goal, wide = share * upto[-1], by + share * by[-1] + unit + spare + wide_min
            # (a token that may come out as nothing is not drawn for sure, one that must come out as nothing never)
            can = (upto - mine - wide <= goal) & (goal <= upto + wide) & (mine + err > unit / 2)
            if not can.any():                                 # u = 1: behind all sums
                can = np.arange(few) == np.flatnonzero(mine + err > unit / 2)[-1]
            found |= {int(v) for v in order[:few][at][can]}
    return found


def check(mpq, cuda, x, u, warm=None, k=None, p=None, least=None, dtype="f32"):
    """Returns the tokens and how many of them could have been others."""
    rows = x.shape[0]
    logits = x.to(TYPES[dtype]).to(cuda)
    to = lambda v, t=torch.float32: None if v is None else torch.as_tensor(v).to(t).to(cuda)      # noqa: E731
    got = mpq.sample(logits, to(u), to(warm), to(k, torch.int32), to(p), to(least)).tolist()
    xs = logits.double().cpu().numpy()
    pick = lambda v, i, other: other if v is None else float(torch.as_tensor(v, dtype=torch.float32)[i])      # noqa: E731
    several = 0
    for i in range(rows):
        may = allowed(xs[i], pick(warm, i, 1.0), int(pick(k, i, 0)), pick(p, i, 1.0), pick(least, i, 0.0), pick(u, i, 0.0))
        assert got[i] in may, (i, got[i], sorted(may)[:5], len(may))
        several += len(may) > 1
    return got, several


@pytest.mark.parametrize("vocab,dtype", [(2, "f32"), (1000, "f16"), (50021, "bf16"), (131072, "f32"), (262145, "f16"), (393216, "f32"), (524289, "bf16"), (786432, "bf16")])
def test_what_weighs_next_to_nothing_is_not_drawn(mpq, cuda, vocab, dtype):
    """One token far above all others, at either end of the row or inside it: every random number draws it."""
    ends = [0.0, 2.0 ** -149, 1e-30, 1e-7, 2.0 ** -24, 0.5, 1 - 2.0 ** -23, 1 - 2.0 ** -24, 1.0]
    for at in (0, vocab // 3, vocab - 1):
        x = torch.zeros((len(ends), vocab))
        x[:, at] = 300.0
        to = lambda v: torch.full((len(ends),), v, device=cuda)                                # noqa: E731
        logits, u = x.to(TYPES[dtype]).to(cuda), torch.tensor(ends, device=cuda)
        k = torch.full((len(ends),), max(1, vocab // 2), dtype=torch.int32, device=cuda)
        for warm in (1.0, 3.0, 0.01):
            for rules in ({}, dict(top_p=to(1 - 2.0 ** -24)), dict(top_k=k), dict(top_k=k, top_p=to(1 - 2.0 ** -24)), dict(min_p=to(1e-30))):
                got = mpq.sample(logits, u, to(warm), **rules).tolist()
                assert got == [at] * len(ends), (at, warm, list(rules), got)


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("rows", [3, 200])
def test_tokens_forbidden_by_the_lowest_value(mpq, cuda, rows, dtype):
    """Never drawn beside allowed ones: with each rule, at both ends of the random numbers, inside a top-k that has more places than
    there are allowed tokens."""
    vocab, g = 20011, torch.Generator().manual_seed(3)
    x = torch.randn((rows, vocab), generator=g).to(TYPES[dtype])
    allow = torch.rand((rows, vocab), generator=g) < 0.0005
    allow[:, 0] = False
    allow[:, 9000] = True
    allow[1::3] = torch.rand((len(range(1, rows, 3)), vocab), generator=g) < 0.5
    allow[2::3] = False
    allow[2::3, 19000] = True
    logits, allow = torch.where(allow, x, torch.finfo(TYPES[dtype]).min).to(cuda), allow.to(cuda)
    to = lambda v, t=torch.float32: torch.full((rows,), v, dtype=t, device=cuda)               # noqa: E731
    for v in (0.0, 2.0 ** -149, 2.0 ** -24, 0.3, 1 - 2.0 ** -24, 1.0):
        for warm in (0.7, 5.0):
            for rules in ({}, dict(top_k=to(40, torch.int32)), dict(top_k=to(3000, torch.int32)), dict(top_k=to(19999, torch.int32)), dict(top_p=to(1 - 2.0 ** -24)),
                          dict(top_k=to(700, torch.int32), top_p=to(0.999)), dict(min_p=to(1e-30)), dict(top_k=to(15000, torch.int32), top_p=to(1 - 2.0 ** -24))):
                got = mpq.sample(logits, to(v), to(warm), **rules)
                assert allow[torch.arange(rows, device=cuda), got].all(), (v, warm, list(rules))


@pytest.mark.parametrize("vocab,dtype", [(300, "f32"), (9001, "f16"), (131072, "f32"), (151001, "bf16"), (786432, "bf16")])
def test_borders(mpq, cuda, vocab, dtype):
    """Flat, ordinary, steep and cold rows, top-p next to 0 and 1, whole numbers of equals, random numbers at the ends of their range."""
    g = torch.Generator().manual_seed(vocab)
    rows, several, drawn = 4, 0, 0
    for spread in (0.0, 0.01, 1.0, 4.0, 40.0):
        x = spread * torch.randn((rows, vocab), generator=g)
        u = torch.rand((rows,), generator=g)
        cases = [dict(), dict(u=[0.0, 2.0 ** -24, 1 - 2.0 ** -24, 1.0]), dict(p=[1 - 2.0 ** -24, 0.99999, 0.5, 2.0 ** -24]),
                 dict(p=[1 - 2.0 ** -24] * 4, u=[1 - 2.0 ** -24, 1 - 2.0 ** -20, 1e-7, 0.5]),
                 dict(warm=[0.5, 0.5, 2.0, 0.1], k=[vocab - 1, 100, 1000, vocab // 2], p=[1 - 2.0 ** -24, 0.99999, 0.999, 0.5], least=[0.0, 0.0, 1e-9, 1e-12])]
        for c in cases if vocab < 500000 else cases[:3]:
            c = dict(c)
            _, n = check(mpq, cuda, x, c.pop("u", u), dtype=dtype, **c)
            several, drawn = several + n, drawn + rows
    assert several <= drawn // 2                              # (most rows leave no choice)

"""Drawing tokens from logits, against the definition in 64 bits."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def draw(x, warm, k, p, least, u):
    """One row: the token, and whether a border lies so near a sum that either side of it is right."""
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if warm <= 0:
        return order[0], False
    if k > 0:
        order = order[:k]
    w = np.exp((x[order] - x[order[0]]) / warm)
    near = False
    if p < 1:
        upto = np.cumsum(w)
        goal = p * upto[-1]
        size = 1 + int((upto < goal).sum())
        near |= bool((np.abs(upto - goal) < 1e-10 * upto[-1]).any())
        order, w = order[:size], w[:size]
    if least > 0:
        near |= bool((np.abs(w / least - 1) < 1e-12).any() and least < 1)
        few = max(1, int((w >= least).sum()))
        order, w = order[:few], w[:few]
    at = np.argsort(order)
    upto = np.cumsum(w[at])
    goal = u * upto[-1]
    near |= bool((np.abs(upto[:-1] - goal) < 1e-10 * upto[-1]).any())
    return order[at][min(len(at) - 1, int((upto <= goal).sum()))], near


def check(mpq, cuda, x, u, warm=None, k=None, p=None, least=None, dtype="f32", open_ends=None):
    rows = x.shape[0]
    logits = x.to(TYPES[dtype]).to(cuda)
    to = lambda v, t=torch.float32: None if v is None else torch.as_tensor(v).to(t).to(cuda)      # noqa: E731
    logprob = torch.full((rows,), 7.0, device=cuda)
    got = mpq.sample(logits, to(u), to(warm), to(k, torch.int32), to(p), to(least), logprob=logprob)
    xs = logits.double().cpu().numpy()
    pick = lambda v, i, other: other if v is None else float(torch.as_tensor(v, dtype=torch.float32)[i])      # noqa: E731
    ambiguous = 0
    for i in range(rows):
        ref, near = draw(xs[i], pick(warm, i, 1.0), int(pick(k, i, 0)), pick(p, i, 1.0), pick(least, i, 0.0), pick(u, i, 0.0))
        ambiguous += near
        assert got[i].item() == ref or near, (i, got[i].item(), ref)
        # The share of the first of the order is exact, the others' sum is made of 32-bit terms.  With d a term's distance from the
        # first: d is rounded (d 2^-24 of the term), its product with log2 e too (d 2^-24; the constant is off by less than d 2^-25 of
        # it), and the fast exponential is off by 2^-22; a thread adds at most eight terms more than its share of the row (512 threads
        # or more), each addition off by 2^-24 of the sum.  Of the logarithm of 1 + rest that is the error over 1 + rest, and one rounding at the end.
        d = xs[i] - xs[i].max()
        terms = np.exp(d)
        terms[np.argmax(xs[i])] = 0.0
        off = (terms[terms > 0] * (2.5 * -d[terms > 0] + 4 + 8 + len(d) / 512)).sum() * 2.0 ** -24 / (1 + terms.sum())
        want = d[got[i].item()] - math.log1p(terms.sum())
        assert abs(logprob[i].item() - want) <= 2.0 ** -24 * abs(want) + off + 1e-15, (i, logprob[i].item(), want)
    assert ambiguous <= (1 + rows // 8 if open_ends is None else open_ends)
    return got


def bell(rows, vocab, seed, spread=3.0):
    g = torch.Generator().manual_seed(seed)
    return spread * torch.randn((rows, vocab), generator=g), torch.rand((rows,), generator=g), g


VOCABS = [1, 2, 3, 31, 32, 33, 255, 1000, 1023, 1025, 4097, 32000, 50021, 131072, 151001]


@pytest.mark.parametrize("dtype", list(TYPES))
@pytest.mark.parametrize("vocab", VOCABS)
def test_each_rule(mpq, cuda, vocab, dtype):
    rows = 5
    x, u, g = bell(rows, vocab, vocab)
    warm = 0.3 + torch.rand((rows,), generator=g)
    check(mpq, cuda, x, u, dtype=dtype)
    check(mpq, cuda, x, u, warm, dtype=dtype)
    check(mpq, cuda, x, u, warm * 0, dtype=dtype)
    check(mpq, cuda, x, u, warm, k=[1, 2, 50, vocab, vocab + 7], dtype=dtype)
    check(mpq, cuda, x, u, warm, p=[0.0, 0.3, 0.9, 0.999, 1.0], dtype=dtype)
    check(mpq, cuda, x, u, warm, least=[0.0, 0.01, 0.2, 1.0, 2.0], dtype=dtype)
    check(mpq, cuda, x, u, warm, [3, 1000, 0, 17, -1], [0.5, 0.95, 1.5, 0.8, 0.99], [0.0, 0.01, 0.1, 0.3, 1e-5], dtype=dtype)


@pytest.mark.parametrize("rows", [1, 2, 18, 19, 37, 74, 75, 148, 149, 300, 700])
def test_rows(mpq, cuda, rows):
    """However many blocks share a row."""
    for vocab, dtype in ((5000, "bf16"), (3001, "f32")):
        x, u, g = bell(rows, vocab, rows)
        some = lambda share, v, off: torch.where(torch.rand((rows,), generator=g) < share, v, torch.full((rows,), float(off)))      # noqa: E731
        warm = some(0.8, 0.2 + torch.rand((rows,), generator=g), 0.0)
        check(mpq, cuda, x, u, warm, some(0.5, torch.randint(1, 400, (rows,), generator=g).float(), 0).int(), some(0.5, torch.rand((rows,), generator=g), 1),
              some(0.5, 0.2 * torch.rand((rows,), generator=g), 0), dtype)


@pytest.mark.parametrize("vocab", [1, 7, 1024, 4096, 65536, 131072])
def test_equals_are_taken_in_the_order_of_their_index(mpq, cuda, vocab):
    """All logits alike, and two classes of equals: every border is a whole number, so exact."""
    rows = 6
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 0.99999, 0.5])
    flat = torch.full((rows, vocab), -2.5)
    got = check(mpq, cuda, flat, u * 0, dtype="bf16")
    assert not got.any()
    to = lambda v, t=torch.float32: torch.tensor(v, dtype=t, device=cuda)                      # noqa: E731
    for dtype in (torch.float32, torch.bfloat16):
        x = flat.to(cuda).to(dtype)
        got = mpq.sample(x, u.to(cuda))
        assert got.tolist() == [min(vocab - 1, int(float(v) * vocab)) for v in u]
        got = mpq.sample(x, u.to(cuda), top_p=to([0.5] * rows))
        kept = max(1, -(-vocab // 2))
        assert got.tolist() == [min(kept - 1, int(float(v) * kept)) for v in u]
        k = max(1, vocab // 3)
        got = mpq.sample(x, u.to(cuda), top_k=to([k] * rows, torch.int32))
        assert got.tolist() == [min(k - 1, int(float(v) * k)) for v in u]
        got = mpq.sample(x, u.to(cuda), top_k=to([k] * rows, torch.int32), top_p=to([0.25] * rows), min_p=to([1.0] * rows))
        kept = -(-k // 4)
        assert got.tolist() == [min(kept - 1, int(float(v) * kept)) for v in u]
        assert not mpq.sample(x, u.to(cuda), to([0.0] * rows)).any()
        y = x.clone()
        y[:, ::2] -= 1000.0                                   # every second one never
        got = mpq.sample(y, u.to(cuda), top_k=to([k] * rows, torch.int32)) if vocab > 1 else None
        if vocab > 1:
            n = min(k, vocab // 2)
            assert got.tolist() == [2 * min(n - 1, int(float(v) * n)) + 1 for v in u]


def test_signed_zeros_are_equal(mpq, cuda):
    x = torch.tensor([[-0.0, 0.0, -0.0, 0.0], [0.0, -0.0, 0.0, -0.0]], device=cuda)
    one = torch.ones(2, device=cuda)
    assert mpq.sample(x, one * 0.9, one * 0).tolist() == [0, 0]
    assert mpq.sample(x, one * 0.9, top_k=torch.tensor([2, 3], dtype=torch.int32, device=cuda)).tolist() == [1, 2]


@pytest.mark.parametrize("dtype", list(TYPES))
def test_masked_logits(mpq, cuda, dtype):
    """-infinity and the type's lowest value: most of a row, all of it but one, all of it."""
    rows, vocab = 6, 20011
    x, u, g = bell(rows, vocab, 5)
    x = x.to(TYPES[dtype]).float()
    low = torch.finfo(TYPES[dtype]).min
    mask = torch.rand((rows, vocab), generator=g) < 0.9
    for value in (-math.inf, low):
        y = torch.where(mask, value, x)
        y[1] = value
        y[1, 777] = 3.0
        got = check(mpq, cuda, y, u, dtype=dtype)
        assert got[1] == 777
        got = check(mpq, cuda, y, u, [0.7] * 6, [50] * 6, [0.9] * 6, [0.01] * 6, dtype=dtype)
        assert got[1] == 777
        for v in (0.0, 1.0 - 2.0 ** -24, 1.0, -3.0, 7.0):     # the first and the last one left, never a masked one
            got = mpq.sample(y.to(TYPES[dtype]).to(cuda), torch.full((rows,), v, device=cuda))
            if value == -math.inf:
                assert not mask[torch.arange(rows), got.cpu()][[0, 2, 3, 4, 5]].any()
    lp = torch.zeros(rows, device=cuda)
    gone = torch.full((rows, vocab), -math.inf, device=cuda, dtype=TYPES[dtype])
    assert mpq.sample(gone, u.to(cuda), logprob=lp).tolist() == [-1] * rows and torch.isnan(lp).all()
    assert mpq.sample(gone, u.to(cuda), torch.zeros(rows, device=cuda)).tolist() == [-1] * rows
    lowest = torch.full((rows, vocab), low, device=cuda, dtype=TYPES[dtype])
    assert mpq.sample(lowest, u.to(cuda) * 0, logprob=lp).tolist() == [0] * rows
    assert torch.allclose(lp, torch.full_like(lp, -math.log(vocab)))


def test_rows_that_cannot_be_drawn_from(mpq, cuda):
    rows, vocab = 9, 3000
    x, u, _ = bell(rows, vocab, 8)
    x, u = x.to(cuda), u.to(cuda)
    warm, k, p, least = torch.ones(rows, device=cuda), torch.full((rows,), 40, dtype=torch.int32, device=cuda), torch.full((rows,), 0.9, device=cuda), torch.zeros(rows, device=cuda)
    ref = mpq.sample(x, u, warm, k, p, least)
    x[1, 2999], x[2, 0], x[3, 5] = math.nan, math.inf, math.inf
    warm[3], warm[4], p[5], least[6], u[7] = 0.0, math.nan, math.nan, math.nan, math.nan
    lp = torch.zeros(rows, device=cuda)
    got = mpq.sample(x, u, warm, k, p, least, logprob=lp)
    assert got[[1, 2, 4, 5, 6, 7]].tolist() == [-1] * 6 and torch.isnan(lp[[1, 2, 4, 5, 6, 7]]).all()
    assert got[3] == 5 and got[0] == ref[0] and got[8] == ref[8]
    warm[:] = math.inf                                        # every token alike
    assert mpq.sample(x[8:], u[8:], warm[8:])[0] == int(float(u[8]) * vocab)
    warm[:] = 1e-30                                           # the first of the order
    assert mpq.sample(x[8:], u[8:], warm[8:])[0] == x[8].argmax()
    assert mpq.sample(x[8:], u[8:], -warm[8:])[0] == x[8].argmax()


@pytest.mark.parametrize("spread", [0.0, 1e-6, 0.01, 30.0, 3000.0])
def test_flat_and_steep_rows(mpq, cuda, spread):
    for dtype in ("f32", "bf16"):
        x, u, _ = bell(4, 40000, 3, spread)
        check(mpq, cuda, x + 11, u, None, [0, 100, 0, 20000], [1.0, 1.0, 0.6, 0.5], [0.0, 0.0, 0.0, 1e-9], dtype=dtype)


@pytest.mark.parametrize("rows,vocab", [(1, 131072), (1, 66001), (37, 20001), (300, 9001), (1, 3000)])
def test_however_many_stay(mpq, cuda, rows, vocab):
    """Numbers of kept tokens around what a block notes (1024 or 2048) and all blocks take (2048); ends of rows in any block."""
    x, u, _ = bell(rows, vocab, vocab, 1.0)
    for dtype in ("f32", "bf16"):
        for n in (900, 1000, 1024, 1100, 2000, 2048, 2100, 4000, 7000, 12000):
            if n < vocab:
                check(mpq, cuda, x[:9], u[:9], k=[n] * len(x[:9]), dtype=dtype)
                threshold = torch.exp(x.to(TYPES[dtype]).float().sort(1, descending=True).values[:, n] - x.to(TYPES[dtype]).float().max(1).values)
                check(mpq, cuda, x[:9], u[:9], least=threshold[:9] * 1.0001, dtype=dtype)
                w = torch.softmax(x[:9].to(TYPES[dtype]).double(), 1).sort(1, descending=True).values
                check(mpq, cuda, x[:9], u[:9], p=w[:, :n].sum(1), dtype=dtype)
    if rows > 9:                                              # ... with as many blocks to a row as there are for so many rows
        for n in (1024, 2048, 7000):
            check(mpq, cuda, x, u, k=[min(n, vocab - 1)] * rows)
            check(mpq, cuda, x, u, p=torch.softmax(x.double(), 1).sort(1, descending=True).values[:, :n].sum(1))


@pytest.mark.parametrize("vocab", [300, 9001, 131072])
def test_rules_at_the_ends_of_their_range(mpq, cuda, vocab):
    """top-p a step below 1 and a step above 0, temperatures from the smallest number to the largest, min-p of next to nothing."""
    x, u, _ = bell(5, vocab, vocab + 3)
    for dtype in ("f32", "f16"):
        for spread in (0.01, 1.0, 4.0):
            y = x * spread
            # (at the end of a steep row tokens weigh less than the 1e-10 of the sum by which a border counts as near: the first four rows)
            check(mpq, cuda, y, u, p=[1 - 2.0 ** -24, 1 - 2.0 ** -20, 0.9999, 0.99999, 1e-30], dtype=dtype, open_ends=4)
            check(mpq, cuda, y, u, [0.5] * 5, [vocab - 1] * 5, [1 - 2.0 ** -24, 0.99999, 0.5, 0.999, 2.0 ** -24], dtype=dtype, open_ends=4)
            check(mpq, cuda, y, u, p=[0.999] * 5, least=[1e-30, 1e-9, 1e-12, 1e-4, 2.0 ** -24], dtype=dtype)
            check(mpq, cuda, y, u, [1e4, 3e38, 100.0, 1e-30, 1e-3], dtype=dtype)
            check(mpq, cuda, y, u, [1e4, 3e38, 100.0, 1e-30, 1e-3], [40, 50, vocab // 2, 3, 9], [0.9, 0.5, 0.99, 0.9, 0.9], [0.0, 0.9, 0.5, 0.1, 1e-9], dtype=dtype)


def test_ordered_rows(mpq, cuda):
    """The largest logits side by side, with few threads of one block."""
    for vocab in (9000, 131072):
        x, u, _ = bell(4, vocab, 2)
        x = x.sort(1).values
        for y in (x, x.flip(1)):
            for k in (40, 700, 1500):
                check(mpq, cuda, y, u, [0.8] * 4, [k] * 4, [1.0, 0.9, 1.0, 0.5], [0.0, 0.0, 0.05, 0.0])
            check(mpq, cuda, y, u, p=[0.3, 0.9, 0.99, 0.9999])


def test_strides_outputs_and_odd_addresses(mpq, cuda):
    for vocab in (4096, 4099):
        for dtype in TYPES.values():
            wide = torch.randn((7, vocab + 5), device=cuda).to(dtype)
            wide[:, :1] = math.inf
            wide[:, vocab + 1:] = math.nan                    # outside the rows
            u = torch.rand(7, device=cuda)
            ref = mpq.sample(wide[:, 1:vocab + 1].contiguous(), u)
            out = torch.full((9,), -5, dtype=torch.int64, device=cuda)
            assert mpq.sample(wide[:, 1:vocab + 1], u, out=out[1:8]) is not None
            assert out.tolist() == [-5] + ref.tolist() + [-5]


def test_largest_vocabularies(mpq, cuda):
    for vocab, dtype in ((393216, "f32"), (786432, "bf16"), (786429, "f16")):
        x, u, _ = bell(2, vocab, 4, 2.0)
        check(mpq, cuda, x, u, [1.0, 0.8], [0, 5000], [0.9, 1.0], None, dtype)
        check(mpq, cuda, x, u, dtype=dtype)


def test_graphs_and_streams(mpq, cuda):
    x, u, _ = bell(20, 9000, 6)
    x, u = x.to(cuda), u.to(cuda)
    k, p = torch.full((20,), 60, dtype=torch.int32, device=cuda), torch.full((20,), 0.8, device=cuda)
    ref = mpq.sample(x, u, None, k, p)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        assert torch.equal(mpq.sample(x, u, None, k, p), ref)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = mpq.sample(x, u, None, k, p)
    graph.replay()
    assert torch.equal(out, ref)
    x.copy_(x.flip(1).contiguous())
    graph.replay()
    assert torch.equal(out, mpq.sample(x, u, None, k, p)) and not torch.equal(out, ref)


def test_frequencies(mpq, cuda):
    """Evenly spaced random numbers draw each token as often as its probability says, off by one at most."""
    n = 4096
    x = torch.tensor([0.0, 2.0, -1.0, 1.0, -math.inf, 0.5], device=cuda)
    u = (torch.arange(n, device=cuda) + 0.5) / n
    got = mpq.sample(x.expand(n, 6).contiguous(), u)
    share = torch.softmax(x.double(), 0) * n
    assert (torch.bincount(got, minlength=6).double() - share).abs().max() <= 1


def test_tensors_that_do_not_fit(mpq, cuda):
    x, u = torch.randn((4, 100), device=cuda), torch.rand(4, device=cuda)
    for bad in (dict(uniform=u[:3]), dict(uniform=u.double()), dict(uniform=u.cpu()), dict(logits=x.double()), dict(logits=x.T.contiguous().T),
                dict(temperature=u[:2]), dict(top_k=u), dict(top_p=u.half()), dict(min_p=u.cpu()), dict(out=torch.zeros(4, dtype=torch.int32, device=cuda)),
                dict(logprob=torch.zeros(3, device=cuda))):
        args = dict(logits=x, uniform=u)
        args.update(bad)
        with pytest.raises(ValueError):
            mpq.sample(**args)
    assert mpq.sample(x[:0], u[:0]).shape == (0,)

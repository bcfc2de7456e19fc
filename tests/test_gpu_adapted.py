"""Product of level bytes with an adapter per request, against 64-bit arithmetic."""
import math

import numpy as np
import pytest
import torch

from tests.test_gpu_linear_levels import TYPES, UNIT, activate, operand

pytestmark = pytest.mark.gpu

EXTREMES = {"f16": torch.float16, "bf16": torch.bfloat16}


def low_rank(cuda, adapters, rank, n, k, dtype, seed, scaled=True):
    g = torch.Generator().manual_seed(seed)
    down = (torch.randn((adapters, rank, k), generator=g) / math.sqrt(k)).to(EXTREMES[dtype])
    up = torch.randn((adapters, n, rank), generator=g).to(EXTREMES[dtype])
    return down, up, 0.5 + torch.rand((adapters,), generator=g) if scaled else None


class Case:
    """`lens` tokens per sequence, `ids` their adapters, `tail` tokens of no sequence behind."""

    def __init__(self, mpq, cuda, lens, ids, n, k, rank, dtype="f16", adapters=4, tail=0, a_bits=8, w_bits=8, seed=1, scaled=True):
        self.mpq, self.cuda, self.n, self.k = mpq, cuda, n, k
        self.m = sum(lens) + tail
        self.a, self.qa, self.sa = operand(mpq, cuda, self.m, k, a_bits, seed)
        self.w, self.qw, self.sw = operand(mpq, cuda, n, k, w_bits, seed + 1, std=2.0 / math.sqrt(k))
        self.down, self.up, self.factor = low_rank(cuda, adapters, rank, n, k, dtype, seed + 2, scaled)
        self.low = mpq.adapters(self.down.to(cuda), self.up.to(cuda), None if self.factor is None else self.factor.to(cuda))
        self.starts = np.concatenate([[0], np.cumsum(lens)]).astype(np.int64)
        self.ids = list(ids)

    def run(self, **kw):
        ints = lambda v: torch.tensor(v, dtype=torch.int32, device=self.cuda)                  # noqa: E731
        return self.mpq.linear_adapted(self.a, self.w, self.low, ints(self.starts), ints(self.ids), **kw)

    def sums(self):
        """The product, and each adapter's part, with the sizes of what is added up in them."""
        acc = self.qa.astype(np.float64) @ self.qw.T.astype(np.float64)
        f = acc * (self.sa[:, None] * self.sw[None, :])
        delta, size = np.zeros_like(f), np.zeros_like(f)
        for b, i in enumerate(self.ids):
            if 0 <= i < len(self.down):
                rows = slice(int(self.starts[b]), int(self.starts[b + 1]))
                x, d, u = self.qa[rows] * self.sa[rows, None], self.down[i].double().numpy(), self.up[i].double().numpy()
                c = 1.0 if self.factor is None else float(self.factor[i])
                delta[rows] = c * (x @ d.T) @ u.T
                size[rows] = c * (np.abs(x) @ np.abs(d.T)) @ np.abs(u.T)
        return f, delta, size

    def check(self, act="none", out="f32", bias=False, residual=False):
        g = torch.Generator().manual_seed(9)
        b = torch.randn((self.n,), generator=g) if bias else None
        r = torch.randn((self.m, self.n), generator=g).to(TYPES[out]) if residual else None
        got = self.run(bias=None if b is None else b.to(self.cuda), act=act, residual=None if r is None else r.to(self.cuda), dtype=TYPES[out])
        f, delta, size = self.sums()
        whole = np.abs(f) + np.abs(delta)
        f = f + delta
        if bias:
            f = f + b.numpy().astype(np.float64)
            whole = whole + np.abs(b.numpy())
        y = activate(f, act)
        ref = y + r.double().numpy() if residual else y
        # As for the product without adapters, and the adapter's own sums: their terms are exact products or fp32 ones, k and
        # rank of them; a sum of N terms in any order is off by at most N 2^-24 of the terms' sizes, a truncating one by twice that.
        # Of random signs they come nowhere near it: 4 + sqrt(N) / 4 units of the sizes are allowed (k = 4100: 20).
        terms = 4 + math.sqrt(self.k + 128) / 4
        tol = UNIT[out] * np.abs(ref) + 16 * 2.0 ** -24 * (whole + np.abs(ref)) + 1.2 * terms * 2.0 ** -24 * size + (2.0 ** -25 if out == "f16" else 0)
        err = np.abs(got.double().cpu().numpy() - ref)
        assert got.dtype == TYPES[out] and got.shape == (self.m, self.n)
        assert np.all(err <= tol), (err - tol).max()
        return got


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("lens,ids,n,k,rank", [
    ([1], [0], 1, 1, 1), ([1], [3], 64, 16, 16), ([2], [1], 5, 33, 7), ([1, 1, 1], [0, -1, 2], 130, 100, 16), ([3, 0, 5], [2, 1, 0], 1000, 512, 32),
    ([9], [1], 257, 4100, 24), ([8, 8], [3, 3], 64, 128, 64), ([1] * 17, [i % 4 for i in range(17)], 100, 640, 16), ([16, 17], [1, -1], 4096, 64, 128),
    ([30, 1, 1, 33], [0, 1, 2, 3], 31, 31, 48), ([128], [2], 256, 256, 16), ([100, 29], [0, 1], 257, 272, 80), ([1, 250, 5], [0, 1, 2], 512, 1040, 8),
    ([600, 400], [1, 0], 120, 48, 16), ([299, 1], [2, 3], 77, 2050, 112)])
def test_sizes(mpq, cuda, lens, ids, n, k, rank, dtype):
    c = Case(mpq, cuda, lens, ids, n, k, rank, dtype, seed=n + k)
    c.check()
    c.check("silu", "bf16", True, True)


# more tiles than multiprocessors: CTA pairs; pieces that end inside tiles, single tokens between them, rows of no sequence
@pytest.mark.parametrize("lens,ids,tail,n,k,rank", [([513], [1], 0, 2177, 272, 16), ([300, 1, 1, 1, 200, 270], [0, 1, -1, 2, 3, 0], 4, 1601, 100, 64),
                                                    ([1] * 600, [i % 5 - 1 for i in range(600)], 3, 2400, 130, 16), ([2000, 2097], [3, 0], 0, 1001, 130, 32),
                                                    ([65, 63], [0, 9], 2, 9001, 48, 128), ([1000, 24], [-1, -1], 0, 2560, 512, 16)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_many_rows(mpq, cuda, lens, ids, tail, n, k, rank, dtype):
    c = Case(mpq, cuda, lens, ids, n, k, rank, dtype, tail=tail, seed=n)
    c.check("none", "f32", True, False)
    c.check("gelu_tanh", "f16", True, True)


# both sides of the rule that chooses the form: rows, and tokens of a sequence on average
@pytest.mark.parametrize("lens,n,k,rank", [([32], 130, 70, 16), ([33], 130, 70, 16), ([12] * 3, 300, 512, 32), ([12, 12, 13], 300, 512, 32), ([5] * 30, 700, 96, 64),
                                           ([12] * 11, 257, 1040, 128), ([13] * 11, 257, 1040, 128), ([64], 3, 5, 16), ([0] * 50 + [200], 520, 260, 48),
                                           ([256], 128, 128, 128), ([40, 0, 0, 1], 9001, 17, 16), ([38], 150, 6656, 16), ([38], 150, 6657, 16), ([66], 70, 20000, 16)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_few_rows_of_long_and_short_sequences(mpq, cuda, lens, n, k, rank, dtype):
    c = Case(mpq, cuda, lens, [(i + 1) % 5 - 1 for i in range(len(lens))], n, k, rank, dtype, tail=2, seed=n + k)
    c.check("none", "f32")
    c.check("silu", "bf16", True, True)


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
@pytest.mark.parametrize("out", list(TYPES))
def test_epilogues(mpq, cuda, act, out):
    for lens, n in (([1], 200), ([15, 5], 200), ([140, 10], 200), ([700], 1601)):
        c = Case(mpq, cuda, lens, [2, 0][:len(lens)], n, 320, 16, "bf16", seed=n)
        for bias, residual in ((False, False), (True, True)):
            c.check(act, out, bias, residual)


@pytest.mark.parametrize("a_bits,w_bits", [(1, 1), (2, 8), (4, 4), (8, 3), (7, 5)])
def test_widths(mpq, cuda, a_bits, w_bits):
    for lens, n in (([5, 1], 100), ([300], 2000)):
        Case(mpq, cuda, lens, [1, 0][:len(lens)], n, 200, 16, "bf16", a_bits=a_bits, w_bits=w_bits).check()
        Case(mpq, cuda, lens, [1, 0][:len(lens)], n, 200, 32, "f16", a_bits=a_bits, w_bits=w_bits, scaled=False).check()


@pytest.mark.parametrize("m,n", [(1, 300), (40, 300), (130, 9001), (600, 1601)])
def test_rows_without_an_adapter_are_the_plain_product(mpq, cuda, m, n):
    """Bit for bit: ids outside the adapters, rows before the first and behind the last sequence."""
    c = Case(mpq, cuda, [m], [-1], n, 208, 32)
    ref = mpq.linear_levels(c.a, c.w, act="gelu", dtype=torch.bfloat16)
    for ids in ([-1], [4], [-(2 ** 31)], [2 ** 31 - 1]):
        c.ids = ids
        assert torch.equal(c.run(act="gelu", dtype=torch.bfloat16), ref)
    c.ids, inside = [1], m // 3
    c.starts = np.array([inside, inside + (m - inside) // 2])
    got = c.run(act="gelu", dtype=torch.bfloat16)
    outside = torch.ones(m, dtype=torch.bool)
    outside[c.starts[0]:c.starts[1]] = False
    assert torch.equal(got[outside], ref[outside])
    c.starts, c.ids = np.array([0]), []                      # no sequences at all
    assert torch.equal(c.run(act="gelu", dtype=torch.bfloat16), ref)


def test_what_is_not_finite_stays_with_its_rows_and_columns(mpq, cuda):
    for lens, n in (([3, 2, 4], 300), ([300, 300, 100], 1601)):
        c = Case(mpq, cuda, lens, [0, 1, 2], n, 64, 16)
        ref = c.run()
        c.low.up[1, 7, 3] = math.nan
        c.low.up[3] = math.nan                               # of nobody
        c.low.down[3] = math.nan
        got = c.run()
        rows = slice(lens[0], lens[0] + lens[1])
        assert torch.isnan(got[rows, 7]).all()
        got[rows, 7] = ref[rows, 7]
        assert torch.equal(got, ref)
        c.low.down[2, 0, 5] = math.inf
        got = c.run()
        at = sum(lens[:2])
        assert not torch.isfinite(got[at:]).any() and torch.isfinite(got[:lens[0]]).all()


@pytest.mark.parametrize("lens", [[5], [9, 1, 30], [200, 340, 60]])
def test_large_and_small_adapters_keep_their_precision(mpq, cuda, lens):
    """An adapter's inner sums may lie far outside the range of 16 bits while its output does not."""
    for big in (1e6, 1e-6):
        c = Case(mpq, cuda, lens, list(range(len(lens))), 1300, 512, 16, "bf16")
        c.down, c.up = (c.down.float() * big).bfloat16(), (c.up.float() / big).bfloat16()
        c.low = mpq.adapters(c.down.to(cuda), c.up.to(cuda), c.factor.to(cuda))
        c.check()
        c = Case(mpq, cuda, lens, list(range(len(lens))), 1300, 512, 16, "f16")
        c.factor = c.factor * big
        c.low = c.low._replace(scale=c.factor.to(cuda))
        c.check()


def test_strides_outputs_and_workspaces(mpq, cuda):
    for lens, n in (([7], 333), ([400, 233], 1601)):
        c = Case(mpq, cuda, lens, [2, 1][:len(lens)], n, 100, 16)
        m = sum(lens)
        res = torch.randn((m, n + 3), device=cuda, dtype=torch.float16)
        ref = c.run(residual=res[:, 1:n + 1], dtype=torch.float16)
        wide = torch.full((m, n + 9), 7.0, device=cuda, dtype=torch.float16)
        ws = torch.empty(mpq.linear_adapted_workspace(m, 16), dtype=torch.uint8, device=cuda)
        got = c.run(residual=res[:, 1:n + 1], out=wide[:, 5:n + 5], workspace=ws)
        assert torch.equal(got, ref) and (wide[:, :5] == 7).all() and (wide[:, n + 5:] == 7).all()
        inplace = res.clone()
        c.run(residual=inplace[:, 1:n + 1], out=inplace[:, 1:n + 1])
        assert torch.equal(inplace[:, 1:n + 1], ref) and torch.equal(inplace[:, :1], res[:, :1]) and torch.equal(inplace[:, n + 1:], res[:, n + 1:])
        with pytest.raises(mpq.MpqError):
            c.run(workspace=ws[:-16])


def test_runs_repeat_and_graphs_replay(mpq, cuda):
    """On another stream, twice, and captured with new activations and ids underneath."""
    for lens, n in (([1, 1, 2], 500), ([300, 1, 400], 1601)):
        c = Case(mpq, cuda, lens, [1, -1, 0], n, 320, 32, "bf16")
        starts, ids = (torch.tensor(v, dtype=torch.int32, device=cuda) for v in (c.starts, c.ids))
        ref = mpq.linear_adapted(c.a, c.w, c.low, starts, ids)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            assert torch.equal(mpq.linear_adapted(c.a, c.w, c.low, starts, ids), ref)
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = mpq.linear_adapted(c.a, c.w, c.low, starts, ids)
        graph.replay()
        assert torch.equal(out, ref)
        ids.copy_(torch.tensor([3, 2, -1], dtype=torch.int32))
        c.a.bytes.copy_(c.a.bytes.flip(0).contiguous())
        c.a.sums.copy_(c.a.sums.flip(0).contiguous())
        graph.replay()
        assert torch.equal(out, mpq.linear_adapted(c.a, c.w, c.low, starts, ids)) and not torch.equal(out, ref)


def test_tensors_that_do_not_fit(mpq, cuda):
    c = Case(mpq, cuda, [3, 2], [0, 1], 40, 64, 16)
    starts, ids = (torch.tensor(v, dtype=torch.int32, device=cuda) for v in (c.starts, c.ids))
    call = lambda low=c.low, starts=starts, ids=ids, **kw: mpq.linear_adapted(c.a, c.w, low, starts, ids, **kw)      # noqa: E731
    call()
    for bad in (dict(low=c.low._replace(k=63)), dict(low=c.low._replace(up=c.low.up[:, :39])), dict(low=c.low._replace(up=c.low.up.bfloat16())),
                dict(low=c.low._replace(down=c.low.down[:, :, :48])), dict(low=c.low._replace(scale=c.low.scale[:3])), dict(starts=starts[:2]),
                dict(ids=ids.long()), dict(starts=starts.cpu()), dict(act="tanh"), dict(workspace=torch.empty(10 ** 6, dtype=torch.uint8))):
        with pytest.raises(ValueError):
            call(**bad)
    with pytest.raises(ValueError):
        call(low=c.low._replace(down=c.low.down.float(), up=c.low.up.float()), dtype=torch.int32)
    with pytest.raises(mpq.MpqError):
        call(low=c.low._replace(down=c.low.down.float(), up=c.low.up.float()))

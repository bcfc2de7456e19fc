"""The paged cache on levels: writing, reading back, and the attention of new tokens over it."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def rand(shape, seed, scale=1.0):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale


def quantize(x, bits):
    """(levels, ranges) of [..., dim] by the quantizer's 32-bit rule."""
    x = x.float().numpy()
    s = np.abs(np.where(np.isnan(x), 0, x)).max(-1)
    H, half_L = 1 << (bits - 1), np.float32(((1 << bits) - 1) / 2)
    inv = np.zeros_like(s)
    ok = np.isfinite(s) & (s > 0)
    inv[ok] = np.float32(1) / s[ok]
    with np.errstate(invalid="ignore", over="ignore"):
        y = (x * inv[..., None]) * half_L
    return np.floor(np.clip(np.where(np.isnan(y), np.float32(0), y), -H, H - 0.5)).astype(np.int64) + H, s


def unpack(held, bits):
    held = held.cpu().numpy().astype(np.int64)
    return held if bits == 8 else np.stack((held & 15, held >> 4), -1).reshape(*held.shape[:-1], -1)


# ------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("name", list(TYPES))
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 32, 1), (5, 3, 64, 16), (33, 2, 96, 7), (64, 8, 128, 24), (10, 1, 256, 128), (7, 5, 160, 3)])
def test_write_and_read(mpq, cuda, bits, name, tokens, heads, dim, page):
    pages = 2 * tokens // page + 2
    cache = mpq.level_cache(pages, heads, page, dim, bits, cuda)
    for t in (cache.k, cache.v):
        t.fill_(0xA5)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(-7.0)
    before = [t.clone() for t in cache[:4]]
    k, v = rand((tokens, heads, dim), 1).to(TYPES[name]), rand((tokens, heads, dim), 2, 3.0).to(TYPES[name])
    slots = torch.randperm(pages * page, generator=torch.Generator().manual_seed(tokens))[:tokens]
    if tokens > 4:
        slots[1], slots[4] = -1, pages * page          # outside the cache on both sides
    mpq.cache_write(cache, k.to(cuda), v.to(cuda), slots.to(cuda))
    kept = [i for i in range(tokens) if 0 <= slots[i] < pages * page]
    touched = np.zeros((pages, page), dtype=bool)
    back = mpq.cache_read(cache, slots.to(cuda), torch.float32)
    for x, held, scale, old, old_s, got in ((k, cache.k, cache.k_scale, before[0], before[1], back[0]),
                                            (v, cache.v, cache.v_scale, before[2], before[3], back[1])):
        u, s = quantize(x, bits)
        have, have_s = unpack(held, bits), scale.cpu().numpy()
        want = np.zeros((tokens, heads, dim), dtype=np.float32)
        L = (1 << bits) - 1
        for i in kept:
            p, o = divmod(int(slots[i]), page)
            touched[p, o] = True
            assert np.array_equal(have[p, :, o], u[i]) and np.array_equal(have_s[p, :, o], s[i])
            want[i] = (2 * u[i] - L).astype(np.float32) * (s[i] / np.float32(L))[:, None]
        assert np.array_equal(got.cpu().numpy(), want)
        # nothing else changed
        same = torch.from_numpy(~touched).to(cuda)[:, None, :].expand(pages, heads, page)
        assert torch.equal(held[same], old[same]) and torch.equal(scale[same], old_s[same])
    narrow = mpq.cache_read(cache, slots.to(cuda), TYPES[name])
    assert torch.equal(narrow[0], back[0].to(TYPES[name])) and torch.equal(narrow[1], back[1].to(TYPES[name]))


def test_strided_keys_and_values(mpq, cuda):
    """Keys and values as slices of one projection's output, also at odd offsets, and broadcast heads."""
    qkv = rand((9, 5 * 64 + 3), 3).to(torch.bfloat16).to(cuda)
    slots = torch.arange(9, device=cuda)
    for at in (0, 1, 3):
        k, v = (qkv[:, at + i * 128:at + i * 128 + 128].unflatten(1, (2, 64)) for i in (0, 1))
        a, b = (mpq.level_cache(2, 2, 8, 64, 8, cuda) for _ in range(2))
        mpq.cache_write(a, k, v, slots)
        mpq.cache_write(b, k.contiguous(), v.contiguous(), slots)
        assert all(torch.equal(x, y) for x, y in zip(a[:4], b[:4]))
        out = torch.zeros((9, 5 * 64 + 3), dtype=torch.bfloat16, device=cuda)
        views = [out[:, at + i * 128:at + i * 128 + 128].unflatten(1, (2, 64)) for i in (0, 1)]
        mpq.cache_read(a, slots, torch.bfloat16, *views)
        ref = mpq.cache_read(a, slots, torch.bfloat16)
        assert torch.equal(views[0], ref[0]) and torch.equal(views[1], ref[1])
        assert not out[:, at + 256:].any()
    one = rand((9, 1, 64), 4).to(cuda).expand(9, 2, 64)
    c = mpq.level_cache(2, 2, 8, 64, 4, cuda)
    mpq.cache_write(c, one, one, slots)
    assert torch.equal(c.k[:, 0], c.k[:, 1])


def test_write_special_values(mpq, cuda):
    k = rand((4, 1, 32), 1)
    k[0] = 0
    k[1, 0, 5] = float("nan")
    k[2, 0, 5] = float("inf")
    cache = mpq.level_cache(1, 1, 4, 32, 8, cuda)
    mpq.cache_write(cache, k.to(cuda), k.to(cuda), torch.arange(4, device=cuda))
    u, s = quantize(k, 8)
    assert np.array_equal(unpack(cache.k, 8)[0, 0], u[:, 0]) and np.array_equal(cache.k_scale.cpu().numpy()[0, 0], s[:, 0])
    back, _ = mpq.cache_read(cache, torch.arange(4, device=cuda), torch.float32)
    assert (back[0] == 0).all() and torch.isfinite(back[1]).all() and torch.isinf(back[2]).all()


def test_no_tokens(mpq, cuda):
    cache = mpq.level_cache(1, 2, 4, 64, 8, cuda)
    none = torch.empty((0, 2, 64), device=cuda)
    mpq.cache_write(cache, none, none, torch.empty(0, dtype=torch.int64, device=cuda))
    assert mpq.cache_read(cache, torch.empty(0, dtype=torch.int64, device=cuda), torch.float16)[0].shape == (0, 2, 64)
    q = torch.empty((0, 4, 64), dtype=torch.float16, device=cuda)
    one = torch.zeros(2, dtype=torch.int32, device=cuda)
    assert mpq.cache_attention(q, cache, one, one[:1], one[:1, None], 0, 4).shape == (0, 4, 64)


# ------------------------------------------------------------------------------------------ attention
class Case:
    """A batch of sequences over a shuffled cache; pages that no sequence owns hold NaN ranges and noise."""

    def __init__(self, mpq, cuda, q_lens, kv_lens, heads, kv_heads, dim, bits, page, dtype, seed=0, max_pages=None):
        self.q_lens, self.kv_lens, self.bits, self.page, self.dtype = q_lens, kv_lens, bits, page, dtype
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        rng = np.random.default_rng(seed)
        used = [-(-n // page) for n in kv_lens]
        pages = sum(used) + 3
        order = rng.permutation(pages)
        per = max_pages or max(1, max(used, default=1))
        self.table = np.full((len(kv_lens), per), -1, dtype=np.int32)
        u = rng.integers(0, 1 << bits, (2, pages, kv_heads, page, dim))
        s = rng.uniform(0.2, 2.5, (2, pages, kv_heads, page)).astype(np.float32)
        free = np.ones((pages, page), dtype=bool)
        at = 0
        for b, n in enumerate(kv_lens):
            self.table[b, :used[b]] = order[at:at + used[b]]
            for j in range(n):
                free[self.table[b, j // page], j % page] = False
            at += used[b]
        s[:, np.broadcast_to(free[:, None, :], (pages, kv_heads, page))] = np.nan
        self.u, self.s = u, s
        starts = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.starts = starts
        self.q = rand((int(starts[-1]), heads, dim), seed + 1, 1.3).to(dtype)
        self.device = cuda
        self.mpq = mpq

    def cache(self):
        held = self.u.astype(np.uint8) if self.bits == 8 else (self.u[..., 0::2] | (self.u[..., 1::2] << 4)).astype(np.uint8)
        t = [torch.from_numpy(held[i].copy()).to(self.device) for i in (0, 1)]
        s = [torch.from_numpy(self.s[i].copy()).to(self.device) for i in (0, 1)]
        return self.mpq.LevelCache(t[0], s[0], t[1], s[1], self.bits)

    def run(self, causal=True, window=0, scale=None, q=None, **kw):
        q = self.q.to(self.device) if q is None else q
        lse = torch.full((q.shape[0], self.heads), 7.0, device=self.device)
        out = self.mpq.cache_attention(q, self.cache(), torch.from_numpy(self.starts).to(self.device),
                                       torch.tensor(self.kv_lens, dtype=torch.int32, device=self.device),
                                       torch.from_numpy(self.table).to(self.device), kw.pop("max_q", max(self.q_lens)),
                                       kw.pop("max_kv", max(self.kv_lens)), causal=causal, window=window, scale=scale, lse=lse, **kw)
        return out, lse

    def check(self, causal=True, window=0, scale=None, **kw):
        """Tolerance: weights are rounded to fp16 (2^-11 of each, and 2^-25 of the row's largest contribution for those
        below 2^-14 of it), scores carry 2^-19 of their own size (fp32 sums of exact products, three products, the
        logarithm of a range), which moves a weight by that much, and the result is rounded once."""
        out, lse = self.run(causal, window, scale, **kw)
        out, lse = out.double().cpu().numpy(), lse.double().cpu().numpy()
        L = (1 << self.bits) - 1
        scale = self.dim ** -0.5 if scale is None else scale
        unit = 2.0 ** -11 if self.dtype == torch.float16 else 2.0 ** -8
        group = self.heads // self.kv_heads
        for b, (nq, nk) in enumerate(zip(self.q_lens, self.kv_lens)):
            if nq == 0:
                continue
            j = np.arange(nk)
            p, o = self.table[b, j // self.page], j % self.page
            pos = nk - nq + np.arange(nq)
            seen = np.broadcast_to(p >= 0, (nq, nk)).copy()
            if causal:
                seen &= j[None] <= pos[:, None]
            if window:
                seen &= j[None] > pos[:, None] - window
            for h in range(self.heads):
                kv = [(2 * self.u[i][p, h // group, o] - L) * (self.s[i][p, h // group, o].astype(np.float64) / L)[:, None] for i in (0, 1)]
                q = self.q[self.starts[b]:self.starts[b + 1], h].double().numpy()
                with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
                    x = np.where(seen, (q @ np.where(np.isfinite(kv[0]), kv[0], 0).T) * scale, -np.inf)
                    m = x.max(1, keepdims=True, initial=-np.inf)
                    w = np.where(seen, np.exp(x - np.where(np.isinf(m), 0, m)), 0)
                    den = w.sum(1)
                    v = np.where(np.isfinite(kv[1]), kv[1], 0)
                    ref = np.where(den[:, None] > 0, w @ v / np.where(den > 0, den, 1)[:, None], 0)
                    spread = np.where(den[:, None] > 0, w @ np.abs(v) / np.where(den > 0, den, 1)[:, None], 0)
                    ref_lse = np.log(den) + np.where(np.isinf(m), 0, m)[:, 0]
                    contribution = np.where(seen, w * np.abs(v).max(1)[None], 0) if nk else np.zeros((nq, 1))
                big = np.where(den > 0, contribution.max(1, initial=0) / np.where(den > 0, den, 1), 0)
                xs = np.abs(np.where(seen, x, 0)).max(1, initial=0)
                got, got_lse = out[self.starts[b]:self.starts[b + 1], h], lse[self.starts[b]:self.starts[b + 1], h]
                tol = unit * np.abs(ref) + (2.0 ** -11 + 2.0 ** -18 + 2.0 ** -18 * xs[:, None]) * spread + (nk * 2.0 ** -25 * big)[:, None] + 2.0 ** -24
                assert np.all(np.abs(got - ref) <= tol), (b, h, np.abs(got - ref).max(), tol.min())
                dead = den == 0
                assert np.all(np.isneginf(got_lse[dead])) and np.all(got[dead] == 0)
                live = ~dead
                assert np.all(np.abs(got_lse - ref_lse)[live] <= 2.0 ** -18 * (1 + xs[live] + np.abs(ref_lse[live])))


HEADS = [(1, 1), (4, 1), (8, 8), (6, 2), (32, 4), (20, 1)]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", HEADS)
def test_single_tokens(mpq, cuda, bits, dim, heads, kv_heads):
    lens = [1, 2, 31, 32, 33, 127, 128, 129, 300, 511, 1000]
    Case(mpq, cuda, [1] * len(lens), lens, heads, kv_heads, dim, bits, 16, torch.bfloat16).check()


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", [(2, 2), (4, 1), (6, 2), (16, 1)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_chunks(mpq, cuda, bits, dim, heads, kv_heads, dtype):
    Case(mpq, cuda, [5, 1, 0, 130, 77, 64], [5, 200, 50, 130, 400, 65], heads, kv_heads, dim, bits, 24, TYPES[dtype]).check()


@pytest.mark.parametrize("page", [1, 3, 8, 24, 100, 128, 1000])
def test_page_sizes(mpq, cuda, page):
    c = Case(mpq, cuda, [1, 40, 3], [77, 150, 260], 4, 2, 64, 8, page, torch.float16)
    c.check()
    Case(mpq, cuda, [1, 1], [277, 515], 4, 2, 128, 4, page, torch.bfloat16).check()


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 2, 33, 128, 200, 100000])
def test_masks(mpq, cuda, causal, window):
    Case(mpq, cuda, [1, 150, 7, 300], [333, 150, 513, 700], 4, 2, 64, 8, 16, torch.bfloat16).check(causal, window)
    Case(mpq, cuda, [1, 2, 3], [333, 150, 513], 4, 2, 128, 4, 16, torch.float16).check(causal, window)


@pytest.mark.parametrize("dim", [64, 128])
def test_rows_that_see_nothing(mpq, cuda, dim):
    """More new tokens than context (their positions are negative), no context at all, and pages outside the cache."""
    Case(mpq, cuda, [5, 3, 140], [2, 0, 7], 4, 2, dim, 8, 16, torch.float16).check()
    Case(mpq, cuda, [1, 1], [0, 3], 4, 2, dim, 4, 16, torch.bfloat16).check()
    for q_lens in ([1, 1], [9, 200]):
        c = Case(mpq, cuda, q_lens, [40, 300], 4, 2, dim, 8, 16, torch.bfloat16)
        c.table[0, :] = -1                               # nothing of the first sequence is there
        c.table[1, 2] = 10 ** 6                          # a hole in the second
        c.table[1, 2:3] = -5
        c.check()


@pytest.mark.parametrize("q_lens,kv_lens", [([1], [5000]), ([1, 1, 1], [4000, 64, 2500]), ([20], [3000]), ([200, 1], [3000, 2000])])
@pytest.mark.parametrize("bits", [8, 4])
def test_split_contexts_and_launch_hints(mpq, cuda, q_lens, kv_lens, bits):
    """The caller's bounds choose the launch only: far too small and far too large ones give right sums."""
    c = Case(mpq, cuda, q_lens, kv_lens, 8, 2, 128, bits, 32, torch.bfloat16)
    c.check()
    c.check(max_kv=100000)
    c.check(max_kv=1)
    c.check(max_q=1)
    c.check(max_q=5000)
    c.check(window=700)


@pytest.mark.parametrize("q_lens,kv_lens,heads,kv_heads", [
    ([1], [900], 32, 8), ([1, 1, 1], [700, 0, 40], 8, 2), ([1, 0, 1], [1024, 5, 129], 5, 5), ([2, 1], [1000, 200], 16, 2),
    ([70], [4000], 8, 2), ([300, 1, 2], [1500, 30, 0], 6, 2), ([40, 33], [2100, 33], 20, 1)])
@pytest.mark.parametrize("dim,bits,dtype", [(128, 8, "bf16"), (64, 4, "f16")])
def test_splits_of_one_cluster(mpq, cuda, q_lens, kv_lens, heads, kv_heads, dim, bits, dtype):
    """Few enough splits join without a workspace: contexts that use all of them, some, one and none."""
    assert mpq.cache_attention_workspace(sum(q_lens), len(q_lens), heads, kv_heads, dim, max(q_lens), max(kv_lens)) == 0
    c = Case(mpq, cuda, q_lens, kv_lens, heads, kv_heads, dim, bits, 24, TYPES[dtype])
    c.check()
    c.check(causal=False)
    c.check(window=600)
    c.check(window=50)


def test_sizes_past_the_call_need_no_workspace(mpq, cuda):
    assert mpq.cache_attention_workspace(2 ** 62, 2 ** 30, 8, 2, 128, 2 ** 62, 2 ** 62) == 0
    assert mpq.cache_attention_workspace(1, 1, 8, 2, 128, 2 ** 62, 2 ** 62) > 0


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("q_len", [1, 4, 40])
def test_long_contexts_keep_their_precision(mpq, cuda, q_len, bits):
    """Over 16,000 tokens the result is an average some hundred times smaller than the values, and sums that carried more
    than the levels themselves (an offset, say) would lose it.  fp16: rounding the result moves it by at most 2^-11 of its
    size, 2^-11 / sqrt(3) = 2.8e-4 of it in the root mean square, and rounding each weight does the same to sums of random
    sign: 4e-4 together, 6e-4 with the scores' own errors."""
    c = Case(mpq, cuda, [q_len], [16000], 4, 1, 64, bits, 16, torch.float16)
    out, _ = c.run(scale=0.01, max_kv=1)                     # nearly equal weights, and no split of the context
    j = np.arange(16000)
    p, o, L = c.table[0, j // 16], j % 16, (1 << bits) - 1
    k, v = ((2 * c.u[i][p, 0, o] - L) * (c.s[i][p, 0, o].astype(np.float64) / L)[:, None] for i in (0, 1))
    x = np.einsum("ihd,jd->ihj", c.q.double().numpy(), k) * 0.01
    x = np.where(j[None, None] <= 16000 - q_len + np.arange(q_len)[:, None, None], x, -np.inf)
    w = np.exp(x - x.max(2, keepdims=True))
    ref = (w @ v) / w.sum(2, keepdims=True)
    err = out.double().cpu().numpy() - ref
    assert np.linalg.norm(err) < 6e-4 * np.linalg.norm(ref)


@pytest.mark.parametrize("q_lens", [[1, 1], [3, 2], [150, 140]])
def test_ranges_of_every_size(mpq, cuda, q_lens):
    """Ranges from 2^-60 to 2^60 among the values, sharp and flat scores, tiny and huge queries, zero ranges."""
    rng = np.random.default_rng(3)
    for spread in (6, 60):
        c = Case(mpq, cuda, q_lens, [200, 333], 4, 2, 64, 8, 16, torch.bfloat16)
        c.s[1] *= np.exp2(rng.uniform(-spread, spread, c.s[1].shape)).astype(np.float32)
        c.check()
    c = Case(mpq, cuda, q_lens, [200, 333], 4, 2, 64, 8, 16, torch.bfloat16)
    c.s[1] = np.where(rng.uniform(size=c.s[1].shape) < 0.5, 0, c.s[1])
    c.s[0] = np.where(rng.uniform(size=c.s[0].shape) < 0.2, 0, c.s[0])
    c.check()
    c.s[1] = np.zeros_like(c.s[1])
    out, _ = c.run()
    assert (out == 0).all()
    for power in (-100, -20, 30, 100):
        c = Case(mpq, cuda, q_lens, [200, 333], 4, 2, 128, 4, 16, torch.bfloat16)
        c.q = (c.q.float() * 2.0 ** power).to(torch.bfloat16)
        c.check(scale=2.0 ** -power * 0.1)
    c = Case(mpq, cuda, q_lens, [200, 333], 4, 2, 64, 8, 16, torch.float16)
    c.check(scale=4.0)
    c.check(scale=0.0)
    c.check(scale=-0.3)


@pytest.mark.parametrize("q_lens", [[2, 3], [160, 200]])
def test_nothing_leaks_from_masked_places(mpq, cuda, q_lens):
    """Infinite, NaN and huge ranges in tokens that a row does not see (later ones, ones before its window, tails of
    pages) change nothing in that row."""
    for bits in (8, 4):
        c = Case(mpq, cuda, q_lens, [300, 257], 4, 2, 64, bits, 16, torch.bfloat16)
        ref, ref_lse = c.run(window=100)
        for b, (nq, nk) in enumerate(zip(c.q_lens, c.kv_lens)):
            for j, bad in ((nk - 1, np.nan), (nk - 2, np.inf), (nk - 1 - nq // 2, 3e38)):
                for i in (0, 1):
                    c.s[i][c.table[b, j // 16], :, j % 16] = bad
        got, got_lse = c.run(window=100)
        for b, (nq, nk) in enumerate(zip(c.q_lens, c.kv_lens)):
            clean = max(0, nq - 1 - nq // 2)                 # rows before the first poisoned token
            lo = int(c.starts[b])
            assert torch.equal(got[lo:lo + clean], ref[lo:lo + clean]) and torch.equal(got_lse[lo:lo + clean], ref_lse[lo:lo + clean])
            if nq > 100:
                assert clean > 50
    for nq in (1, 150):
        c = Case(mpq, cuda, [nq], [300], 4, 2, 64, 8, 16, torch.bfloat16)
        ref, _ = c.run(window=20)
        c.s[:, c.table[0, 0]] = np.nan                       # long before any window
        c.s[:, c.table[0, 1]] = np.inf
        got, _ = c.run(window=20)
        assert torch.equal(got, ref)


def test_strided_queries_and_results(mpq, cuda):
    for q_lens in ([1, 1, 1], [40, 1, 150]):
        c = Case(mpq, cuda, q_lens, [100, 30, 200], 4, 2, 64, 8, 16, torch.bfloat16)
        ref, _ = c.run()
        total = sum(q_lens)
        for at in (0, 1, 8):
            wide = torch.zeros((total, 4 * 64 + 13), dtype=torch.bfloat16, device=cuda)
            view = wide[:, at:at + 256].unflatten(1, (4, 64))
            view.copy_(c.q)
            assert torch.equal(c.run(q=view)[0], ref)
            target = torch.zeros_like(wide)
            got, _ = c.run(out=target[:, at:at + 256].unflatten(1, (4, 64)))
            assert torch.equal(got, ref) and not target[:, :at].any() and not target[:, at + 256:].any()
        swapped = c.q.to(cuda).transpose(0, 1).contiguous().transpose(0, 1)          # [heads][tokens][dim] in memory
        assert torch.equal(c.run(q=swapped)[0], ref)


def test_repeated_runs_are_identical_and_on_another_stream(mpq, cuda):
    for q_lens in ([1] * 4, [30, 1, 200, 5]):
        c = Case(mpq, cuda, q_lens, [1000, 30, 2000, 700], 8, 2, 128, 8, 16, torch.bfloat16)
        ref, ref_lse = c.run()
        for _ in range(3):
            got, lse = c.run()
            assert torch.equal(got, ref) and torch.equal(lse, ref_lse)
        torch.cuda.synchronize()
        st = torch.cuda.Stream()
        with torch.cuda.stream(st):
            got, _ = c.run()
        st.synchronize()
        assert torch.equal(got, ref)


def test_written_tokens_are_attended(mpq, cuda):
    """Write, then attend: the attention over the cache equals the attention over what is read back from it."""
    g = torch.Generator().manual_seed(0)
    n, heads, kv_heads, dim = 90, 4, 2, 64
    k, v = (torch.randn((n, kv_heads, dim), generator=g).to(torch.float16).to(cuda) for _ in range(2))
    q = torch.randn((n, heads, dim), generator=g).to(torch.float16).to(cuda)
    cache = mpq.level_cache(8, kv_heads, 16, dim, 8, cuda)
    table = torch.tensor([[5, 0, 7, 2, 1, 6]], dtype=torch.int32, device=cuda)
    slots = (table[0].long()[torch.arange(n, device=cuda) // 16] * 16 + torch.arange(n, device=cuda) % 16)
    mpq.cache_write(cache, k, v, slots)
    out = mpq.cache_attention(q, cache, torch.tensor([0, n], dtype=torch.int32, device=cuda),
                              torch.tensor([n], dtype=torch.int32, device=cuda), table, n, n)
    kr, vr = (t.double().repeat_interleave(2, 1) for t in mpq.cache_read(cache, slots, torch.float32))
    x = torch.einsum("ihd,jhd->hij", q.double(), kr) / math.sqrt(dim)
    x = x.masked_fill(torch.ones((n, n), dtype=torch.bool, device=cuda).triu(1), -math.inf)
    ref = torch.einsum("hij,jhd->ihd", torch.softmax(x, -1), vr)
    # weights to fp16 (2^-11 of at most the largest value, about 4.5) and the result's rounding
    assert float((out.double() - ref).abs().max()) < 2.0 ** -11 * 4.5 * 2

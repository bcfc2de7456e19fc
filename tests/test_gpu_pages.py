"""Page tables and slot maps made on the device, against lists on the host."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu


class Host:
    """The same state in lists."""

    def __init__(self, sequences, per, pages, page_size):
        self.table, self.lens = [[0] * per for _ in range(sequences)], [0] * sequences
        self.stack, self.per, self.page_size = list(range(pages - 1, -1, -1)), per, page_size

    def extend(self, seqs, new, tokens):
        P, n_seq = self.page_size, len(self.lens)
        named = [0 <= q < n_seq and n >= 0 for q, n in zip(seqs, new)]
        count = lambda n: -(-n // P)                                                           # noqa: E731
        need = [count(self.lens[q] + n) - count(self.lens[q]) if ok else 0 for q, n, ok in zip(seqs, new, named)]
        total = sum(n for n, ok in zip(new, named) if ok)
        missing = max(0, sum(need) - len(self.stack))
        if total > tokens:
            missing = -2
        if any(ok and count(self.lens[q] + n) > self.per for q, n, ok in zip(seqs, new, named)):
            missing = -1
        if missing:
            return [-1] * tokens, [0] * (len(seqs) + 1), [0] * len(seqs), [[0] * self.per for _ in seqs], missing
        slots, starts, lens, rows = [], [0], [], []
        for q, n, ok, more in zip(seqs, new, named, need):
            if not ok:
                starts.append(len(slots))
                lens.append(0)
                rows.append([0] * self.per)
                continue
            have = count(self.lens[q])
            for i in range(more):
                self.table[q][have + i] = self.stack.pop()
            slots += [self.table[q][j // P] * P + j % P for j in range(self.lens[q], self.lens[q] + n)]
            self.lens[q] += n
            starts.append(len(slots))
            lens.append(self.lens[q])
            rows.append(self.table[q][:have + more] + [0] * (self.per - have - more))
        return slots + [-1] * (tokens - len(slots)), starts, lens, rows, 0

    def trim(self, seqs, keep):
        back = []
        for q, k in zip(seqs, keep):
            if 0 <= q < len(self.lens) and 0 <= k < self.lens[q]:
                back += self.table[q][-(-k // self.page_size):-(-self.lens[q] // self.page_size)]
                self.lens[q] = k
        self.stack += back[::-1]


def same(state, host):
    assert state.lens.tolist() == host.lens and state.count.tolist() == [len(host.stack), 0]
    assert state.free[:len(host.stack)].tolist() == host.stack
    for row, mine, n in zip(state.table.tolist(), host.table, host.lens):
        used = -(-n // host.page_size)
        assert row[:used] == mine[:used]


def ints(v, cuda):
    return torch.tensor(v, dtype=torch.int32, device=cuda)


@pytest.mark.parametrize("sequences,per,pages,page_size,most", [(1, 1, 1, 1, 1), (5, 7, 20, 4, 9), (64, 40, 900, 16, 300), (700, 13, 4000, 24, 60),
                                                                (2000, 130, 100000, 1, 90), (40, 3, 120, 1000, 2500)])
def test_random_steps(mpq, cuda, sequences, per, pages, page_size, most):
    rng = random.Random(sequences * 7 + per)
    state, host = mpq.page_state(sequences, per, pages, page_size, cuda), Host(sequences, per, pages, page_size)
    kinds = set()
    for step in range(25):
        batch = rng.randint(0, sequences) if step % 3 else sequences
        seqs = rng.sample(range(sequences), batch)
        for i in range(batch):
            if rng.random() < 0.1:
                seqs[i] = rng.choice([-1, sequences, -7, 2 ** 31 - 1])
        new = [rng.choice([0, 1, 1, rng.randint(0, most), -1 if rng.random() < 0.05 else 2]) for _ in seqs]
        total = sum(max(0, n) for n in new)
        tokens = max(0, total + rng.choice([0, 0, 5, 77, -1 if step % 5 == 0 else 0]))
        plan = mpq.pages_extend(state, ints(seqs, cuda), ints(new, cuda), tokens)
        want = host.extend(seqs, new, tokens)
        kinds.add(min(0, want[4]) if want[4] <= 0 else 1)
        for got, w, name in zip(plan, want, plan._fields):
            assert got.tolist() == ([w] if name == "missing" else w), (step, name)
        same(state, host)
        some = rng.sample(range(sequences), rng.randint(0, sequences))
        keep = [rng.choice([0, -1, host.lens[q], rng.randint(0, host.lens[q] + 3), max(0, host.lens[q] - 1)]) for q in some]
        mpq.pages_trim(state, ints(some, cuda), ints(keep, cuda))
        host.trim(some, keep)
        same(state, host)
    assert 0 in kinds


def test_all_sequences_in_their_order(mpq, cuda):
    state, host = mpq.page_state(6, 5, 30, 4, cuda), Host(6, 5, 30, 4)
    for new in ([3, 0, 9, 4, 5, 1], [1, 1, 1, 1, 1, 1], [4, 16, 0, 0, 2, 3]):
        plan = mpq.pages_extend(state, None, ints(new, cuda), sum(new))
        want = host.extend(range(6), new, sum(new))
        assert [t.tolist() for t in plan] == [*want[:4], [want[4]]]
    mpq.pages_trim(state, None, ints([0, 3, 2], cuda))
    host.trim(range(3), [0, 3, 2])
    same(state, host)


@pytest.mark.parametrize("batch", [1, 511, 512, 513, 1024, 1500, 8192])
def test_batches_past_the_threads_of_a_block(mpq, cuda, batch):
    state, host = mpq.page_state(batch, 3, 2 * batch + 5, 4, cuda), Host(batch, 3, 2 * batch + 5, 4)
    new = [(7 * i) % 5 for i in range(batch)]
    plan = mpq.pages_extend(state, None, ints(new, cuda), sum(new) + 1)
    want = host.extend(range(batch), new, sum(new) + 1)
    assert [t.tolist() for t in plan] == [*want[:4], [want[4]]]
    same(state, host)


def test_a_shortage_changes_nothing(mpq, cuda):
    """Pages, the row of a sequence, or the slots do not suffice: the state is what it was, and what the batch's calls see is empty."""
    for new, tokens, says in (([9, 9, 9], 40, 2), ([1, 17, 1], 40, -1), ([4, 4, 4], 11, -2), ([2 ** 31 - 1] * 3, 40, -1)):
        state = mpq.page_state(3, 4, 7, 4, cuda)
        before = [t.clone() for t in state[:4]]
        plan = mpq.pages_extend(state, None, ints(new, cuda), tokens)
        assert plan.missing.item() == says
        assert (plan.slots == -1).all() and not plan.q_starts.any() and not plan.kv_lens.any() and not plan.table.any()
        assert all(torch.equal(a, b) for a, b in zip(state[:4], before))


def test_a_trim_undoes_an_extend(mpq, cuda):
    g = torch.Generator().manual_seed(3)
    state = mpq.page_state(50, 64, 2000, 8, cuda)
    mpq.pages_extend(state, None, torch.randint(0, 300, (50,), generator=g, dtype=torch.int32).to(cuda), 20000)
    lens, free, count = state.lens.clone(), state.free.clone(), state.count.clone()
    seqs = torch.randperm(50, generator=g).to(torch.int32)[:33].to(cuda)
    plan = mpq.pages_extend(state, seqs, torch.randint(0, 100, (33,), generator=g, dtype=torch.int32).to(cuda), 5000)
    assert plan.missing.item() == 0 and not torch.equal(state.lens, lens)
    mpq.pages_trim(state, seqs, lens[seqs.long()])
    assert torch.equal(state.lens, lens) and torch.equal(state.free, free) and torch.equal(state.count, count)


def test_slots_past_32_bits(mpq, cuda):
    state = mpq.page_state(1, 2, 2, 2 ** 30 - 1, cuda)
    state.free.copy_(ints([2 ** 31 - 1, 2 ** 31 - 2], cuda))
    plan = mpq.pages_extend(state, None, ints([5], cuda), 5)
    at = (2 ** 31 - 2) * (2 ** 30 - 1)
    assert plan.slots.tolist() == [at, at + 1, at + 2, at + 3, at + 4]


def test_a_captured_step_goes_on_where_the_last_one_ended(mpq, cuda):
    state, host = mpq.page_state(4, 8, 32, 4, cuda), Host(4, 8, 32, 4)
    seqs, new = ints([2, 0, -1], cuda), ints([1, 1, 1], cuda)
    mpq.pages_extend(state, None, ints([3, 5, 4, 0], cuda), 16)
    host.extend(range(4), [3, 5, 4, 0], 16)
    side = torch.cuda.Stream()
    out = mpq.pages_extend(state, seqs, new, 4)
    host.extend([2, 0, -1], [1, 1, 1], 4)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        mpq.pages_extend(state, seqs, new, 4, out=out)
    for _ in range(9):
        graph.replay()
        want = host.extend([2, 0, -1], [1, 1, 1], 4)
        assert [t.tolist() for t in out] == [*want[:4], [want[4]]]
    same(state, host)


def test_tensors_that_do_not_fit(mpq, cuda):
    state = mpq.page_state(4, 8, 32, 4, cuda)
    one = ints([1, 1], cuda)
    for call in (lambda: mpq.pages_extend(state, one[:1], one, 4), lambda: mpq.pages_extend(state, one.long(), one, 4),
                 lambda: mpq.pages_extend(state, one, one.cpu(), 4), lambda: mpq.pages_extend(state._replace(lens=state.lens[:3]), one, one, 4),
                 lambda: mpq.pages_extend(state, one, ints([1, 1, 1, 1], cuda)[::2], 4),
                 lambda: mpq.pages_extend(state, one, one, 4, out=mpq.pages_extend(state, one, one, 5)),
                 lambda: mpq.pages_trim(state, one, one.float()), lambda: mpq.pages_trim(state._replace(count=state.count[:1]), one, one)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(mpq.MpqError):
        mpq.pages_extend(state._replace(page_size=0), one, one, 4)

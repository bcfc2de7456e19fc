"""NaNs and infinities that a row of the attention does see: they come out, in the result and in its logarithm, whatever
the form of the launch; a row that sees nothing keeps its zeros."""
import numpy as np
import pytest
import torch

from tests.test_gpu_level_cache import Case

pytestmark = pytest.mark.gpu

# tiles of 8, 16 and 256 rows; one split, splits that one cluster joins, splits that a second launch joins
FORMS = [(q_lens, kv_lens, hint) for q_lens in ([1, 1], [5, 3], [60, 33])
         for kv_lens, hint in (([190, 333], 1), ([900, 700], 900), ([5000, 3000], 5000))]


def states(got, lse):
    """Per (token, head): 1 all NaN, 0 all finite, -1 zeros and minus infinity; anything else is an error."""
    got, lse = got.float().cpu().numpy(), lse.cpu().numpy()
    nan, fine = np.isnan(got).all(2) & np.isnan(lse), np.isfinite(got).all(2) & np.isfinite(lse)
    dead = (got == 0).all(2) & np.isneginf(lse)
    assert (nan | fine | dead).all()
    return np.where(nan, 1, np.where(fine, 0, -1))


@pytest.mark.parametrize("q_lens,kv_lens,hint", FORMS)
@pytest.mark.parametrize("dim,bits", [(64, 8), (128, 4)])
def test_queries_that_are_not_finite(mpq, cuda, q_lens, kv_lens, hint, dim, bits):
    c = Case(mpq, cuda, q_lens, kv_lens, 4, 1, dim, bits, 16, torch.bfloat16)
    ref, ref_lse = c.run(max_kv=hint)
    bad = np.zeros((sum(q_lens), 4), dtype=bool)
    for i, (token, head, value) in enumerate([(0, 1, np.nan), (sum(q_lens) - 1, 3, np.inf), (sum(q_lens) - 1, 0, -np.inf)]):
        c.q[token, head, 5 * i + 1] = value
        bad[token, head] = True
    c.q[0, 2] = float("nan")
    bad[0, 2] = True
    got, lse = c.run(max_kv=hint)
    assert np.array_equal(states(got, lse) == 1, bad)
    keep = torch.from_numpy(~bad).to(cuda)
    assert torch.equal(got[keep], ref[keep]) and torch.equal(lse[keep], ref_lse[keep])
    # nothing of either sequence is there: zeros, also for the queries that are not finite
    c.table[:] = -1
    assert (states(*c.run(max_kv=hint)) == -1).all()


@pytest.mark.parametrize("q_lens,kv_lens,hint", FORMS)
@pytest.mark.parametrize("value", [np.nan, np.inf])
@pytest.mark.parametrize("window", [1, 7])
def test_ranges_that_are_not_finite(mpq, cuda, q_lens, kv_lens, hint, value, window):
    """Every third of the last tokens has such a key range: the rows whose window holds one, and no others, are NaN
    (with a window of 1 a row sees nothing else)."""
    c = Case(mpq, cuda, q_lens, kv_lens, 4, 1, 64, 8, 16, torch.float16)
    ref, ref_lse = c.run(window=window, max_kv=hint)
    bad = np.zeros(sum(q_lens), dtype=bool)
    for b, (nq, nk) in enumerate(zip(q_lens, kv_lens)):
        places = np.arange(nk - 1, nk - nq - 1, -3)
        for j in places:
            c.s[0][c.table[b, j // 16], :, j % 16] = value
        pos = nk - nq + np.arange(nq)
        bad[c.starts[b]:c.starts[b + 1]] = ((places[None] <= pos[:, None]) & (places[None] > pos[:, None] - window)).any(1)
    got, lse = c.run(window=window, max_kv=hint)
    assert bad.any() and np.array_equal(states(got, lse) == 1, np.broadcast_to(bad[:, None], (len(bad), 4)))
    keep = torch.from_numpy(~bad).to(cuda)
    assert torch.equal(got[keep], ref[keep]) and torch.equal(lse[keep], ref_lse[keep])


@pytest.mark.parametrize("q_lens,kv_lens,hint", FORMS)
@pytest.mark.parametrize("which", [0, 1])
def test_stretches_of_ranges_that_are_not_finite(mpq, cuda, q_lens, kv_lens, hint, which):
    """NaN ranges of all keys (or values) of a stretch that whole warps, and whole splits, have to themselves."""
    for first, last in ((0, 100), (0, 5000), (32, 64), (1024, 3000)):
        c = Case(mpq, cuda, q_lens, kv_lens, 4, 1, 64, 8, 16, torch.bfloat16)
        for b, nk in enumerate(kv_lens):
            j = np.arange(first, min(last, nk - q_lens[b] + 1))
            c.s[which][c.table[b, j // 16], :, j % 16] = np.nan
        state = states(*c.run(max_kv=hint))
        for b, nk in enumerate(kv_lens):
            assert (state[c.starts[b]:c.starts[b + 1]] == (1 if first <= nk - q_lens[b] else 0)).all()

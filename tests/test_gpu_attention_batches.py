"""The attention's batches: tokens that belong to no sequence, and more than 32 sequences."""
import numpy as np
import pytest
import torch

from tests.test_gpu_level_cache import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("pad", [1, 3, 70])
@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [190, 333]), ([1] * 32, [40] * 32), ([5, 3], [190, 333]), ([64], [64]), ([60, 33], [190, 333]),
                                            ([0, 0], [40, 0]), ([1, 1], [5000, 3000]), ([60, 33], [5000, 3000])])
@pytest.mark.parametrize("heads,kv_heads", [(4, 1), (6, 2)])
def test_tokens_of_no_sequence_see_nothing(mpq, cuda, q_lens, kv_lens, heads, kv_heads, pad):
    """The padding of a step whose size is fixed: zeros and minus infinity, and nothing else changes."""
    c = Case(mpq, cuda, q_lens, kv_lens, heads, kv_heads, 64, 8, 16, torch.float16)
    total = sum(q_lens)
    q = torch.full((total + pad, heads, 64), float("nan"), dtype=torch.float16, device=cuda)
    q[:total] = c.q
    for max_kv in (1, max(kv_lens)):
        for max_q in (1, max(1, *q_lens), total + pad):
            out = torch.full_like(q, 5.0)
            got, lse = c.run(q=q, out=out, max_q=max_q, max_kv=max_kv)
            assert (got[total:] == 0).all() and torch.isneginf(lse[total:]).all()
            if total:
                ref, ref_lse = c.run(max_q=max_q, max_kv=max_kv)
                assert torch.isfinite(got[:total]).all()
                assert np.allclose(got[:total].float().cpu(), ref.float().cpu(), atol=2.0 ** -10) and np.allclose(lse[:total].cpu(), ref_lse.cpu(), atol=1e-4)


@pytest.mark.parametrize("batch", [33, 64, 70])
@pytest.mark.parametrize("form", ["rows", "tiles"])
@pytest.mark.parametrize("splits", ["one", "cluster", "launch"])
def test_more_sequences_than_a_warp_looks_at_in_one_trip(mpq, cuda, batch, form, splits):
    """The search for a tile's and a token's sequence walks the batch 32 at a time: idle sequences around the 32nd and at
    the end, long contexts on either side of it, single tokens and chunks."""
    rng = np.random.default_rng(batch)
    kv_lens = [int(v) for v in rng.integers(1, 300, batch)]
    for i in (3, 31, 32, batch - 2):
        kv_lens[i] = 4000 + i
    q_lens = [1] * batch if form == "rows" else [int(min(n, v)) for n, v in zip(kv_lens, rng.integers(1, 3 if splits == "launch" else 40, batch))]
    for i in (30, 32, batch - 1):
        q_lens[i] = 0
    if form == "tiles":
        q_lens[31] = 12
    hint = {"one": 1, "cluster": 1200 if form == "rows" else 900, "launch": 100000}[splits]
    need = mpq.cache_attention_workspace(sum(q_lens), batch, 4, 1, 64, max(q_lens), hint)
    assert (need > 0) == (splits == "launch")
    c = Case(mpq, cuda, q_lens, kv_lens, 4, 1, 64, 8, 16, torch.bfloat16)
    c.check(max_kv=hint)
    c.check(max_kv=hint, window=500)

"""Drawing tokens from numbers at the ends of their ranges, and from ones that are none."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_numbers_that_are_none(mpq, cuda):
    """A NaN among a row's own numbers, at any temperature; +infinity is drawn at none over 0."""
    vocab = 5000
    x = torch.randn((5, vocab), device=cuda)
    x[4, 77] = math.inf
    best = x.argmax(1)
    for warm in (0.0, -1.0):
        for spoilt in ("uniform", "top_p", "min_p"):
            args = dict(uniform=torch.full((5,), 0.5, device=cuda), top_p=torch.full((5,), 0.9, device=cuda), min_p=torch.full((5,), 0.1, device=cuda))
            args[spoilt][1] = math.nan
            args[spoilt][4] = math.nan
            logprob = torch.zeros(5, device=cuda)
            got = mpq.sample(x, temperature=torch.full((5,), warm, device=cuda), logprob=logprob, **args)
            assert got[[1, 4]].tolist() == [-1, -1] and torch.isnan(logprob[[1, 4]]).all()
            assert torch.equal(got[[0, 2, 3]], best[[0, 2, 3]]) and torch.isfinite(logprob[[0, 2, 3]]).all()
        logprob = torch.zeros(5, device=cuda)
        got = mpq.sample(x, torch.full((5,), 0.5, device=cuda), torch.full((5,), warm, device=cuda), logprob=logprob)
        assert torch.equal(got, best) and torch.isnan(logprob[4]) and torch.isfinite(logprob[:4]).all()

"""Drawing tokens from numbers at the ends of their ranges, and from ones that are none."""
import math

import pytest
import torch

from tests.test_gpu_sample_ends import TYPES, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [900, 9001])
def test_temperatures_and_spans_at_the_ends_of_their_range(mpq, cuda, vocab, dtype):
    """Logits that lie farther apart than the largest number, at temperatures to match, and the smallest numbers at the smallest ones."""
    g = torch.Generator().manual_seed(vocab)
    top, rows = torch.finfo(TYPES[dtype]).max, 4
    x = (2 * torch.rand((rows, vocab), generator=g) - 1) * top
    x[:, 5], x[:, 7] = top, -top
    u = torch.tensor([0.1, 0.4, 0.7, 0.95])
    rules = [dict(), dict(k=[vocab // 2] * 4), dict(p=[0.9, 0.5, 0.999, 0.1]), dict(least=[0.05, 0.3, 0.9, 0.2]), dict(k=[40] * 4, p=[0.7] * 4, least=[0.1] * 4),
             dict(k=[vocab - 100] * 4, p=[0.9] * 4)]
    for warm in (3.4e38, 1e38, 2e37):
        for c in rules:
            check(mpq, cuda, x, u, [warm] * 4, dtype=dtype, **c)
    y = x.to(TYPES[dtype]).to(cuda)
    forever = torch.full((rows,), math.inf, device=cuda)      # every token alike
    assert mpq.sample(y, u.to(cuda), forever).tolist() == [int(float(v) * vocab) for v in u]
    assert mpq.sample(y, u.to(cuda), forever, min_p=torch.full((rows,), 0.5, device=cuda)).tolist() == [int(float(v) * vocab) for v in u]
    tiny = torch.randint(-2000, 1, (rows, vocab), generator=g).float() * (2.0 ** -149 if dtype == "f32" else 2.0 ** -133)
    assert tiny.unique().numel() > 500
    for warm in (2.0 ** -140, 2.0 ** -130, 2.0 ** -125) if dtype == "f32" else (2.0 ** -128, 2.0 ** -125, 2.0 ** -122):
        for c in rules:
            check(mpq, cuda, tiny, u, [warm] * 4, dtype=dtype, **c)


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

"""Tensors that the binding of the decoder block's operators refuses, and workspaces of other types that it takes."""
import pytest
import torch

from tests.test_gpu_level_cache import Case

pytestmark = pytest.mark.gpu


def test_workspaces(mpq, cuda):
    c = Case(mpq, cuda, [1, 1], [5000, 3000], 4, 1, 64, 8, 16, torch.bfloat16)
    ref, ref_lse = c.run()
    need = mpq.cache_attention_workspace(2, 2, 4, 1, 64, 1, 5000)
    assert need > 0
    for t in (torch.empty(need, dtype=torch.uint8, device=cuda), torch.empty((need + 3) // 4, device=cuda),
              torch.empty((need // 16 + 1, 2), dtype=torch.int64, device=cuda)):
        got, lse = c.run(workspace=t)
        assert torch.equal(got, ref) and torch.equal(lse, ref_lse)
    with pytest.raises(mpq.MpqError):
        c.run(workspace=torch.empty(need // 4 - 4, device=cuda))
    for t in (torch.empty(need, dtype=torch.uint8), torch.empty((need, 2), dtype=torch.uint8, device=cuda)[:, 0]):
        with pytest.raises(ValueError, match="workspace"):
            c.run(workspace=t)

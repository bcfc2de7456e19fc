"""What the binding of the decoder block's operators looks at before it hands pointers on; no GPU is needed."""
import pytest
import torch


def test_a_workspace_is_looked_at(mpq):
    with pytest.raises(ValueError, match="workspace on a CUDA device"):
        mpq._workspace(torch.empty(1024, dtype=torch.uint8))
    with pytest.raises(ValueError, match="workspace on a CUDA device"):
        mpq._workspace(torch.empty(1024, dtype=torch.uint8)[::2])

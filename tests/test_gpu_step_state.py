"""What a step's calls remember and refuse."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda:0")


def test_adapters_in_another_order_are_refused(mpq, cuda):
    """As many elements, another layout."""
    a, w = mpq.encode_levels(torch.randn((5, 64), device=cuda)), mpq.encode_levels(torch.randn((48, 64), device=cuda))
    down, up = torch.randn((2, 16, 64), device=cuda).half(), torch.randn((2, 48, 16), device=cuda).half()
    low, starts, ids = mpq.adapters(down, up), ints(0, 5), ints(1)
    mpq.linear_adapted(a, w, low, starts, ids)
    for bad in (dict(up=up.transpose(1, 2).contiguous()), dict(up=up.reshape(4, 24, 16)), dict(up=up.reshape(-1)), dict(up=up.reshape(1, 96, 16)),
                dict(down=down.reshape(4, 8, 64)), dict(down=down.transpose(1, 2).contiguous()), dict(down=down.reshape(1, 32, 64)), dict(down=down.reshape(32, 64))):
        with pytest.raises(ValueError):
            mpq.linear_adapted(a, w, low._replace(**bad), starts, ids)

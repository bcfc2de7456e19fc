"""What a step's calls remember and refuse."""
import pytest
import torch

from paper_1905_13389_b200 import decoder

pytestmark = pytest.mark.gpu


def ints(*v):
    return torch.tensor(v, dtype=torch.int32, device="cuda:0")


def test_a_shortage_is_remembered_until_it_is_looked_for(mpq, cuda):
    """A step that lacks pages between steps that do not, in eager calls and in a graph that is replayed."""
    pages = decoder.DevicePages(4, 16, 3, 4, cuda)
    first, one = ints(0), ints(16)
    pages.extend(first, ints(0), 16, 16, 64)                  # (warms up)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pages.extend(first, one, 16, 16, 64)
    pages.check()
    for lost in (False, True):
        for _ in range(4):
            graph.replay()
        if lost:
            graph.replay()                                    # a fifth page
        pages.trim(ints(0), ints(32))
        graph.replay()                                        # ... and again one that fits
        if lost:
            with pytest.raises(MemoryError, match="earlier"):
                pages.check()
        pages.check()
        pages.trim(ints(0), ints(0))
    for _ in range(2):                                        # the same without a graph
        pages.extend(ints(0, 1), ints(40, 40), 80, 40, 64)
        pages.extend(ints(2), ints(3), 3, 3, 64)
        with pytest.raises(MemoryError, match="earlier"):
            pages.check()
        pages.check()
    pages.extend(ints(0, 1), ints(40, 40), 80, 40, 64)        # the last batch itself says what it lacked
    with pytest.raises(MemoryError, match="pages are missing"):
        pages.check()
    pages.check()


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

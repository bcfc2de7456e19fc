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


class Elsewhere(torch.Tensor):
    """A tensor that says it is on another device."""

    def get_device(self):
        return 1


def every_call(mpq, cuda):
    """name -> (call, its tensors)"""
    x, w = torch.randn((6, 64), device=cuda), mpq.encode_levels(torch.randn((8, 64), device=cuda))
    a = mpq.encode_levels(x)
    cache = mpq.level_cache(4, 2, 16, 64, 8, cuda)
    k, slots = torch.randn((6, 2, 64), dtype=torch.float16, device=cuda), torch.arange(6, device=cuda)
    ints = lambda *v: torch.tensor(v, dtype=torch.int32, device=cuda)                          # noqa: E731
    held = lambda lv, *t: mpq.Levels(*t, lv.bits, lv.k)                                        # noqa: E731
    paged = lambda *t: mpq.LevelCache(*t, 8)                                                   # noqa: E731
    return {
        "norm": (lambda x, g, r, ro, v: mpq.rmsnorm_levels(x, g, 1e-6, residual=r, residual_out=ro, values=v),
                 [x, torch.ones(64, device=cuda), x.clone(), torch.empty_like(x), torch.empty_like(x)]),
        "encode": (lambda x, v: mpq.encode_levels(x, values=v), [x, torch.empty_like(x)]),
        "encode into": (lambda x, b, s, u: mpq.encode_levels(x, out=held(a, b, s, u)), [x, *a[:3]]),
        "linear": (lambda ab, as_, au, wb, ws, wu, b, r, o: mpq.linear_levels(held(a, ab, as_, au), held(w, wb, ws, wu), bias=b, residual=r, out=o),
                   [*a[:3], *w[:3], torch.zeros(8, device=cuda), torch.zeros((6, 8), device=cuda), torch.zeros((6, 8), device=cuda)]),
        "write": (lambda ck, cs, cv, ct, k, v, s: mpq.cache_write(paged(ck, cs, cv, ct), k, v, s), [*cache[:4], k, k, slots]),
        "read": (lambda ck, cs, cv, ct, s, k, v: mpq.cache_read(paged(ck, cs, cv, ct), s, torch.float16, k, v),
                 [*cache[:4], slots, torch.empty_like(k), torch.empty_like(k)]),
        "attention": (lambda ck, cs, cv, ct, q, st, n, t, o, lse: mpq.cache_attention(q, paged(ck, cs, cv, ct), st, n, t, 6, 6, out=o, lse=lse),
                      [*cache[:4], k, ints(0, 6), ints(6), ints(1)[None], torch.empty_like(k), torch.empty((6, 2), device=cuda)]),
    }


def test_tensors_of_another_device_are_refused(mpq, cuda, monkeypatch):
    calls = every_call(mpq, cuda)
    for name, (call, tensors) in calls.items():
        call(*tensors)
        for i in range(len(tensors)):
            moved = list(tensors)
            moved[i] = moved[i].as_subclass(Elsewhere)
            with pytest.raises(ValueError):
                call(*moved)
                pytest.fail("%s took tensor %d from another device" % (name, i))
    monkeypatch.setattr(mpq, "_current_device", lambda: 1)
    for call, tensors in calls.values():
        with pytest.raises(ValueError, match="current device"):
            call(*tensors)

"""Bounded waits of the product with adapters that run out (see test_gpu_waits): results are right or NaN, the count says so, and
the device is fit for the next call.  In a process of its own, since the count is one of the process."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CHILD = """
import sys
import torch
from paper_1905_13389_b200 import binding as mpq
from tests.test_gpu_adapted import Case

cuda = torch.device("cuda:0")
if sys.argv[1] == "few":
    cases = [Case(mpq, cuda, [1] * 40 + [24], [i % 5 - 1 for i in range(41)], 30000, 300, 16), Case(mpq, cuda, [5], [2], 256, 33000, 64, "bf16"),
             Case(mpq, cuda, [30, 10], [0, 1], 19000, 9000, 32)]
else:                                                         # tiles of one adapter, and tiles of several
    cases = [Case(mpq, cuda, [513], [1], 2177, 272, 64), Case(mpq, cuda, [1300, 1, 1299], [1, -1, 0], 4000, 1500, 128, "bf16"),
             Case(mpq, cuda, [100] * 3, [0, 1, 2], 9001, 3300, 16)]
calls = [lambda c=c, a=a: c.run(act=a, dtype=torch.bfloat16).flatten() for c, a in zip(cases, ("none", "relu", "silu"))]
ref = [c() for c in calls]
assert mpq.wait_failures() == 0
seen = 0
for polls in (0, 0, 0, 1, 2, 5):
    mpq.wait_limit(polls)
    for c, r in zip(calls, ref):
        before = mpq.wait_failures()
        got = c()
        after = mpq.wait_failures()
        wrong = got != r
        assert torch.isnan(got[wrong]).all(), "a result that is neither right nor NaN"
        assert after >= before and (after > before or not wrong.any())
        seen += int(after > before and bool(wrong.any()))
    mpq.wait_limit()
    before = mpq.wait_failures()
    for c, r in zip(calls, ref):
        assert torch.equal(c(), r)
    assert mpq.wait_failures() == before
assert seen >= len(calls), seen
print("waits ran out in %d calls, %d CTAs" % (seen, mpq.wait_failures()))
"""


@pytest.mark.parametrize("what", ["few", "pairs"])
def test_a_wait_that_runs_out_leaves_nan_and_a_healthy_device(mpq, cuda, what):
    r = subprocess.run([sys.executable, "-c", CHILD, what], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "waits ran out" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def test_no_wait_runs_out_in_ordinary_calls(mpq, cuda):
    import torch

    from tests.test_gpu_adapted import Case
    before = mpq.wait_failures()
    for lens, n, k in (([5], 256, 4096), ([64], 30000, 300), ([2600], 4000, 1500), ([700, 600], 4000, 1500)):
        Case(mpq, cuda, lens, [1, 2][:len(lens)], n, k, 32).run(dtype=torch.float16)
    assert mpq.wait_failures() == before

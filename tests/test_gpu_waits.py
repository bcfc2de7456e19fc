"""What happens when a bounded wait of a tensor-core kernel runs out.  A limit of no or a few polls makes healthy waits run
out: the kernels have to return, count it, store NaN for what they have not computed and nothing wrong, and leave the device
fit for the next call.  In a process of its own, since the count is one of the process."""
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
from tests.test_gpu_level_cache import Case
from tests.test_gpu_linear_levels import operand

cuda = torch.device("cuda:0")
what = sys.argv[1]
if what == "attention":
    # one split, splits that one cluster joins, splits that a second launch joins; one and two tiles of rows in a CTA
    def call(q_lens, kv_lens, heads, hint, dim, bits):
        c = Case(mpq, cuda, q_lens, kv_lens, heads, 2, dim, bits, 16, torch.bfloat16)
        return lambda: torch.cat([t.flatten().float() for t in c.run(max_kv=hint)])
    calls = [call(*a) for a in (([40, 200], [700, 300], 4, 1, 64, 8), ([40], [4000], 8, 4000, 128, 4), ([300], [9000], 4, 9000, 128, 8), ([70, 5], [0, 2], 4, 1, 64, 4))]
else:
    # few rows with the whole of k and with parts of it, and CTA pairs with one tile each and with several
    sizes = [(64, 30000, 300), (5, 256, 33000), (40, 19000, 9000)] if what == "few" else [(513, 2177, 272), (2600, 4000, 1500), (300, 9001, 33000)]
    def call(m, n, k, act):
        a, w = operand(mpq, cuda, m, k, 8, 1)[0], operand(mpq, cuda, n, k, 8, 2)[0]
        return lambda: mpq.linear_levels(a, w, act=act, dtype=torch.bfloat16).flatten()
    calls = [call(*s, act) for s, act in zip(sizes, ("none", "relu", "silu"))]

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


@pytest.mark.parametrize("what", ["few", "pairs", "attention"])
def test_a_wait_that_runs_out_leaves_nan_and_a_healthy_device(mpq, cuda, what):
    r = subprocess.run([sys.executable, "-c", CHILD, what], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "waits ran out" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


DECODER = """
import torch
from paper_1905_13389_b200 import binding as mpq, decoder

cuda = torch.device("cuda:0")
config = decoder.Config(layers=1, width=256, heads=8, kv_heads=2, dim=64, inner=768)
model, pages = decoder.EncodedDecoder(config, decoder.random_weights(config, cuda), pages=32, page_size=16), decoder.Pages(32, 16)
x = torch.randn((70, config.width), device=cuda).to(torch.bfloat16)
model.forward(x, pages.extend({0: 70}, cuda))
model.check()
mpq.wait_limit(0)
model.forward(x, pages.extend({1: 70}, cuda))
mpq.wait_limit()
try:
    model.check()
except RuntimeError as e:
    print("noticed:", e)
model.forward(x, pages.extend({2: 70}, cuda))
model.check()
"""


def test_the_decoder_notices_a_wait_that_ran_out(mpq, cuda):
    r = subprocess.run([sys.executable, "-c", DECODER], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "noticed:" in r.stdout, r.stdout[-2000:] + r.stderr[-4000:]


def test_no_wait_runs_out_in_ordinary_calls(mpq, cuda):
    """One call of each tensor-core form, in this process and with the ordinary limit."""
    import torch

    from tests.test_gpu_level_cache import Case
    from tests.test_gpu_linear_levels import operand
    before = mpq.wait_failures()
    for m, n, k in ((5, 256, 4096), (64, 30000, 300), (2600, 4000, 1500)):
        mpq.linear_levels(operand(mpq, cuda, m, k, 8, 1)[0], operand(mpq, cuda, n, k, 8, 2)[0])
    Case(mpq, cuda, [300], [3000], 4, 2, 128, 8, 16, torch.bfloat16).run()
    assert mpq.wait_failures() == before

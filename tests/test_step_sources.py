"""What the sources of the operators around a server's step have to keep to, and no result shows."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1905_13389_b200", "csrc")


@pytest.mark.parametrize("name", ["mpq_pages.cu", "mpq_linear_levels.cu", "mpq_adapters.cu", "mpq_adapters.cuh", "mpq_sample.cu"])
def test_nothing_is_read_as_constant_that_the_kernel_before_may_still_write(name):
    """These kernels start while the one before them still runs.  A read-only load may be moved over the wait for it; `up` alone, which is
    there before the product begins, is read that way."""
    with open(os.path.join(CSRC, name)) as f:
        code = re.sub(r"//.*", "", f.read())
    assert "griddepcontrol.wait" in code or "chain_entry()" in code or "chain_wait()" in code
    assert not re.search(r"ld\.global\.nc|__restrict__", code)
    for line in code.splitlines():
        assert "__ldg" not in line or re.search(r"\(g\.up\)|\(up \+", line), line

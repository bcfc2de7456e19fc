"""What the binding of the decoder block's operators looks at before it hands pointers on; no GPU is needed."""
import os
import subprocess
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_a_workspace_is_looked_at(mpq):
    with pytest.raises(ValueError, match="workspace on a CUDA device"):
        mpq._workspace(torch.empty(1024, dtype=torch.uint8))
    with pytest.raises(ValueError, match="workspace on a CUDA device"):
        mpq._workspace(torch.empty(1024, dtype=torch.uint8)[::2])


def test_the_binding_imports_where_torch_has_no_cuda():
    """As on a torch built without CUDA: sizes and refusals need no device."""
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    delattr(torch._C, name)\n"
            "from paper_1905_13389_b200 import binding as mpq\n"
            "assert mpq.level_row_bytes(17) == 32 and mpq.row_words(100) == 4\n"
            "try:\n"
            "    mpq.encode_levels(torch.zeros((4, 64)))\n"
            "except ValueError:\n"
            "    print('refused')\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0 and "refused" in r.stdout, r.stderr

"""The paged cache's operators on the checked build (-DH2O_BOUNDS), the stand-in for a memory checker."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_14048_b200", "csrc")


@pytest.mark.gpu
def test_pages_cases_pass_on_the_checked_build():
    import torch

    assert torch.cuda.is_available(), "needs a CUDA device; there is no CPU fallback"
    lib = os.path.join(ROOT, "paper_2306_14048_b200", "libh2o_b200_bounds.so")
    assert os.path.exists(lib)
    res = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "pages_bounds_cases.py")], env=dict(os.environ, H2O_B200_LIB=lib),
                         capture_output=True, text=True, timeout=900)
    assert res.returncode == 0 and "PAGES_BOUNDS_CASES_PASSED" in res.stdout, res.stdout[-3000:] + res.stderr[-3000:]


@pytest.mark.parametrize("name,checks", [("rotate.cu", ["H2O_IN_RANGE("]), ("pages_attend_tc.cu", ["token_ok(", "partial_ok(", "page_in("]),
                                         ("store_attend_mma.cu", ["page_in("]), ("store_attend_fma.cu", ["page_in("])])
def test_every_kernel_checks_its_indices(name, checks):
    text = open(os.path.join(CSRC, name)).read()
    for check in checks:
        assert check in text, check

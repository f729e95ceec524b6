"""The K/V store operators on the checked build (-DH2O_BOUNDS), the stand-in for a memory checker."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_14048_b200", "csrc")


@pytest.mark.gpu
def test_store_cases_pass_on_the_checked_build():
    import torch

    assert torch.cuda.is_available(), "needs a CUDA device; there is no CPU fallback"
    lib = os.path.join(ROOT, "paper_2306_14048_b200", "libh2o_b200_bounds.so")
    assert os.path.exists(lib)
    res = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "store_bounds_cases.py")], env=dict(os.environ, H2O_B200_LIB=lib),
                         capture_output=True, text=True, timeout=900)
    assert res.returncode == 0 and "STORE_BOUNDS_CASES_PASSED" in res.stdout, res.stdout[-3000:] + res.stderr[-3000:]


@pytest.mark.parametrize("name", ["store.cu", "store_join.cu", "store_attend_fma.cu", "store_attend_mma.cu", "store_attend_tc.cu"])
def test_every_store_kernel_checks_its_indices(name):
    """Rows, tokens and partial results pass through the checks of store.cuh (or H2O_IN_RANGE itself)."""
    text = open(os.path.join(CSRC, name)).read()
    wanted = {"store.cu": ["H2O_IN_RANGE("], "store_join.cu": ["token_ok(", "partial_ok("]}
    for check in wanted.get(name, ["row_ok(", "token_ok(", "partial_ok("]):
        assert check in text, check

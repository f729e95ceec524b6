"""Tests of the paged cache run against the checked build of the library (every token, partial result and page verified before
use: a check that fires leaves H2O_ERR_STATE in the status word, which these tests find to be 0).

Executed as a script by tests/test_gpu_pages_bounds.py in a process of its own, with H2O_B200_LIB naming
libh2o_b200_bounds.so: the binding loads one library per process."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

NAMES = "anything or leaves_out or no_page or empty or one_token or long_sequences or window_prompts or captured or upper_bounds or thousands"


def main():
    import paper_2306_14048_b200 as pkg

    assert pkg.lib.h2o_debug_bounds_checked() == 1, "this script must run against the checked build"
    at = lambda name: os.path.join(ROOT, "tests", name)
    rc = pytest.main(["-x", "-q", "--tb=short", "-p", "no:cacheprovider", "-m", "gpu", "-k", NAMES, at("test_gpu_pages.py"), at("test_gpu_pages_values.py")])
    if rc == 0:
        print("PAGES_BOUNDS_CASES_PASSED")
    return int(rc)


if __name__ == "__main__":
    sys.exit(main())

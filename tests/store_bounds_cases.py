"""Tests of the K/V store operators run against the checked build of the library (every row, token and partial result verified
before use: a check that fires leaves H2O_ERR_STATE in the status word, which these tests find to be 0).

Executed as a script by tests/test_gpu_store_bounds.py in a process of its own, with H2O_B200_LIB naming
libh2o_b200_bounds.so: the binding loads one library per process."""
import os
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

NAMES = ("point_anywhere or hold_anything or cross_one_token or cross_prompts or long_keys or strides or prefix_shapes or prefix_groups "
         "or last_rows or out_of_range or bit_exact or read_is_exact or beyond_what")


def main():
    import paper_2306_14048_b200 as pkg

    assert pkg.lib.h2o_debug_bounds_checked() == 1, "this script must run against the checked build"
    at = lambda name: os.path.join(ROOT, "tests", name)
    rc = pytest.main(["-x", "-q", "--tb=short", "-p", "no:cacheprovider", "-m", "gpu", "-k", NAMES, at("test_gpu_store_ranges.py"), at("test_gpu_store.py")])
    if rc == 0:
        print("STORE_BOUNDS_CASES_PASSED")
    return int(rc)


if __name__ == "__main__":
    sys.exit(main())

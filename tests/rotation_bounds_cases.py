"""Tests of rotary positions and of the paged cache run against the checked build of the library, with the status words looked at
after every call: a check that fires leaves H2O_ERR_STATE there.

Executed as a script by tests/test_gpu_pages_checked.py in a process of its own, with H2O_B200_LIB naming
libh2o_b200_bounds.so: the binding loads one library per process."""
import os
import sys

import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
sys.path.insert(0, ROOT)

NAMES = "many_tokens or rotation or positions or append or gradient or layouts or few_heads or captured"


def watched(kind, name):
    call = getattr(kind, name)

    def watch(self, *args, **kwargs):
        call(self, *args, **kwargs)
        if not torch.cuda.is_current_stream_capturing():
            torch.cuda.synchronize()
            assert self.status() == 0, name

    setattr(kind, name, watch)


def main():
    import paper_2306_14048_b200 as pkg

    assert pkg.lib.h2o_debug_bounds_checked() == 1, "this script must run against the checked build"
    for kind, name in ((pkg.H2ORotary, "apply"), (pkg.H2OPages, "append"), (pkg.H2OPages, "attend")):
        watched(kind, name)
    at = lambda name: os.path.join(ROOT, "tests", name)
    rc = pytest.main(["-x", "-q", "--tb=short", "-p", "no:cacheprovider", "-m", "gpu", "-k", NAMES, at("test_gpu_rotation.py"), at("test_gpu_pages.py")])
    if rc == 0:
        print("ROTATION_BOUNDS_CASES_PASSED")
    return int(rc)


if __name__ == "__main__":
    sys.exit(main())

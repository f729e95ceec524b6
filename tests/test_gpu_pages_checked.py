"""The checked build (-DH2O_BOUNDS) goes over a rotation's items and over the places of a paged cache's tables before it uses them."""
import os
import re
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2306_14048_b200", "csrc")


@pytest.mark.gpu
def test_rotations_pass_on_the_checked_build():
    import torch

    assert torch.cuda.is_available(), "needs a CUDA device; there is no CPU fallback"
    lib = os.path.join(ROOT, "paper_2306_14048_b200", "libh2o_b200_bounds.so")
    assert os.path.exists(lib)
    res = subprocess.run([sys.executable, os.path.join(ROOT, "tests", "rotation_bounds_cases.py")], env=dict(os.environ, H2O_B200_LIB=lib),
                         capture_output=True, text=True, timeout=900)
    assert res.returncode == 0 and "ROTATION_BOUNDS_CASES_PASSED" in res.stdout, res.stdout[-3000:] + res.stderr[-3000:]


def _source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def _body(text, head):
    """The function that starts with `head`, up to the brace that closes it."""
    at = text.index(head)
    depth, i = 0, text.index("{", at)
    while True:
        depth += {"{": 1, "}": -1}.get(text[i], 0)
        i += 1
        if depth == 0:
            return text[at:i]


def test_attention_reads_the_table_in_one_checked_place():
    entry = _body(_source("store.cuh"), "int table_entry(")
    assert entry.count("pages.table[") == 1 and entry.index("H2O_IN_RANGE(seq") < entry.index("H2O_IN_RANGE(x") < entry.index("pages.table[")
    assert _source("store.cuh").count("pages.table[") == 1
    for name in ("pages_attend_tc.cu", "store_attend_mma.cu", "store_attend_fma.cu", "store_join.cu"):
        assert "pages.table[" not in _source(name), name
    for name in ("pages_attend_tc.cu", "store_attend_mma.cu", "store_attend_fma.cu"):
        assert "table_entry(" in _source(name) and "page_rows_ok(" in _source(name), name


def test_the_rotation_checks_what_it_is_about_to_use():
    kernel = _body(_source("rotate.cu"), "move_kernel(")
    piece = _body(kernel, "auto piece =")
    for what in ("k, here", "head, a.q_heads + 2 * a.kv_heads", "c, cut.per"):  # before the head's address is formed
        assert "H2O_IN_RANGE(%s, a.status)" % what in piece[:piece.index("p.from =")], what
    for kind in piece[piece.index("KIND == Kind::Single"):].split("} else {"):  # the channels, and the sines
        assert kind.count("H2O_IN_RANGE(") >= 2 and "half * here, a.status)" in kind
    for line in kernel.split("\n"):  # the table: behind checks of its own place, not behind the entry's
        if "a.table[" in line:
            assert line.index("H2O_IN_RANGE(s, a.batch") < line.index("H2O_IN_RANGE(in, a.max_pages") < line.index("a.table[")
    assert kernel.count("a.table[") == 1 and "H2O_IN_RANGE(page, a.n_pages" not in kernel
    sines = kernel[kernel.index("half * here; i += kThreads"):]
    assert sines.index("H2O_IN_RANGE(k, here") < sines.index("turn.positions[")

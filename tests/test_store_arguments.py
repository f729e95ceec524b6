"""What the K/V store operators take and refuse before any CUDA call; needs no GPU.  Addresses here are never read."""
import ctypes

import pytest
import torch

HERE = 0x10000  # an aligned address nobody reads


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


def _handle(b, **kw):
    """A handle as the library lays it out: its configuration comes first."""
    f = dict(n_heads=4, head_dim=128, format=b.H2O_BF16, rows=100, row_stride=512, k=HERE, v=HERE)
    f.update(kw)
    c = b.h2o_store_config_t(**f)
    buf = (ctypes.c_char * 2048)()
    ctypes.memmove(buf, ctypes.byref(c), ctypes.sizeof(c))
    return ctypes.cast(buf, ctypes.c_void_p), buf


def _queries(b, **kw):
    f = dict(q=HERE, out=2 * HERE, q_rows=50, dtype=b.H2O_BF16, query_group=2, batch=3, max_q=1)
    f.update(kw)
    return b.h2o_queries_t(**f)


@pytest.mark.parametrize("scale,rc", [(3.4e38, -1), (2.4e38, -1), (2.3e38, -3), (1e-45, -3), (-1.0, -3)])
def test_softmax_scales_that_leave_fp32_are_refused(b, scale, rc):
    """Logits are kept in base 2, so c log2(e) has to be a number.  (-3: past the checks of arguments, no scratch given.)"""
    h, _ = _handle(b, rows=100000)
    q = _queries(b, softmax_scale=scale, batch=1)
    r = b.h2o_ranges_t(HERE, HERE, 50000)
    assert b.lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(r), None, 0, None) == rc
    if rc == -1:
        assert b.lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(r), 1, None, 1, ctypes.byref(r), None, 0, None) == rc
        assert b.lib.h2o_cross_scratch_bytes(h, ctypes.byref(q), ctypes.byref(r)) == 0


def test_poll_limit_needs_a_store(b):
    assert b.lib.h2o_debug_store_set_polls(None, 5) == -1
    h, _ = _handle(b)
    for polls in (0, 7, -1, 2 ** 31 - 1):
        assert b.lib.h2o_debug_store_set_polls(h, polls) == 0

"""How a step over a paged cache is cut into chunks, read off the scratch that a call asks for.  Needs no GPU (the library then counts
on 148 multiprocessors; with one, on its own)."""
import ctypes

import pytest
import torch

HERE = 0x10000  # an aligned address nobody reads
SMS = torch.cuda.get_device_properties(0).multi_processor_count if torch.cuda.is_available() else 148


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


def _chunks(b, batch, heads, group, dim, length, window=0, sinks=0, page=16):
    cfg = b.h2o_pages_config_t(n_heads=heads, head_dim=dim, format=b.H2O_BF16, n_pages=10, page_size=page, k=HERE, v=HERE)
    cfg.head_stride, cfg.row_stride, cfg.page_stride = dim, dim * heads, dim * heads * page
    handle = (ctypes.c_char * 4096)()  # a handle starts with its configuration
    ctypes.memmove(handle, ctypes.byref(cfg), ctypes.sizeof(cfg))
    q = b.h2o_queries_t(q=HERE, out=2 * HERE, q_rows=batch, dtype=b.H2O_BF16, query_group=group, batch=batch, max_q=1)
    s = b.h2o_sequences_t(table=HERE, length=HERE, max_pages=(length + page - 1) // page, max_length=length)
    size = b.lib.h2o_pages_scratch_bytes(ctypes.byref(handle), ctypes.byref(q), ctypes.byref(s), window, sinks)
    rows = batch * heads * group
    for n in range(1, 65):
        if size == (rows * n * dim * 4 + 255) // 256 * 256 + (rows * n * 4 + 255) // 256 * 256:
            return n
    assert size == 0
    return 1


def _at_once(dim, group):
    return SMS * (3 if dim == 64 and group <= 8 else 2)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("group", [1, 4, 16])
@pytest.mark.parametrize("heads", [6, 8, 12, 16, 24, 32, 36])
@pytest.mark.parametrize("length", [5000, 9000, 20000, 45000])
def test_the_blocks_of_one_long_sequence_run_at_once(b, dim, group, heads, length):
    n = _chunks(b, 1, heads, group, dim, length)
    assert heads * n <= _at_once(dim, group)
    if length >= 20000:  # and fill most of the GPU, if they may be many
        assert heads * n >= min(heads * 32, SMS) * 3 // 4


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("batch,heads", [(2, 8), (4, 8), (3, 12), (8, 4)])
@pytest.mark.parametrize("window", [1020, 2500, 4000, 6000])
def test_the_blocks_of_windows_run_at_once(b, dim, batch, heads, window):
    """Sequences far longer than the window have the same number of keys: nothing is left for lengths that differ."""
    assert batch * heads * _chunks(b, batch, heads, 4, dim, 20000, window, 4) <= _at_once(dim, 4)


@pytest.mark.parametrize("batch,heads,length", [(4, 8, 20000), (4, 8, 33000), (9, 4, 20000), (2, 16, 9000)])
def test_heads_of_64_are_cut_finer(b, batch, heads, length):
    """Three of their blocks fit an SM, two with heads of 128: four sequences of 8 heads were 20 % slower with as few chunks."""
    narrow, wide = _chunks(b, batch, heads, 1, 64, length), _chunks(b, batch, heads, 1, 128, length)
    assert narrow >= wide * 5 // 4
    for n, dim in ((narrow, 64), (wide, 128)):  # lengths of two thirds of the longest
        assert batch * heads * n * 2 / 3 <= _at_once(dim, 1)

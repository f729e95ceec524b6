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


def test_strides_that_are_never_used_do_not_matter(b):
    """One head, or one token: its stride says nothing about the memory."""
    from types import SimpleNamespace

    me = SimpleNamespace(_index=-1, head_dim=64, n_heads=1, device="cpu", _h=None)  # (-1: where CPU tensors say they are)
    queries = lambda q, out: b.H2OStore._queries(me, q, out, None, 1, None, 0.0, q.shape[0])
    rows = lambda k, v: b.H2OStore._rows(me, k, v, None, 0)
    one_head = torch.zeros(1, 5, 64).transpose(0, 1)  # [5, 1, 64], the head's stride 5 * 64
    assert one_head.stride() == (64, 320, 1)
    queries(one_head, torch.zeros(5, 1, 64)), queries(torch.zeros(5, 1, 64), one_head)
    assert rows(one_head, torch.zeros(5, 1, 64))[5] == 64
    one_token = torch.zeros(7, 9, 1, 64)[:1, 3]  # [1, 1, 64]
    assert one_token.stride(0) == 576
    queries(one_token, torch.zeros(1, 1, 64))
    assert rows(one_token, torch.zeros(1, 1, 64))[5] == 0
    me.n_heads = 2
    two = torch.zeros(2, 5, 64).transpose(0, 1)
    rows(torch.zeros(7, 9, 2, 64)[:1, 3], torch.zeros(1, 2, 64))
    for call in (lambda: queries(two, torch.zeros(5, 2, 64)), lambda: queries(torch.zeros(5, 2, 64), two), lambda: rows(two, two),
                 lambda: rows(torch.zeros(5, 2, 64), torch.zeros(5, 3, 64)[:, :2]), lambda: rows(torch.zeros(5, 2, 128)[:, :, ::2], torch.zeros(5, 2, 64)),
                 lambda: rows(torch.zeros(5, 2, 64), two)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_stores_with_strides_that_are_never_used(b):
    """The same for a store's rows: one head, and a single row; what they hold is what is attended."""
    x = torch.randn((2, 1, 40, 64), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    q = torch.randn((1, 1, 64), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    at = dict(begin=torch.tensor([3], device="cuda"), length=torch.tensor([30], dtype=torch.int32, device="cuda"), max_len=30)
    outs = []
    for k, v in ((x[0].transpose(0, 1), x[1].transpose(0, 1)), (x[0].transpose(0, 1).contiguous(), x[1].transpose(0, 1))):
        out = torch.empty_like(q)
        b.H2OStore(k, v).cross_attend(q, out=out, **at)
        outs.append(out)
    assert torch.equal(*outs)
    p = (x[0, 0, 3:33].double() @ q[0, 0].double() / 8).softmax(0)
    assert ((p @ x[1, 0, 3:33].double()) - outs[0].double()).abs().max() < 2.0 ** -7  # (outputs below 1: 2^-9 and the sums)
    wide = torch.randn((1, 5, 2, 64), generator=torch.Generator().manual_seed(3)).bfloat16().cuda()
    k, v = wide[:, 1], torch.ones((1, 2, 64), dtype=torch.bfloat16, device="cuda")  # a single row each, of other strides
    out = torch.empty((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    b.H2OStore(k, v).cross_attend(q.expand(1, 2, 64).contiguous(), torch.tensor([0], device="cuda"),
                                  torch.tensor([1], dtype=torch.int32, device="cuda"), out, max_len=1)
    assert (out == 1.0).all()

"""Refusals of the paged cache and of rotary positions, which need no GPU: every argument error is found on the host, before any
CUDA call.  A handle is laid out here as the library does it (its configuration comes first).  Addresses are never read."""
import ctypes
from types import SimpleNamespace

import numpy as np
import pytest
import torch

import pages_reference as ref

HERE = 0x10000  # an aligned address nobody reads


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


def _config(b, **kw):
    f = dict(n_heads=4, head_dim=128, format=b.H2O_BF16, n_pages=10, page_size=16, k=HERE, v=HERE)
    f.update(kw)
    return b.h2o_pages_config_t(**f)


def _handle(b, **kw):
    c = _config(b, **kw)
    if c.page_stride == 0:
        c.head_stride, c.row_stride = c.head_dim, c.head_dim * c.n_heads
        c.page_stride = c.row_stride * c.page_size
    buf = (ctypes.c_char * 4096)()
    ctypes.memmove(buf, ctypes.byref(c), ctypes.sizeof(c))
    return ctypes.cast(buf, ctypes.c_void_p), buf


def _make(kind, defaults, kw):
    defaults.update(kw)
    return kind(**defaults)


def _queries(b, **kw):
    return _make(b.h2o_queries_t, dict(q=HERE, out=2 * HERE, lse=HERE, cu_q=HERE, q_rows=50, dtype=b.H2O_BF16, query_group=2, batch=3, max_q=20), kw)


def _sequences(b, **kw):
    return _make(b.h2o_sequences_t, dict(table=HERE, length=HERE, max_pages=8, max_length=100), kw)


def _tokens(b, **kw):
    return _make(b.h2o_tokens_t, dict(k=HERE, v=HERE, q=HERE, q_out=2 * HERE, cu=HERE, positions=HERE, n_tokens=50, query_group=2, batch=3), kw)


def _rotary(b, **kw):
    return _make(b.h2o_rotary_t, dict(frequency=HERE, axis=HERE, rotary_dim=64, axes=3), kw)


def _refer(x):
    return None if x is None else ctypes.byref(x)


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(n_heads=0), -1), (dict(n_pages=0), -1), (dict(page_size=0), -1), (dict(device=-1), -1),
    (dict(format=2), -2), (dict(format=3), -2), (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(page_size=12), -2),
    (dict(page_size=65544), -2), (dict(n_heads=65536), -2), (dict(k=HERE + 8), -1), (dict(v=HERE + 2), -1),
    (dict(page_stride=8192), -1), (dict(page_stride=8192, row_stride=512, head_stride=100), -1),
    (dict(page_stride=8192, row_stride=516, head_stride=128), -1), (dict(page_stride=8192, row_stride=-512, head_stride=128), -1),
    (dict(page_stride=1 << 40, row_stride=512, head_stride=128), -2),
])
def test_configurations_refused(b, kw, code):
    out = ctypes.c_void_p()
    assert b.lib.h2o_pages_create(ctypes.byref(out), ctypes.byref(_config(b, **kw))) == code
    assert not out.value


def test_null_arguments(b):
    out = ctypes.c_void_p()
    assert b.lib.h2o_pages_create(None, ctypes.byref(_config(b))) == -1
    assert b.lib.h2o_pages_create(ctypes.byref(out), None) == -1
    assert b.lib.h2o_pages_destroy(None) == 0
    assert b.lib.h2o_debug_pages_set_polls(None, 5) == -1
    h, _ = _handle(b)
    q, s, t, r = (ctypes.byref(f(b)) for f in (_queries, _sequences, _tokens, _rotary))
    assert b.lib.h2o_pages_append(None, t, s, r, None) == -1 and b.lib.h2o_pages_append(h, None, s, r, None) == -1
    assert b.lib.h2o_pages_append(h, t, None, r, None) == -1
    assert b.lib.h2o_pages_attend(None, q, s, 0, 0, HERE, 1 << 40, None) == -1
    assert b.lib.h2o_pages_attend(h, None, s, 0, 0, HERE, 1 << 40, None) == -1
    assert b.lib.h2o_pages_attend(h, q, None, 0, 0, HERE, 1 << 40, None) == -1
    assert b.lib.h2o_pages_scratch_bytes(None, q, s, 0, 0) == 0 and b.lib.h2o_pages_scratch_bytes(h, None, None, 0, 0) == 0
    assert b.lib.h2o_rotate(None, HERE, HERE, 1, 5, 4, 128, 0, 0, HERE, 0, 0, None) == -1
    for polls in (0, 7, -1, 2 ** 31 - 1):
        assert b.lib.h2o_debug_pages_set_polls(h, polls) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a device")
def test_no_device_is_an_error(b):
    out = ctypes.c_void_p()
    assert b.lib.h2o_pages_create(ctypes.byref(out), ctypes.byref(_config(b))) == -5


BAD_ROTARY = [(dict(frequency=None), -1), (dict(frequency=HERE + 4), -1), (dict(rotary_dim=0), -1), (dict(rotary_dim=63), -1), (dict(rotary_dim=130), -1),
              (dict(axes=0), -1), (dict(axes=9), -2), (dict(pairs=2), -1), (dict(pairs=-1), -1), (dict(device=-1), -1)]


@pytest.mark.parametrize("kw,code", BAD_ROTARY)
def test_rotary_refusals(b, kw, code):
    h, _ = _handle(b)
    r = ctypes.byref(_rotary(b, **kw))
    assert b.lib.h2o_rotate(r, HERE, HERE, 1, 5, 4, 128, 0, 0, HERE, 0, 0, None) == code
    assert b.lib.h2o_pages_append(h, ctypes.byref(_tokens(b)), ctypes.byref(_sequences(b)), r, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(x=None), -1), (dict(out=None), -1), (dict(x=HERE + 2), -1), (dict(out=HERE + 8), -1), (dict(dtype=2), -2), (dict(n=-1), -1), (dict(n=1 << 31), -2),
    (dict(heads=0), -1), (dict(heads=65536), -2), (dict(dim=0), -1), (dict(dim=100), -2), (dict(dim=520), -2), (dict(dim=56), -1), (dict(xs=500), -1),
    (dict(xs=516), -1), (dict(os=-8), -1), (dict(pos=None), -1), (dict(pos=HERE + 4), -1), (dict(ps=4), -1), (dict(ps=-1), -1),
    (dict(out=HERE, os=1024), -1),
])
def test_rotate_refusals(b, kw, code):
    f = dict(x=HERE, out=2 * HERE, dtype=1, n=5, heads=4, dim=128, xs=0, os=0, pos=HERE, ps=0)
    f.update(kw)
    got = b.lib.h2o_rotate(ctypes.byref(_rotary(b)), f["x"], f["out"], f["dtype"], f["n"], f["heads"], f["dim"], f["xs"], f["os"], f["pos"], f["ps"], 0, None)
    assert got == code


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=HERE + 4), -1), (dict(q_out=None), -1), (dict(q=HERE + 2), -1), (dict(cu=HERE + 2), -1), (dict(positions=HERE + 4), -1),
    (dict(n_tokens=-1), -1), (dict(n_tokens=1 << 31), -2), (dict(batch=-1), -1), (dict(batch=65536), -2), (dict(query_group=0), -1),
    (dict(query_group=20000), -2), (dict(kv_stride=100), -1), (dict(kv_stride=516), -1), (dict(kv_stride=-8), -1), (dict(q_stride=1000), -1),
    (dict(q_out_stride=1028), -1), (dict(position_stride=40), -1), (dict(position_stride=-1), -1), (dict(cu=None, n_tokens=2), -1),
    (dict(q_out=HERE, q_out_stride=2048), -1),
])
def test_append_refusals(b, kw, code):
    h, _ = _handle(b)
    assert b.lib.h2o_pages_append(h, ctypes.byref(_tokens(b, **kw)), ctypes.byref(_sequences(b)), ctypes.byref(_rotary(b)), None) == code


def test_append_for_another_device_is_refused(b):
    h, _ = _handle(b)
    assert b.lib.h2o_pages_append(h, ctypes.byref(_tokens(b)), ctypes.byref(_sequences(b)), ctypes.byref(_rotary(b, device=1)), None) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=HERE + 2), -1), (dict(out=HERE), -1), (dict(lse=HERE + 1), -1), (dict(cu_q=HERE + 2), -1),
    (dict(q_rows=-1), -1), (dict(batch=-1), -1), (dict(max_q=-1), -1), (dict(batch=65536), -2), (dict(query_group=0), -1),
    (dict(query_group=33), -2), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=3e38), -1), (dict(dtype=0), -2),
    (dict(dtype=3), -2), (dict(q_stride=1000), -1), (dict(out_stride=1028), -1), (dict(q_stride=-8), -1), (dict(cu_q=None), -1),
    (dict(cu_q=None, max_q=1, q_rows=2), -1), (dict(q_rows=1 << 31), -2),
])
def test_query_refusals(b, kw, code):
    h, _ = _handle(b)
    assert b.lib.h2o_pages_attend(h, ctypes.byref(_queries(b, **kw)), ctypes.byref(_sequences(b)), 0, 0, HERE, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(table=None), -1), (dict(length=None), -1), (dict(table=HERE + 2), -1), (dict(length=HERE + 1), -1), (dict(max_pages=-1), -1),
    (dict(max_length=-1), -1), (dict(table_stride=7), -1), (dict(table_stride=-8), -1), (dict(table_stride=1 << 40), -2),
])
def test_sequence_refusals(b, kw, code):
    h, _ = _handle(b)
    s = ctypes.byref(_sequences(b, **kw))
    assert b.lib.h2o_pages_attend(h, ctypes.byref(_queries(b)), s, 0, 0, HERE, 1 << 40, None) == code
    assert b.lib.h2o_pages_append(h, ctypes.byref(_tokens(b)), s, None, None) == code


@pytest.mark.parametrize("window,sinks", [(-1, 0), (0, -1), (5, -4)])
def test_window_refusals(b, window, sinks):
    h, _ = _handle(b)
    assert b.lib.h2o_pages_attend(h, ctypes.byref(_queries(b)), ctypes.byref(_sequences(b)), window, sinks, HERE, 1 << 40, None) == -1


def test_empty_calls_do_nothing(b):
    h, _ = _handle(b)
    s = _sequences(b)
    for kw in (dict(batch=0), dict(q_rows=0), dict(max_q=0)):
        q = _queries(b, **kw)
        assert b.lib.h2o_pages_attend(h, ctypes.byref(q), ctypes.byref(s), 0, 0, None, 0, None) == 0
        assert b.lib.h2o_pages_scratch_bytes(h, ctypes.byref(q), ctypes.byref(s), 0, 0) == 0
    for kw in (dict(batch=0), dict(n_tokens=0, k=None, v=None)):
        assert b.lib.h2o_pages_append(h, ctypes.byref(_tokens(b, **kw)), ctypes.byref(s), None, None) == 0
    assert b.lib.h2o_rotate(ctypes.byref(_rotary(b)), None, None, 1, 0, 4, 128, 0, 0, None, 0, 0, None) == 0


def test_packed_arguments_match_the_structures(b):
    for pack, kind, values in ((b._pack_tokens, b.h2o_tokens_t, range(1, 14)), (b._pack_sequences, b.h2o_sequences_t, range(1, 6))):
        got = kind.from_buffer_copy(pack(*values))
        assert ctypes.sizeof(kind) == len(pack(*values))
        assert [getattr(got, n) for n, _ in kind._fields_] == list(values)


# ---- what the Python side refuses, with CPU tensors (whose device index is -1) ----
def _pages(b, heads=2, dim=64, page=16, pages=5, fmt=None):
    me = SimpleNamespace(_index=-1, device="cpu", n_heads=heads, head_dim=dim, format=b.H2O_F32 if fmt is None else fmt, page_size=page,
                         n_pages=pages, _h=None, _need={})
    for name in ("_sequences", "_cu", "_heads"):
        setattr(me, name, getattr(b.H2OPages, name).__get__(me))
    return me


def test_python_argument_checks(b):
    z = torch.zeros
    with pytest.raises(ValueError):
        b.H2OPages(z(4, 16, 2, 64), z(4, 16, 2, 64))  # not on a device
    for kw in (dict(head_dim=60), dict(head_dim=64, rotary_dim=66), dict(head_dim=64, rotary_dim=7), dict(head_dim=64, frequencies=[1.0]),
               dict(head_dim=8, frequencies=[1.0, 2.0, 3.0, float("nan")]), dict(head_dim=8, axes=[0, 1]), dict(head_dim=8, axes=[0, 1, 8, 2]),
               dict(head_dim=8, axes=[0.0, 1.0, 1.0, 0.0]), dict(head_dim=64, pairs="both"), dict(head_dim=1024), dict(head_dim=64, device="cpu")):
        with pytest.raises(ValueError):
            b.H2ORotary(**kw)
    me = _pages(b)
    table, length = z(3, 4, dtype=torch.int32), z(3, dtype=torch.int32)
    me._sequences(table, length, 9), me._sequences(z(3, 9, dtype=torch.int32)[:, 2:6], length, 9)
    for bad in ((table.long(), length), (table, length.long()), (table[:2], length), (table.t().contiguous().t(), length), (table[0].expand(3, 4), length),
                (table[:, ::2], length), (table, length.expand(2, 3)), (table, z(6, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            me._sequences(*bad, 9)
    for cu, batch, tokens in ((None, 3, 2), (z(3, dtype=torch.int32), 3, 9), (z(4), 3, 9), (z(8, dtype=torch.int32)[::2], 3, 9)):
        with pytest.raises(ValueError):
            me._cu(cu, batch, tokens)
    q = z(5, 4, 64)
    assert me._heads(q, q, "out") == (2, 256, 256) and me._heads(z(1, 2, 64), z(1, 2, 64), "out") == (1, 0, 0)
    for a, o in ((z(5, 3, 64), z(5, 3, 64)), (z(5, 4, 128), z(5, 4, 128)), (q, z(5, 2, 64)), (q.bfloat16(), q.bfloat16()), (q, q.bfloat16()),
                 (z(1, 4, 64).expand(5, 4, 64), q), (q, z(4, 5, 64).transpose(0, 1)), (z(5, 4, 128)[..., ::2], q)):
        with pytest.raises(ValueError):
            me._heads(a, o, "out")
    append = b.H2OPages.append
    k = z(3, 2, 64)
    for kw in (dict(v=z(3, 2, 128)), dict(k=z(3, 3, 64), v=z(3, 3, 64)), dict(v=k.bfloat16()), dict(v=z(3, 4, 64)[:, :2]), dict(q=z(3, 4, 64)),
               dict(q_out=z(3, 4, 64)), dict(q=z(4, 4, 64), q_out=z(4, 4, 64)), dict(positions=z(3, dtype=torch.int64)), dict(k=k[:2], v=k[:2]),
               dict(rotary=SimpleNamespace(_index=0, head_dim=64)), dict(rotary=SimpleNamespace(_index=-1, head_dim=128))):
        f = dict(k=k, v=k, table=table, length=length)
        f.update(kw)
        with pytest.raises(ValueError):
            append(me, **f)
    attend = b.H2OPages.attend
    for kw in (dict(max_q=2), dict(lse=z(5, 3)), dict(lse=z(5, 4).double()), dict(lse=z(4, 5).t())):
        f = dict(q=q, table=table, length=length, out=q, max_len=9)
        f.update(kw)
        with pytest.raises(ValueError):
            attend(me, **f)


def test_python_position_checks(b):
    me = SimpleNamespace(_index=-1, device="cpu", axes=3)
    check = b.H2ORotary._positions
    p = torch.zeros((3, 7), dtype=torch.int64)
    assert check(me, p, 7)[1] == 7 and check(me, torch.zeros((3, 20), dtype=torch.int64)[:, 5:12], 7)[1] == 20
    for bad in (p.int(), p[:2], p[0], p.t().contiguous().t(), torch.zeros((3, 14), dtype=torch.int64)[:, ::2], p[:1].expand(3, 7)):
        with pytest.raises(ValueError):
            check(me, bad, 7)
    me.axes = 1
    assert check(me, p[0], 7)[1] == 0 and check(me, p[1:2], 7)[1] == 0


def test_references_agree_with_torch():
    """The tests' own attention and rotation against torch's elementary operations in 64 bits."""
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((n, h, 16), generator=g, dtype=torch.float64) for n, h in ((5, 4), (9, 2), (9, 2)))
    seen = ref.visible(5, 9, 4, 2)
    assert seen[0].tolist() == [True, True, True, True, True, False, False, False, False]
    assert seen[4].tolist() == [True, True, False, False, False, True, True, True, True]
    out, lse, _, _ = ref.attend(q.numpy(), k.numpy(), v.numpy(), seen, 0.25, "f32", False)
    z = torch.einsum("nhd,mhd->hnm", q, k.repeat_interleave(2, 1)) * 0.25
    z = z.masked_fill(~torch.from_numpy(seen), -np.inf)
    np.testing.assert_allclose(out, torch.einsum("hnm,mhd->nhd", z.softmax(-1), v.repeat_interleave(2, 1)).numpy(), atol=1e-12)
    np.testing.assert_allclose(lse, z.logsumexp(-1).T.numpy(), atol=1e-12)
    x = torch.randn((3, 2, 6), generator=g, dtype=torch.float64)
    y, _ = ref.rotate(x.numpy(), np.array([[0, 1, 2]]), [1.0, 0.5], [0, 0], True, "f32")
    z = torch.complex(x[..., :2], x[..., 2:4]) * torch.exp(1j * torch.tensor([[[0.0, 0.0]], [[1.0, 0.5]], [[2.0, 1.0]]], dtype=torch.float64))
    np.testing.assert_allclose(y, torch.cat([z.real, z.imag, x[..., 4:]], -1).numpy(), atol=1e-12)

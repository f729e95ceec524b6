"""Refusals of the paged cache and of rotary positions, which need no GPU: every argument error is found on the host, before any
CUDA call.  A handle is laid out here as the library does it (its configuration comes first).  Addresses are never read."""
import ctypes

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


# ---- what the Python side refuses, with CPU tensors (whose device index is -1): a refusal comes before the library is called ----
def _call(b, name, **kw):
    z = torch.zeros
    if name == "rotate":
        f = dict(at=0, device=-1, dim=64, axes=1, x=z(5, 4, 64), positions=z(5, dtype=torch.int64), out=z(5, 4, 64), inverse=False, stream=0)
    else:
        f = dict(at=0, device=-1, heads=2, dim=64, format=b.H2O_F32)
        if name == "append":
            f.update(k=z(3, 2, 64), v=z(3, 2, 64), table=z(3, 4, dtype=torch.int32), length=z(3, dtype=torch.int32), cu=None, rotary=0, r_device=0, r_dim=0,
                     r_axes=0, positions=None, q=None, q_out=None, stream=0)
        else:
            f.update(q=z(5, 4, 64), table=z(3, 4, dtype=torch.int32), length=z(3, dtype=torch.int32), out=z(5, 4, 64), max_len=9, window=0, sinks=0, cu=None,
                     max_q=1, lse=None, scale=0.0, stream=0)
    assert set(kw) <= set(f)
    f.update(kw)
    return getattr(b._pages, name)(*f.values())


def _refused(b, name, **kw):
    with pytest.raises(ValueError):
        _call(b, name, **kw)


def test_python_argument_checks(b):
    z = torch.zeros
    with pytest.raises(ValueError):
        b.H2OPages(z(4, 16, 2, 64), z(4, 16, 2, 64))  # not on a device
    for kw in (dict(head_dim=60), dict(head_dim=64, rotary_dim=66), dict(head_dim=64, rotary_dim=7), dict(head_dim=64, frequencies=[1.0]),
               dict(head_dim=8, frequencies=[1.0, 2.0, 3.0, float("nan")]), dict(head_dim=8, axes=[0, 1]), dict(head_dim=8, axes=[0, 1, 8, 2]),
               dict(head_dim=8, axes=[0.0, 1.0, 1.0, 0.0]), dict(head_dim=64, pairs="both"), dict(head_dim=1024), dict(head_dim=64, device="cpu")):
        with pytest.raises(ValueError):
            b.H2ORotary(**kw)


@pytest.mark.parametrize("name", ["append", "attend"])
def test_sequences_and_cu_are_checked(b, name):
    z = torch.zeros
    i32 = lambda *n: z(*n, dtype=torch.int32)
    assert _call(b, name) == -1  # (past these checks: no handle)
    for kw in (dict(table=i32(3, 9)[:, 2:6]), dict(table=i32(3, 0)), dict(cu=i32(4))):
        assert _call(b, name, **kw) == -1
    table, length = i32(3, 4), i32(3)
    for kw in (dict(table=table.long()), dict(length=length.long()), dict(table=table[:2]), dict(table=table.t().contiguous().t()),
               dict(table=table[0].expand(3, 4)), dict(table=table[:, ::2]), dict(length=length.expand(2, 3)), dict(length=i32(6)[::2]),
               dict(table=None), dict(length=[1, 2, 3]), dict(cu=i32(3)), dict(cu=z(4)), dict(cu=i32(8)[::2]), dict(cu=i32(4, 1)),
               dict(table=i32(9, 4), length=i32(9))):  # (without cu: a token for each sequence)
        _refused(b, name, **kw)


def test_append_tensors_are_checked(b):
    z = torch.zeros
    k, q = z(3, 2, 64), z(3, 4, 64)
    assert _call(b, "append", q=q, q_out=q) == -1
    assert _call(b, "append", rotary=HERE, r_device=-1, r_dim=64, r_axes=3, positions=z((3, 3), dtype=torch.int64)) == -1
    for kw in (dict(v=z(3, 2, 128)), dict(k=z(3, 3, 64), v=z(3, 3, 64)), dict(v=k.bfloat16()), dict(k=k.bfloat16(), v=k.bfloat16()), dict(v=z(3, 4, 64)[:, :2]),
               dict(k=z(1, 2, 64).expand(3, 2, 64)), dict(k=k[0], v=k[0]), dict(q=q), dict(q_out=q), dict(q=z(4, 4, 64), q_out=z(4, 4, 64)),
               dict(q=q, q_out=q.bfloat16()), dict(q=z(3, 3, 64), q_out=z(3, 3, 64)), dict(positions=z(3, dtype=torch.int64)), dict(k=k[:2], v=k[:2]),
               dict(rotary=HERE, r_device=0, r_dim=64, r_axes=1), dict(rotary=HERE, r_device=-1, r_dim=128, r_axes=1),
               dict(rotary=HERE, r_device=-1, r_dim=64, r_axes=3, positions=z(3, dtype=torch.int64))):
        _refused(b, "append", **kw)


def test_query_tensors_are_checked(b):
    z = torch.zeros
    q = z(5, 4, 64)
    assert _call(b, "attend", lse=z(5, 4)) == -1
    one = z(1, 5, 64).transpose(0, 1)  # one head: its stride says nothing
    assert _call(b, "attend", heads=1, q=one, out=z(5, 1, 64)) == -1
    for kw in (dict(q=z(5, 3, 64), out=z(5, 3, 64)), dict(q=z(5, 4, 128), out=z(5, 4, 128)), dict(out=z(5, 2, 64)), dict(q=q.bfloat16(), out=q.bfloat16()),
               dict(out=q.bfloat16()), dict(q=z(1, 4, 64).expand(5, 4, 64)), dict(out=z(4, 5, 64).transpose(0, 1)), dict(q=z(5, 4, 128)[..., ::2]),
               dict(max_q=2), dict(lse=z(5, 3)), dict(lse=z(5, 4).double()), dict(lse=z(4, 5).t()), dict(max_len=2 ** 40), dict(window=2 ** 31),
               dict(sinks=-2 ** 40), dict(device=0)):
        _refused(b, "attend", **kw)
    with pytest.raises(TypeError):
        b._pages.attend(1, 2)
    with pytest.raises(TypeError):
        _call(b, "attend", max_len="9")


def test_rotate_tensors_are_checked(b):
    z = torch.zeros
    p = z((3, 5), dtype=torch.int64)
    assert _call(b, "rotate") == -1 and _call(b, "rotate", axes=3, positions=p) == -1
    assert _call(b, "rotate", axes=3, positions=z((3, 20), dtype=torch.int64)[:, 5:10]) == -1 and _call(b, "rotate", positions=p[1:2]) == -1
    for bad in (p.int(), p[:2], p[0], p.t().contiguous().t(), z((3, 10), dtype=torch.int64)[:, ::2], p[:1].expand(3, 5)):
        _refused(b, "rotate", axes=3, positions=bad)
    x = z(5, 4, 64)
    for kw in (dict(x=z(5, 4, 128)), dict(out=z(5, 4, 32)), dict(x=x.double(), out=x.double()), dict(out=x.bfloat16()), dict(x=x[0], out=x[0]),
               dict(x=z(1, 4, 64).expand(5, 4, 64)), dict(out=z(4, 5, 64).transpose(0, 1)), dict(device=3), dict(positions=p[0].expand(2, 5)), dict(x=None)):
        _refused(b, "rotate", **kw)


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

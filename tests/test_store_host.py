"""Refusals of the K/V store operators, which need no GPU: every argument error is found on the host, before any CUDA
call.  The handle is laid out here as the library does it (its configuration comes first)."""
import ctypes

import numpy as np
import pytest
import torch

import store_reference as ref


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


HERE = 0x10000  # an aligned address nobody reads


def _config(b, **kw):
    f = dict(n_heads=4, head_dim=128, format=b.H2O_BF16, device=0, rows=100, row_stride=0, k=HERE, v=HERE, k_scale=HERE, v_scale=HERE, status=None)
    f.update(kw)
    return b.h2o_store_config_t(*[f[n] for n, _ in b.h2o_store_config_t._fields_])


def _handle(b, **kw):
    c = _config(b, **kw)
    if c.row_stride == 0:
        c.row_stride = c.n_heads * c.head_dim
    buf = (ctypes.c_char * 1024)()
    ctypes.memmove(buf, ctypes.byref(c), ctypes.sizeof(c))
    return ctypes.cast(buf, ctypes.c_void_p), buf


def _queries(b, **kw):
    f = dict(q=HERE, out=2 * HERE, lse=HERE, cu_q=HERE, q_rows=50, q_stride=0, out_stride=0, softmax_scale=0.0, dtype=b.H2O_BF16,
             query_group=2, batch=3, max_q=20)
    f.update(kw)
    return b.h2o_queries_t(*[f[n] for n, _ in b.h2o_queries_t._fields_])


def _ranges(b, **kw):
    f = dict(begin=HERE, length=HERE, max_length=90)
    f.update(kw)
    return b.h2o_ranges_t(f["begin"], f["length"], f["max_length"])


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=None), -1), (dict(n_heads=0), -1), (dict(rows=0), -1), (dict(device=-1), -1),
    (dict(head_dim=96), -2), (dict(head_dim=256), -2), (dict(format=2), -2), (dict(format=9), -2), (dict(k=HERE + 8), -1),
    (dict(row_stride=511), -1), (dict(row_stride=516), -1), (dict(row_stride=-8), -1), (dict(rows=1 << 31), -2),
    (dict(format=3, k_scale=None), -1), (dict(format=3, v_scale=None), -1), (dict(format=3, row_stride=512), -1),
    (dict(format=3, rows=1 << 30), -2), (dict(n_heads=65536), -2), (dict(row_stride=1 << 40), -2),
])
def test_store_configurations_refused(b, kw, code):
    out = ctypes.c_void_p()
    assert b.lib.h2o_store_create(ctypes.byref(out), ctypes.byref(_config(b, **kw))) == code
    assert not out.value


def test_null_arguments(b):
    out = ctypes.c_void_p()
    assert b.lib.h2o_store_create(None, ctypes.byref(_config(b))) == -1
    assert b.lib.h2o_store_create(ctypes.byref(out), None) == -1
    assert b.lib.h2o_store_destroy(None) == 0
    assert b.lib.h2o_store_write(None, HERE, HERE, 1, 1, 0, None, 0, None) == -1
    assert b.lib.h2o_cross_attend(None, ctypes.byref(_queries(b)), ctypes.byref(_ranges(b)), None, 0, None) == -1
    h, _ = _handle(b)
    assert b.lib.h2o_cross_attend(h, None, ctypes.byref(_ranges(b)), None, 0, None) == -1
    assert b.lib.h2o_cross_attend(h, ctypes.byref(_queries(b)), None, None, 0, None) == -1
    assert b.lib.h2o_cross_scratch_bytes(h, None, None) == 0


@pytest.mark.skipif(torch.cuda.is_available(), reason="without a device")
def test_no_device_is_an_error(b):
    out = ctypes.c_void_p()
    assert b.lib.h2o_store_create(ctypes.byref(out), ctypes.byref(_config(b))) == -5


@pytest.mark.parametrize("kw,code", [
    (dict(k=None), -1), (dict(v=HERE + 4), -1), (dict(n=-1), -1), (dict(dtype=2), -2), (dict(dtype=3), -2), (dict(stride=100), -1),
    (dict(stride=515), -1), (dict(stride=-8), -1), (dict(rows=None, first=-1), -1), (dict(rows=None, first=96), -1),
    (dict(rows=None, first=0, n=101), -1), (dict(n=1 << 31), -2), (dict(rows=HERE + 4), -1), (dict(fmt=1), -2), (dict(fmt=0), -2),
    (dict(rows=None, first=2 ** 62), -1),
])
@pytest.mark.parametrize("call", ["h2o_store_write", "h2o_store_read"])
def test_write_and_read_refusals(b, call, kw, code):
    f = dict(k=HERE, v=HERE, dtype=1, n=5, stride=0, rows=HERE, first=0, fmt=3)
    f.update(kw)
    h, _ = _handle(b, format=f["fmt"])
    assert getattr(b.lib, call)(h, f["k"], f["v"], f["dtype"], f["n"], f["stride"], f["rows"], f["first"], None) == code


def test_nothing_to_write(b):
    h, _ = _handle(b, format=3)
    assert b.lib.h2o_store_write(h, None, None, 1, 0, 0, None, 0, None) == 0


BAD_QUERIES = [
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=HERE + 2), -1), (dict(out=HERE), -1), (dict(lse=HERE + 1), -1), (dict(cu_q=HERE + 2), -1),
    (dict(q_rows=-1), -1), (dict(batch=-1), -1), (dict(max_q=-1), -1), (dict(batch=65536), -2), (dict(query_group=0), -1),
    (dict(query_group=33), -2), (dict(softmax_scale=float("nan")), -1), (dict(softmax_scale=float("inf")), -1), (dict(dtype=0), -2),
    (dict(dtype=2), -2), (dict(q_stride=1000), -1), (dict(out_stride=1028), -1), (dict(q_stride=-8), -1), (dict(cu_q=None), -1),
    (dict(cu_q=None, max_q=1, q_rows=2), -1), (dict(q_rows=1 << 31), -2),
]


@pytest.mark.parametrize("kw,code", BAD_QUERIES)
def test_query_refusals(b, kw, code):
    h, _ = _handle(b)
    q, r = _queries(b, **kw), _ranges(b)
    assert b.lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(r), HERE, 1 << 40, None) == code
    assert b.lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(r), 1, None, 3, ctypes.byref(r), HERE, 1 << 40, None) == code


@pytest.mark.parametrize("kw,code", [(dict(begin=None), -1), (dict(length=None), -1), (dict(begin=HERE + 4), -1), (dict(length=HERE + 2), -1), (dict(max_length=-1), -1)])
def test_range_refusals(b, kw, code):
    h, _ = _handle(b)
    q, good, bad = _queries(b), _ranges(b), _ranges(b, **kw)
    assert b.lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(bad), HERE, 1 << 40, None) == code
    assert b.lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(good), 1, None, 3, ctypes.byref(bad), HERE, 1 << 40, None) == code
    assert b.lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(bad), 1, None, 3, ctypes.byref(good), HERE, 1 << 40, None) == code


@pytest.mark.parametrize("groups,cu,most,code", [(0, HERE, 3, -1), (2, None, 3, -1), (1, None, 2, -1), (1, HERE + 2, 3, -1), (1, HERE, 0, -1), (65536, HERE, 3, -2)])
def test_group_refusals(b, groups, cu, most, code):
    h, _ = _handle(b)
    q, r = _queries(b), _ranges(b)
    assert b.lib.h2o_prefix_attend(h, ctypes.byref(q), ctypes.byref(r), groups, cu, most, ctypes.byref(r), HERE, 1 << 40, None) == code


def test_scratch_is_checked(b):
    h, _ = _handle(b, rows=100000)
    q, r = _queries(b, cu_q=None, max_q=1, batch=1), _ranges(b, max_length=50000)
    need = b.lib.h2o_cross_scratch_bytes(h, ctypes.byref(q), ctypes.byref(r))
    assert need > 0  # a long range for one token is split
    call = lambda p, n: b.lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(r), p, n, None)
    assert call(None, need) == -3 and call(HERE, need - 1) == -3 and call(HERE + 128, need) == -3


def test_empty_calls_do_nothing(b):
    h, _ = _handle(b)
    r = _ranges(b)
    for kw in (dict(batch=0, cu_q=HERE), dict(q_rows=0), dict(max_q=0)):
        q = _queries(b, **kw)
        assert b.lib.h2o_cross_attend(h, ctypes.byref(q), ctypes.byref(r), None, 0, None) == 0
        assert b.lib.h2o_cross_scratch_bytes(h, ctypes.byref(q), ctypes.byref(r)) == 0


def test_python_checks(b):
    with pytest.raises(ValueError):
        b.H2OStore(torch.zeros(4, 2, 128), torch.zeros(4, 2, 128))  # not on a device


def test_reference_quantiser_against_torch():
    """The tests' own quantiser (integer arithmetic) against torch's float8 type."""
    g = torch.Generator().manual_seed(1)
    x = torch.randn((40, 3, 64), generator=g) * torch.exp2(torch.randint(-20, 12, (40, 3, 1), generator=g).float())
    code, scale = ref.quantise(x)
    e = torch.from_numpy(scale.astype(np.int32)) - 127
    y = torch.ldexp(x.transpose(0, 1), -e.unsqueeze(-1)).clamp(-448, 448).to(torch.float8_e4m3fn)
    assert np.array_equal(y.view(torch.uint8).numpy(), code)
    want = torch.ldexp(y.double(), e.unsqueeze(-1)).numpy()
    np.testing.assert_array_equal(ref.values(code, scale), want)
    assert float(torch.finfo(torch.float8_e4m3fn).max) == 448.0


def test_broadcast_tensors_are_refused(b):
    """An expanded tensor has a token stride of 0, which the library would read as dense."""
    from types import SimpleNamespace

    me = SimpleNamespace(_index=-1, head_dim=64, n_heads=2, device="cpu", _h=None)  # (-1: where CPU tensors say they are)
    wide, one = torch.zeros(5, 2, 64), torch.zeros(1, 2, 64)
    queries = lambda q, out: b.H2OStore._queries(me, q, out, None, 1, None, 0.0, 5)
    rows = lambda k: b.H2OStore._rows(me, k, k, None, 0)
    queries(wide, wide.clone())
    rows(wide), rows(one)
    for call in (lambda: queries(one.expand(5, 2, 64), wide), lambda: queries(wide, one.expand(5, 2, 64)),
                 lambda: queries(wide[:, :1].expand(5, 2, 64), wide), lambda: rows(one.expand(5, 2, 64))):
        with pytest.raises(ValueError):
            call()

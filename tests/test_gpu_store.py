"""The K/V store operators on a B200 against 64-bit references: 8-bit write and read, cross attention, shared prefix."""
import math

import numpy as np
import pytest
import torch

import store_reference as ref
from workloads import Workload, make_decode_inputs, make_prompt_inputs

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rows(seed, rows, heads, dim, dtype, spread=True):
    """K or V rows; with `spread` their magnitudes differ by row (an 8-bit row then has its own scale)."""
    g = _gen(seed)
    x = torch.randn((rows, heads, dim), generator=g)
    if spread:
        x = x * torch.exp2(torch.randint(-4, 3, (rows, heads, 1), generator=g).float())
    return x.to(dtype)


def _make(pkg, fmt, k, v, rows_pad=0):
    """A store of these rows, the 64-bit values of its K and V, and its tensors."""
    if fmt == "kv8":
        (ck, sk), (cv, sv) = ref.quantise(k), ref.quantise(v)
        t = [torch.from_numpy(x).cuda() for x in (ck, cv, sk, sv)]
        return pkg.H2OStore(*t), ref.values(ck, sk).transpose(1, 0, 2), ref.values(cv, sv).transpose(1, 0, 2)
    if rows_pad:  # rows of a wider array
        wide = torch.full((k.shape[0], k.shape[1] * k.shape[2] + rows_pad), math.nan, dtype=k.dtype)
        ks, vs = (torch.cat([x.flatten(1), wide[:, -rows_pad:]], 1).cuda()[:, :k[0].numel()].view(k.shape) for x in (k, v))
    else:
        ks, vs = k.cuda(), v.cuda()
    return pkg.H2OStore(ks, vs), k.double().numpy(), v.double().numpy()


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _layout(lengths, seed, gap=3):
    """Ranges of these lengths in a store, in another order and with gaps; total rows."""
    order = torch.randperm(len(lengths), generator=_gen(seed)).tolist()
    at, begin = gap, [0] * len(lengths)
    for i in order:
        begin[i] = at
        at += lengths[i] + gap
    return begin, at


def _poison(k, v, begin, length):
    """NaN and infinities in every row that no range covers."""
    out = torch.ones(k.shape[0], dtype=torch.bool)
    for b, n in zip(begin, length):
        out[b:b + n] = False
    k[out], v[out] = math.nan, math.inf
    return k, v


# ---------------------------------------------------------------------------------------------------------------
# 8-bit write and read
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim,tokens", [(1, 64, 1), (3, 128, 5), (32, 128, 67), (5, 64, 300), (7, 128, 1000)])
def test_write_is_bit_exact_and_leaves_other_rows(pkg, dtype, heads, dim, tokens):
    rows = tokens + 9
    k, v = (_rows(s, tokens, heads, dim, DT[dtype]) for s in (1, 2))
    k[0] = 0.0
    v[-1, 0] *= 2.0 ** -40
    k[tokens // 2, 0] = torch.randn(dim, generator=_gen(5)) * 2.0 ** 17  # beyond the largest scale: saturates
    v[0, 0, 3], v[0, 0, 5], v[0, 0, 6] = math.nan, math.inf, -math.inf
    store = pkg.H2OStore.empty_kv8(rows, heads, dim)
    for t in (store.k, store.v, store.k_scale, store.v_scale):
        t.fill_(0xA5)
    to = torch.randperm(rows, generator=_gen(3))[:tokens]
    store.write(k.cuda(), v.cuda(), rows=to.cuda())
    for x, code, scale in ((k, store.k, store.k_scale), (v, store.v, store.v_scale)):
        want = np.full((heads, rows, dim), 0xA5, np.uint8), np.full((heads, rows), 0xA5, np.uint8)
        c, s = ref.quantise(x)
        want[0][:, to], want[1][:, to] = c, s
        got = code.cpu().numpy()
        nan = (want[0] & 0x7F) == 0x7F
        assert np.array_equal((got & 0x7F) == 0x7F, nan)
        assert np.array_equal(np.where(nan, 0, got), np.where(nan, 0, want[0]))
        assert np.array_equal(scale.cpu().numpy(), want[1])


def test_every_rounding_of_the_8_bit_format(pkg):
    """All bf16 values of a binade range against the largest value of their row: each code, each tie, both signs."""
    bits = torch.arange(0x3A00, 0x4400, dtype=torch.int32)  # bf16 patterns 2^-11 .. 2^9
    x = torch.cat([bits, bits + 0x8000 - 0x10000]).to(torch.int16).view(torch.bfloat16)
    n = (len(x) + 126) // 127
    k = torch.zeros(n * 127, dtype=torch.bfloat16)
    k[: len(x)] = x
    k = torch.cat([k.view(n, 127), torch.full((n, 1), 448.0, dtype=torch.bfloat16)], 1).view(n, 1, 128)
    store = pkg.H2OStore.empty_kv8(n, 1, 128)
    store.write(k.cuda(), (-k).cuda())
    for x, code, scale in ((k, store.k, store.k_scale), (-k, store.v, store.v_scale)):
        c, s = ref.quantise(x)
        assert np.array_equal(code.cpu().numpy(), c) and np.array_equal(scale.cpu().numpy(), s)


@pytest.mark.parametrize("exponent", [-30, -24, -23, -7, 0, 14, 15, 16, 40])
def test_scale_is_the_smallest_power_of_two(pkg, exponent):
    base = torch.tensor([1.0, 1.75, 1.7578125, 1.9921875, 1.25, 1.5], dtype=torch.float32) * 2.0 ** exponent
    k = torch.zeros((6, 1, 64), dtype=torch.float32)
    k[:, 0, 11] = base
    store = pkg.H2OStore.empty_kv8(6, 1, 64)
    store.write(k.cuda(), k.cuda())
    c, s = ref.quantise(k)
    assert np.array_equal(store.k_scale.cpu().numpy(), s) and np.array_equal(store.k.cpu().numpy(), c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_read_is_exact(pkg, dtype, dim):
    rows, heads, n = 517, 5, 301
    code = torch.randint(0, 256, (2, heads, rows, dim), generator=_gen(1), dtype=torch.uint8)
    scale = torch.randint(112, 135, (2, heads, rows), generator=_gen(2), dtype=torch.uint8)
    store = pkg.H2OStore(code[0].cuda(), code[1].cuda(), scale[0].cuda(), scale[1].cuda())
    at = torch.randint(0, rows, (n,), generator=_gen(3))
    at[7], at[8], at[9] = -1, rows, 2 ** 40
    k = torch.full((n, heads, dim), 7.0, dtype=DT[dtype], device="cuda")
    v = k.clone()
    store.read(k, v, rows=at.cuda())
    there = (at >= 0) & (at < rows)
    for got, c, s in ((k, code[0], scale[0]), (v, code[1], scale[1])):
        want = np.full((n, heads, dim), 7.0)
        want[there.numpy()] = ref.values(c, s).transpose(1, 0, 2)[at[there].numpy()]
        np.testing.assert_array_equal(got.double().cpu().numpy(), want)  # 4 significant bits: exact in either type


def test_write_and_read_strided_consecutive_and_out_of_range(pkg):
    heads, dim, n = 4, 64, 33
    packed = _rows(1, n, 2 * heads + 1, dim, torch.bfloat16).cuda()  # K, V and something else of one projection
    k, v = packed[:, :heads], packed[:, heads:2 * heads]
    store = pkg.H2OStore.empty_kv8(64, heads, dim)
    store.write(k, v, first_row=31)
    out = torch.full((n, 2 * heads + 1, dim), 3.0, dtype=torch.float32, device="cuda")
    store.read(out[:, 1:heads + 1], out[:, heads + 1:], first_row=31)
    for x, got in ((k, out[:, 1:heads + 1]), (v, out[:, heads + 1:])):
        c, s = ref.quantise(x)
        np.testing.assert_array_equal(got.double().cpu().numpy(), ref.values(c, s).transpose(1, 0, 2))
    assert (out[:, 0] == 3.0).all()
    before = [t.clone() for t in (store.k, store.v, store.k_scale, store.v_scale)]
    store.write(k[:3], v[:3], rows=_i64([-1, 64, -2 ** 40]))  # all outside: nothing happens
    store.write(k[:0], v[:0])
    for a, b in zip(before, (store.k, store.v, store.k_scale, store.v_scale)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------------------------------------------
# Cross attention
# ---------------------------------------------------------------------------------------------------------------
def _check_cross(pkg, fmt, q_dtype, heads, group, dim, q_len, kv_len, seed=0, max_len=None, scale=0.0, q_pad=0, rows_pad=0,
                 poison=True, stream=None):
    begin, rows = _layout(kv_len, seed + 1)
    k, v = (_rows(seed + s, rows, heads, dim, DT.get(fmt, torch.bfloat16)) for s in (2, 3))
    if poison:
        _poison(k, v, begin, kv_len)
    store, k64, v64 = _make(pkg, fmt, k, v, rows_pad)
    tokens, hq = sum(q_len), heads * group
    extra = 2  # rows of q behind the last sequence
    q = torch.randn((tokens + extra, hq * dim + q_pad), generator=_gen(seed + 4)).to(DT[q_dtype])
    q = (q * 1.5).cuda()[:, :hq * dim].view(tokens + extra, hq, dim)
    out = torch.full((tokens + extra, hq * dim + q_pad), 5.0, dtype=DT[q_dtype], device="cuda")[:, :hq * dim].view(tokens + extra, hq, dim)
    lse = torch.full((tokens + extra, hq), 5.0, dtype=torch.float32, device="cuda")
    cu = np.concatenate([[0], np.cumsum(q_len)]).tolist()
    torch.cuda.synchronize()
    one = all(n == 1 for n in q_len)
    kw = {} if one else {"cu_q": _i32(cu), "max_q": max(q_len)}
    store.cross_attend(q, _i64(begin), _i32(kv_len), out, max_len=max(kv_len) if max_len is None else max_len, lse=lse,
                       softmax_scale=scale, stream=stream, **kw)
    torch.cuda.synchronize()
    assert store.status() == 0
    c = scale if scale > 0 else 1.0 / math.sqrt(dim)
    for b, n in enumerate(q_len):
        sl = slice(cu[b], cu[b] + n)
        m = kv_len[b] if max_len is None else min(kv_len[b], max_len)
        want = ref.attend(q[sl].double().cpu().numpy(), k64[begin[b]:begin[b] + m], v64[begin[b]:begin[b] + m],
                          [m] * n, float(np.float32(c)), fmt, q_dtype)
        ref.compare(out[sl], want[0], want[2], "out of sequence %d" % b)
        ref.compare(lse[sl], want[1], want[3], "lse of sequence %d" % b)
    assert (out[tokens:] == 5.0).all() and (lse[tokens:] == 5.0).all()
    return out, lse


FORMATS = [("f32", "f32"), ("bf16", "bf16"), ("kv8", "bf16"), ("kv8", "f32")]


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(1, 1), (3, 1), (2, 4), (1, 5), (2, 8), (1, 12), (1, 32)])
def test_cross_one_token(pkg, fmt, q_dtype, dim, heads, group):
    kv = [1, 0, 15, 16, 17, 31, 32, 33, 64, 65, 130, 257]
    _check_cross(pkg, fmt, q_dtype, heads, group, dim, [1] * len(kv), kv, seed=group)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(2, 1), (1, 3), (1, 8)])
def test_cross_prompts(pkg, fmt, q_dtype, dim, heads, group):
    _check_cross(pkg, fmt, q_dtype, heads, group, dim, [5, 0, 1, 130, 64, 33], [70, 9, 200, 129, 0, 1], seed=group)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("q,kv", [(1, 4099), (7, 2049), (257, 1023), (40, 1500)])
def test_cross_long_keys_are_split_and_joined(pkg, fmt, q_dtype, dim, q, kv):
    _check_cross(pkg, fmt, q_dtype, 1, 1, dim, [q, q], [kv, 300], seed=q)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
def test_cross_strides_scale_and_cut_lengths(pkg, fmt, q_dtype):
    pad = 0 if fmt == "kv8" else 24
    _check_cross(pkg, fmt, q_dtype, 2, 2, 64, [3, 40, 1], [100, 77, 300], q_pad=40, rows_pad=pad, scale=0.3)
    _check_cross(pkg, fmt, q_dtype, 2, 2, 128, [1, 1, 1], [100, 77, 300], q_pad=8, rows_pad=pad, max_len=80)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
def test_cross_more_sequences_than_blocks(pkg, fmt, q_dtype):
    kv = torch.randint(0, 40, (300,), generator=_gen(1)).tolist()
    _check_cross(pkg, fmt, q_dtype, 3, 1, 64, [1] * 300, kv)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("n", [1, 70, 150])
def test_cross_extreme_values(pkg, fmt, q_dtype, n):
    """NaN among the keys reaches the queries that see it and no others; logits of -infinity count for nothing; large
    logits do not overflow."""
    dim, heads = 128, 1
    kv = [40, 40, 40, 70]
    begin, rows = _layout(kv, 1)
    dt = DT.get(fmt, torch.bfloat16)
    k, v = (_rows(s, rows, heads, dim, dt, spread=False) for s in (2, 3))
    v[begin[0] + 3, 0, 9] = math.nan          # sequence 0: one channel of one value
    if fmt != "kv8":                          # (8-bit rows have no infinities)
        k[begin[1]:begin[1] + 40, 0, 0] = -math.inf    # sequence 1: every logit -infinity
        k[begin[2]:begin[2] + 39, 0, 0] = -math.inf    # sequence 2: all but one
    k[begin[3] + 5] *= 50.0                   # sequence 3: logits of hundreds
    store, k64, v64 = _make(pkg, fmt, k, v)
    q = torch.randn((4 * n, heads, dim), generator=_gen(4)).to(DT[q_dtype]).abs().cuda()
    out, lse = torch.empty_like(q), torch.empty((4 * n, heads), dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": _i32([0, n, 2 * n, 3 * n, 4 * n]), "max_q": n}
    store.cross_attend(q, _i64(begin), _i32(kv), out, max_len=70, lse=lse, **kw)
    with np.errstate(invalid="ignore"):
        for b in range(4):
            sl = slice(b * n, b * n + n)
            want = ref.attend(q[sl].double().cpu().numpy(), k64[begin[b]:begin[b] + kv[b]], v64[begin[b]:begin[b] + kv[b]],
                              [kv[b]] * n, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
            ref.compare(out[sl], want[0], want[2], "out %d" % b)
            ref.compare(lse[sl], want[1], want[3], "lse %d" % b)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("n", [1, 70, 150])
@pytest.mark.parametrize("at", [0, 200, 299])
def test_cross_nan_keys(pkg, fmt, q_dtype, n, at):
    """A NaN key gives NaN to every query that sees it, wherever it lies; its neighbours in the store give nothing."""
    dim = 128
    k, v = (_rows(s, 600, 1, dim, DT.get(fmt, torch.bfloat16), spread=False) for s in (2, 3))
    k[at, 0, 77] = math.nan
    if at == 0:
        k[:300, 0, 77] = math.nan  # nothing but NaN
    store, k64, v64 = _make(pkg, fmt, k, v)
    q = torch.randn((2 * n, 1, dim), generator=_gen(4)).to(DT[q_dtype]).cuda()
    out, lse = torch.empty_like(q), torch.empty((2 * n, 1), dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": _i32([0, n, 2 * n]), "max_q": n}
    store.cross_attend(q, _i64([0, 300]), _i32([300, 299]), out, max_len=300, lse=lse, **kw)
    assert torch.isnan(out[:n]).all() and torch.isnan(lse[:n]).all()
    want = ref.attend(q[n:].double().cpu().numpy(), k64[300:599], v64[300:599], [299] * n, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
    ref.compare(out[n:], want[0], want[2], "out")
    ref.compare(lse[n:], want[1], want[3], "lse")


@pytest.mark.parametrize("fmt,q_dtype", [("kv8", "bf16"), ("kv8", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("n", [1, 70])
def test_cross_queries_and_values_of_far_apart_magnitudes(pkg, fmt, q_dtype, n):
    """Values whose rows differ by 2^20 in size, the large ones with the small probabilities; tiny and huge queries."""
    dim, rows = 128, 96
    k, v = (_rows(s, rows, 1, dim, torch.bfloat16, spread=False) for s in (2, 3))
    v[::2] *= 2.0 ** -12
    v[1::2] *= 2.0 ** 6
    u = torch.nn.functional.normalize(torch.randn(dim, generator=_gen(5)), dim=0)
    k[:, 0] *= 0.1
    k[1::2, 0] -= (8.0 * u).to(torch.bfloat16)  # the large values get probabilities of e^-12 or so
    store, k64, v64 = _make(pkg, fmt, k, v)
    q = (torch.randn((3 * n, 1, dim), generator=_gen(4)) * 0.1 + 17.0 * u).to(DT[q_dtype])
    q[n:2 * n] *= 2.0 ** -30
    q[2 * n:] *= 2.0 ** 3
    q = q.cuda()
    out, lse = torch.empty_like(q), torch.empty((3 * n, 1), dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": _i32([0, n, 2 * n, 3 * n]), "max_q": n}
    store.cross_attend(q, _i64([0, 0, 0]), _i32([rows] * 3), out, max_len=rows, lse=lse, **kw)
    want = ref.attend(q.double().cpu().numpy(), k64, v64, [rows] * 3 * n, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


# ---------------------------------------------------------------------------------------------------------------
# Shared prefix
# ---------------------------------------------------------------------------------------------------------------
def _check_prefix(pkg, fmt, q_dtype, heads, group, dim, q_len, own_len, members, prefix_len, seed=0):
    begin, rows = _layout(prefix_len + own_len, seed + 1)
    k, v = (_rows(seed + s, rows, heads, dim, DT.get(fmt, torch.bfloat16)) for s in (2, 3))
    _poison(k, v, begin, prefix_len + own_len)
    store, k64, v64 = _make(pkg, fmt, k, v)
    groups = len(members)
    pb, ob = begin[:groups], begin[groups:]
    tokens, hq, batch = sum(q_len), heads * group, len(q_len)
    q = (torch.randn((tokens + 1, hq, dim), generator=_gen(seed + 4)) * 1.5).to(DT[q_dtype]).cuda()
    out = torch.full_like(q, 5.0)
    lse = torch.full((tokens + 1, hq), 5.0, dtype=torch.float32, device="cuda")
    cu = np.concatenate([[0], np.cumsum(q_len)]).tolist()
    cg = np.concatenate([[0], np.cumsum(members)]).tolist()
    kw = {} if all(n == 1 for n in q_len) else {"cu_q": _i32(cu), "max_q": max(q_len)}
    if groups > 1:
        kw.update(cu_group=_i32(cg), max_group=max(members))
    store.prefix_attend(q, _i64(pb), _i32(prefix_len), _i64(ob), _i32(own_len), out, max_prefix=max(prefix_len),
                        max_own=max(own_len), lse=lse, **kw)
    torch.cuda.synchronize()
    assert store.status() == 0
    which = np.repeat(np.arange(groups), members)
    for b in range(batch):
        g, n = which[b], q_len[b]
        p0, p1, o0 = pb[g], prefix_len[g], ob[b]
        kk, vv = (np.concatenate([x[p0:p0 + p1], x[o0:o0 + own_len[b]]]) for x in (k64, v64))
        seen = [p1 + max(0, own_len[b] - (n - 1 - i)) for i in range(n)]
        sl = slice(cu[b], cu[b] + n)
        want = ref.attend(q[sl].double().cpu().numpy(), kk, vv, seen, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
        ref.compare(out[sl], want[0], want[2], "out of sequence %d" % b)
        ref.compare(lse[sl], want[1], want[3], "lse of sequence %d" % b)
    assert (out[tokens:] == 5.0).all() and (lse[tokens:] == 5.0).all()


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group,batch", [(1, 1, 1), (2, 1, 7), (1, 4, 5), (2, 2, 40), (1, 8, 33), (1, 1, 150)])
def test_prefix_one_token(pkg, fmt, q_dtype, dim, heads, group, batch):
    own = torch.randint(0, 70, (batch,), generator=_gen(batch)).tolist()
    own[0] = 0
    _check_prefix(pkg, fmt, q_dtype, heads, group, dim, [1] * batch, own, [batch], [777], seed=batch)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
def test_prefix_groups_and_empty_ranges(pkg, fmt, q_dtype, dim):
    members = [3, 0, 1, 6]
    _check_prefix(pkg, fmt, q_dtype, 2, 2, dim, [1] * 10, [4, 0, 9, 0, 65, 64, 63, 1, 2, 0], members, [100, 50, 0, 1], seed=3)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,group", [(2, 1), (1, 4)])
def test_prefix_prompts(pkg, fmt, q_dtype, dim, heads, group):
    """Several query tokens to a sequence, causal among its own rows; more query tokens than own rows; none at all."""
    q_len, own = [5, 1, 0, 70, 33, 9, 129], [5, 40, 7, 70, 64, 4, 200]
    _check_prefix(pkg, fmt, q_dtype, heads, group, dim, q_len, own, [7], [130], seed=group)
    _check_prefix(pkg, fmt, q_dtype, heads, group, dim, q_len, own, [2, 1, 3, 1], [0, 64, 65, 300], seed=group + 9)


# ---------------------------------------------------------------------------------------------------------------
# As they are used
# ---------------------------------------------------------------------------------------------------------------
def test_two_runs_give_the_same_bits(pkg):
    for fmt, q_dtype in FORMATS:
        for n in (1, 90):
            a, b = (_check_cross(pkg, fmt, q_dtype, 2, 2, 128, [n] * 3, [2000, 700, 65], seed=5) for _ in range(2))
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_on_another_stream(pkg):
    s = torch.cuda.Stream()
    for fmt, q_dtype in FORMATS:
        _check_cross(pkg, fmt, q_dtype, 1, 2, 128, [1, 1], [1800, 65], stream=s)
        _check_cross(pkg, fmt, q_dtype, 1, 2, 64, [70, 3], [180, 65], stream=s)


def test_captured_graphs_follow_lengths_and_do_not_share_scratch(pkg):
    """Two captured graphs of one store, replayed at the same time on two streams with other lengths than captured."""
    dim, rows, batch = 128, 6000, 3
    k, v = (_rows(s, rows, 1, dim, torch.bfloat16) for s in (1, 2))
    store, k64, v64 = _make(pkg, "bf16", k, v)
    runs = []
    for i in range(2):
        q = torch.randn((batch, 2, dim), generator=_gen(10 + i)).bfloat16().cuda()
        r = dict(q=q, out=torch.empty_like(q), lse=torch.empty((batch, 2), dtype=torch.float32, device="cuda"),
                 begin=_i64([0, 100, 2000]), length=_i32([10, 10, 10]), stream=torch.cuda.Stream(), graph=torch.cuda.CUDAGraph())
        call = lambda r=r: store.cross_attend(r["q"], r["begin"], r["length"], r["out"], max_len=3500, lse=r["lse"])
        with torch.cuda.stream(r["stream"]):
            call()
        torch.cuda.synchronize()
        with torch.cuda.graph(r["graph"], stream=r["stream"]):
            call()
        runs.append(r)
    lengths = [[3500, 0, 1234], [77, 3001, 3400]]
    for r, n in zip(runs, lengths):
        r["length"].copy_(_i32(n))
    torch.cuda.synchronize()
    for _ in range(20):
        for r in runs:
            with torch.cuda.stream(r["stream"]):
                r["graph"].replay()
    torch.cuda.synchronize()
    for r, n in zip(runs, lengths):
        for b in range(batch):
            at = int(r["begin"][b])
            want = ref.attend(r["q"][b:b + 1].double().cpu().numpy(), k64[at:at + n[b]], v64[at:at + n[b]], [n[b]],
                              float(np.float32(1 / math.sqrt(dim))), "bf16", "bf16")
            ref.compare(r["out"][b:b + 1], want[0], want[2], "out")
            ref.compare(r["lse"][b:b + 1], want[1], want[3], "lse")


@pytest.mark.parametrize("fmt", ["bf16", "kv8", "f32"])
@pytest.mark.parametrize("n", [1, 70])
def test_rows_beyond_32_bit_offsets(pkg, fmt, n):
    dim, heads = 128, 2
    if fmt == "kv8":
        rows = (1 << 32) // (heads * dim) + 1000  # the second head's rows start beyond 2^31 bytes and end beyond 2^32
        ck = torch.empty((heads, rows, dim), dtype=torch.uint8, device="cuda")
        sk = torch.empty((heads, rows), dtype=torch.uint8, device="cuda")
        store = pkg.H2OStore(ck, ck, sk, sk)  # K and V are the same memory here
        at = rows - 300
        x = _rows(1, 300, heads, dim, torch.bfloat16)
        store.write(x.cuda(), x.cuda(), first_row=at)
        c, s = ref.quantise(x)
        k64 = ref.values(c, s).transpose(1, 0, 2)
        back = torch.empty((300, heads, dim), dtype=torch.float32, device="cuda")
        store.read(back, back.clone(), first_row=at)
        np.testing.assert_array_equal(back.double().cpu().numpy(), k64)
    else:
        stride = heads * dim + (1 << 20)
        rows = (1 << 32) // (stride * (2 if fmt == "bf16" else 4)) + 700
        base = torch.empty(rows * stride, dtype=DT[fmt], device="cuda")
        k = base.as_strided((rows, heads, dim), (stride, dim, 1))
        at = rows - 300
        x = _rows(1, 300, heads, dim, DT[fmt])
        k[at:] = x.cuda()
        store = pkg.H2OStore(k, k)
        k64 = x.double().numpy()
    q_dtype = "f32" if fmt == "f32" else "bf16"
    q = torch.randn((n, heads, dim), generator=_gen(3)).to(DT[q_dtype]).cuda()
    out, lse = torch.empty_like(q), torch.empty((n, heads), dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": _i32([0, n]), "max_q": n}
    store.cross_attend(q, _i64([at]), _i32([300]), out, max_len=300, lse=lse, **kw)
    want = ref.attend(q.double().cpu().numpy(), k64, k64, [300] * n, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


def test_device_arrays_that_point_outside_are_cut(pkg):
    """begin, length and cu_q are device arrays the host never sees: whatever they hold, the kernels stay in bounds."""
    dim, rows = 128, 200
    for fmt, q_dtype in FORMATS:
        k, v = (_rows(s, rows, 1, dim, DT.get(fmt, torch.bfloat16)) for s in (1, 2))
        store, k64, v64 = _make(pkg, fmt, k, v)
        q = torch.randn((4, 1, dim), generator=_gen(3)).to(DT[q_dtype]).cuda()
        out, lse = torch.full_like(q, 5.0), torch.empty((4, 1), dtype=torch.float32, device="cuda")
        store.cross_attend(q, _i64([-5, 150, 2 ** 40, 0]), _i32([20, 2 ** 30, 7, -3]), out, max_len=2 ** 31 - 1, lse=lse)
        for b, (at, n) in enumerate([(0, 20), (150, 50), (0, 0), (0, 0)]):
            want = ref.attend(q[b:b + 1].double().cpu().numpy(), k64[at:at + n], v64[at:at + n], [n],
                              float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
            ref.compare(out[b:b + 1], want[0], want[2], "out")
            ref.compare(lse[b:b + 1], want[1], want[3], "lse")
        out.fill_(5.0)
        store.cross_attend(q, _i64([0, 0]), _i32([9, 9]), out, max_len=9, cu_q=_i32([-7, 3, 2 ** 31 - 1]), max_q=2)
        assert (out[2] == 5.0).all() and (out[[0, 1, 3]] != 5.0).any(-1).all()  # token 2 is a third one of sequence 0


def test_decoder_layer_with_cache_store_and_prefix(pkg):
    """A run of them together: a decoder step with an H2O cache for its own tokens (self attention with eviction) and
    cross attention to encoder states that were quantised as they were written; then samples of one prompt whose own
    rows are appended to the store step by step."""
    heads, dim, batch = 4, 128, 3
    wl = Workload("layer", batch, heads, dim, "bf16", (40, 97, 64), 3, (8, 8, 8), (8, 8, 8), 1, 77)
    cache = pkg.H2OCache(wl.batch, heads, dim, wl.dtype, wl.heavy, wl.recent)
    q, k, v, cu = make_prompt_inputs(wl, device="cuda")
    x = torch.empty_like(q)
    cache.prefill_select(q, k, v, cu, x)
    enc_len = [50, 120, 1]
    enc = torch.nn.functional.pad(torch.tensor(enc_len).cumsum(0), (1, 0))
    ek, ev = (_rows(s, int(enc[-1]), heads, dim, torch.bfloat16) for s in (5, 6))
    store = pkg.H2OStore.empty_kv8(int(enc[-1]) + 400, heads, dim)
    store.write(ek.cuda(), ev.cuda())
    k64, v64 = (ref.values(*ref.quantise(t)).transpose(1, 0, 2) for t in (ek, ev))
    scale = float(np.float32(1 / math.sqrt(dim)))
    y = torch.empty_like(x)
    store.cross_attend(x, _i64(enc[:-1].tolist()), _i32(enc_len), y, max_len=120, cu_q=_i32(list(cu)), max_q=97)
    for step in range(3):
        dq, dk, dv = make_decode_inputs(wl, step, device="cuda")
        o = torch.empty_like(dq)
        cache.decode_step(dq, dk, dv, o)
        z = torch.empty_like(o)
        store.cross_attend(o, _i64(enc[:-1].tolist()), _i32(enc_len), z, max_len=120)
        for b in range(batch):
            sl = slice(int(enc[b]), int(enc[b + 1]))
            want = ref.attend(o[b:b + 1].double().cpu().numpy(), k64[sl], v64[sl], [enc_len[b]], scale, "kv8", "bf16")
            ref.compare(z[b:b + 1], want[0], want[2], "cross step")
    for b in range(batch):
        sl, qs = slice(int(enc[b]), int(enc[b + 1])), slice(int(cu[b]), int(cu[b + 1]))
        want = ref.attend(x[qs].double().cpu().numpy(), k64[sl], v64[sl], [enc_len[b]] * int(cu[b + 1] - cu[b]), scale, "kv8", "bf16")
        ref.compare(y[qs], want[0], want[2], "cross prompt")
    assert cache.status() == 0
    cache.close()
    # samples of one prompt: the prefix is the encoder's rows of sequence 1; each sample's rows are appended
    samples, p0, p1 = 5, int(enc[1]), 120
    own0 = [int(enc[-1]) + 20 * b for b in range(samples)]
    mine = [np.zeros((2, 0, heads, dim)) for _ in range(samples)]
    for step in range(4):
        nq, nk, nv = (torch.randn((samples, heads, dim), generator=_gen(100 * step + s)).bfloat16() for s in range(3))
        store.write(nk.cuda(), nv.cuda(), rows=_i64([b + step for b in own0]))
        o, nqc = torch.empty_like(nq).cuda(), nq.cuda()
        store.prefix_attend(nqc, _i64([p0]), _i32([p1]), _i64(own0), _i32([step + 1] * samples), o, max_prefix=p1, max_own=20)
        nk64, nv64 = (ref.values(*ref.quantise(t)).transpose(1, 0, 2) for t in (nk, nv))
        for b in range(samples):
            mine[b] = np.concatenate([mine[b], np.stack([nk64[b], nv64[b]])[:, None]], 1)
            want = ref.attend(nq[b:b + 1].double().numpy(), np.concatenate([k64[p0:p0 + p1], mine[b][0]]),
                              np.concatenate([v64[p0:p0 + p1], mine[b][1]]), [p1 + step + 1], scale, "kv8", "bf16")
            ref.compare(o[b:b + 1], want[0], want[2], "sample")


# (query tokens of the sequences, their own rows, sequences of the groups, their prefixes), by how they are worked on:
# few rows and keys in one launch; few rows in chunks; many rows of a group and few of a sequence; many of both, with the
# prefix in one piece and in several
SHAPES = [
    ([2, 4, 0, 3], [2, 70, 9, 33], [2, 2], [33, 440]),
    ([1, 3, 2, 4], [1, 64, 2, 300], [2, 2], [2100, 31]),
    ([1] * 40, list(range(40)), [25, 15], [1500, 700]),
    ([40, 17, 64, 33], [40, 20, 200, 33], [3, 1], [96, 65]),
    ([60, 130, 33], [200, 130, 40], [3], [5000]),
]


def _prefix_case(pkg, fmt, q_dtype, dim, shape, seed, group=2, heads=1):
    """Tensors of such a call, with `call` and `check`; the sequences' own ranges and the prefixes may be changed."""
    q_len, own, members, pre = shape
    begin, rows = _layout(pre + own, seed + 1)
    k, v = (_rows(seed + s, rows, heads, dim, DT.get(fmt, torch.bfloat16)) for s in (2, 3))
    store, k64, v64 = _make(pkg, fmt, k, v)
    cu, cg = (np.concatenate([[0], np.cumsum(x)]).tolist() for x in (q_len, members))
    hq = heads * group
    r = dict(q=(torch.randn((cu[-1] + 1, hq, dim), generator=_gen(seed + 4)) * 1.5).to(DT[q_dtype]).cuda(), store=store,
             pb=_i64(begin[:len(pre)]), pl=_i32(pre), ob=_i64(begin[len(pre):]), ol=_i32(own), cu=_i32(cu), cg=_i32(cg))
    r["out"], r["lse"] = torch.full_like(r["q"], 5.0), torch.full((cu[-1] + 1, hq), 5.0, dtype=torch.float32, device="cuda")

    def call(stream=None, **kw):
        most = dict(max_prefix=max(pre), max_own=max(own), max_q=max(q_len), max_group=max(members))
        most.update(kw)
        store.prefix_attend(r["q"], r["pb"], r["pl"], r["ob"], r["ol"], r["out"], cu_group=r["cg"], cu_q=r["cu"], lse=r["lse"],
                            stream=stream, **most)

    def check(untouched=()):
        assert store.status() == 0
        pb, pl, ob, ol = (r[x].tolist() for x in ("pb", "pl", "ob", "ol"))
        which = np.repeat(np.arange(len(members)), members)
        for b, n in enumerate(q_len):
            sl, g = slice(cu[b], cu[b] + n), which[b]
            if b in untouched:
                assert (r["out"][sl] == 5.0).all() and (r["lse"][sl] == 5.0).all()
                continue
            kk, vv = (np.concatenate([x[pb[g]:pb[g] + pl[g]], x[ob[b]:ob[b] + ol[b]]]) for x in (k64, v64))
            seen = [pl[g] + max(0, ol[b] - (n - 1 - i)) for i in range(n)]
            want = ref.attend(r["q"][sl].double().cpu().numpy(), kk, vv, seen, float(np.float32(1 / math.sqrt(dim))), fmt, q_dtype)
            ref.compare(r["out"][sl], want[0], want[2], "out of sequence %d" % b)
            ref.compare(r["lse"][sl], want[1], want[3], "lse of sequence %d" % b)
        assert (r["out"][cu[-1]:] == 5.0).all() and (r["lse"][cu[-1]:] == 5.0).all()

    return r, call, check


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_shapes(pkg, fmt, q_dtype, dim, shape):
    _, call, check = _prefix_case(pkg, fmt, q_dtype, dim, SHAPES[shape], 30 + shape, heads=2)
    call()
    check()


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_graphs_replayed_at_once(pkg, fmt, q_dtype, shape):
    """Two captured calls on two streams at the same time, and eager ones on a third, with other ranges than captured."""
    runs = []
    for i in range(2):
        r, call, check = _prefix_case(pkg, fmt, q_dtype, 128, SHAPES[shape], 50 + i)
        r["stream"], graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        r["stream"].wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(r["stream"]):
            call()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=r["stream"]):
            call()
        runs.append((r, graph, check))
    third = torch.cuda.Stream()
    e, eager, check_eager = _prefix_case(pkg, fmt, q_dtype, 128, SHAPES[shape], 70)
    for i, (r, _, _) in enumerate(runs):
        r["pl"].sub_(torch.tensor([7 + 20 * i] + [i] * (len(r["pl"]) - 1), device="cuda", dtype=torch.int32))
        r["ol"].sub_(1 + i).clamp_(min=0)
        r["out"].fill_(5.0), r["lse"].fill_(5.0)
    torch.cuda.synchronize()
    for _ in range(10):
        for r, graph, _ in runs:
            with torch.cuda.stream(r["stream"]):
                graph.replay()
        eager(stream=third)
    torch.cuda.synchronize()
    for _, _, check in runs:
        check()
    check_eager()


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_ranges_may_be_the_same(pkg, fmt, q_dtype, shape):
    """All sequences with one own range, which lies in the prefix, and all groups with one prefix."""
    r, call, check = _prefix_case(pkg, fmt, q_dtype, 64, SHAPES[shape], 90)
    r["pb"].fill_(0), r["pl"].fill_(31)
    r["ob"].fill_(5), r["ol"].copy_(r["ol"].clamp(max=25))
    call()
    check()


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_beyond_what_the_call_allows_for(pkg, fmt, q_dtype, shape):
    """Longer ranges are cut, sequences and tokens beyond the bounds are left out; nothing else changes."""
    r, call, check = _prefix_case(pkg, fmt, q_dtype, 128, SHAPES[shape], 110)
    pre, own = int(r["pl"].max()) - 9, int(r["ol"].max()) // 2
    call(max_prefix=pre, max_own=own)
    r["pl"].clamp_(max=pre), r["ol"].clamp_(max=own)  # (for the check)
    check()
    q_len, _, members, _ = SHAPES[shape]
    if max(q_len) == 1:
        r["out"].fill_(5.0), r["lse"].fill_(5.0)
        call(max_group=members[0] - 2)
        check(untouched=(members[0] - 2, members[0] - 1))
    else:  # the last token of the longest sequence
        r["out"].fill_(5.0), r["lse"].fill_(5.0)
        call(max_q=max(q_len) - 1)
        b = int(np.argmax(q_len))
        last = int(r["cu"][b + 1]) - 1
        assert (r["out"][last] == 5.0).all() and (r["lse"][last] == 5.0).all()
        assert (r["out"][:last] != 5.0).any(-1).all()



@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_of_nothing(pkg, fmt, q_dtype, shape):
    r, call, check = _prefix_case(pkg, fmt, q_dtype, 64, SHAPES[shape], 130)
    r["pl"].zero_(), r["ol"].zero_()
    for kw in (dict(), dict(max_prefix=0), dict(max_own=0), dict(max_prefix=0, max_own=0)):
        r["out"].fill_(5.0), r["lse"].fill_(5.0)
        call(**kw)
        check()


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_prefix_nan_stays_with_its_group(pkg, fmt, q_dtype, shape):
    """A NaN among the first group's prefix: every query of that group is NaN, no other; then one among a sequence's own."""
    q_len, own, members, pre = SHAPES[shape]
    for where in ("prefix", "own"):
        r, call, check = _prefix_case(pkg, fmt, q_dtype, 128, SHAPES[shape], 150)
        at = int(r["pb"][0]) + pre[0] // 2 if where == "prefix" else int(r["ob"][1])
        if fmt == "kv8":
            r["store"].k[:, at, 3] = 0x7F
        else:
            r["store"].k[at, :, 3] = math.nan
        call()
        hit = range(members[0]) if where == "prefix" else [1]
        for b in hit:  # (every token sees row 0 of its own range, where it has one)
            sl = slice(int(r["cu"][b]), int(r["cu"][b + 1]))
            assert torch.isnan(r["out"][sl]).all() and torch.isnan(r["lse"][sl]).all()
            r["out"][sl], r["lse"][sl] = 5.0, 5.0
        check(untouched=list(hit))


def test_broadcast_store_rows_are_refused(pkg):
    one = torch.zeros((1, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        pkg.H2OStore(one.expand(9, 2, 64), one.expand(9, 2, 64))


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,length", [(1, 300), (70, 300), (70, 700), (150, 700)])
def test_cross_one_key_at_every_place(pkg, fmt, q_dtype, dim, n, length):
    """The same store row at every place of a range: NaN there gives NaN everywhere; a logit there that is hundreds above
    all before it takes the whole weight."""
    at, batch = 800, 97
    g = _gen(7)
    u = torch.nn.functional.normalize(torch.randn(dim, generator=g), dim=0)
    q = ((torch.randn((n, 1, dim), generator=g) * 0.05 + 6.0 * u).to(DT[q_dtype])).repeat(batch, 1, 1).cuda()
    begin = [at - 7 * i if i % 2 else at - i for i in range(batch)]
    kw = {} if n == 1 else {"cu_q": _i32([n * i for i in range(batch + 1)]), "max_q": n}
    for what in ("nan", 400.0, 1100.0, 20000.0):
        k, v = (_rows(s, 1600, 1, dim, DT.get(fmt, torch.bfloat16), spread=False) for s in (2, 3))
        if what == "nan":
            k[at, 0, 5] = math.nan
        else:
            k[at, 0] = (u * what / 6.0 * math.sqrt(dim)).to(k.dtype)  # a logit of about `what`
        store, k64, v64 = _make(pkg, fmt, k, v)
        out, lse = torch.empty_like(q), torch.empty((batch * n, 1), dtype=torch.float32, device="cuda")
        store.cross_attend(q, _i64(begin), _i32([length] * batch), out, max_len=length, lse=lse, **kw)
        for b in range(batch):
            sl, here = slice(b * n, b * n + n), at < begin[b] + length
            if here and what == "nan":
                assert torch.isnan(out[sl]).all() and torch.isnan(lse[sl]).all(), b
            elif here:  # the others' weights are below e^-100
                x = (q[b * n:b * n + n, 0].double().cpu().numpy() @ k64[at, 0]) * float(np.float32(1 / math.sqrt(dim)))
                assert x.min() > 200.0
                want = np.broadcast_to(v64[at], (n, 1, dim))
                ref.compare(out[sl], want, np.abs(want) * 2.0 ** -7 + 1e-30, "out %d" % b)
                size = (np.abs(q[sl, 0].double().cpu().numpy()) @ np.abs(k64[at, 0])) * float(np.float32(1 / math.sqrt(dim)))
                ref.compare(lse[sl, 0], x, size * (dim + 8) * 2.0 ** -23, "lse %d" % b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim,tokens,scattered", [(2, 64, 65607, True), (1, 128, 65538, False), (5, 128, 4999, True)])
def test_write_and_read_many_tokens(pkg, dtype, heads, dim, tokens, scattered):
    """Several tokens to a thread with a remainder, and more tokens than one launch takes."""
    rows = tokens + 5
    k, v = (_rows(s, tokens, heads, dim, DT[dtype]) for s in (1, 2))
    store = pkg.H2OStore.empty_kv8(rows, heads, dim)
    for t in (store.k, store.v, store.k_scale, store.v_scale):
        t.fill_(0x77)
    to = torch.randperm(rows, generator=_gen(3))[:tokens] if scattered else torch.arange(3, tokens + 3)
    at = dict(rows=to.cuda()) if scattered else dict(first_row=3)
    store.write(k.cuda(), v.cuda(), **at)
    back = [torch.empty((tokens, heads, dim), dtype=torch.float32, device="cuda") for _ in range(2)]
    store.read(*back, **at)
    for x, code, scale, got in ((k, store.k, store.k_scale, back[0]), (v, store.v, store.v_scale, back[1])):
        c, s = ref.quantise(x)
        want = np.full((heads, rows, dim), 0x77, np.uint8), np.full((heads, rows), 0x77, np.uint8)
        want[0][:, to], want[1][:, to] = c, s
        assert np.array_equal(code.cpu().numpy(), want[0]) and np.array_equal(scale.cpu().numpy(), want[1])
        np.testing.assert_array_equal(got.double().cpu().numpy(), ref.values(c, s).transpose(1, 0, 2))


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("n", [1, 3, 40])
def test_store_of_one_row_and_the_last_rows(pkg, fmt, q_dtype, n):
    """A store of a single row; and ranges that end with the store, inside a tile."""
    for rows, length in ((1, 1), (37, 37), (131, 5)):
        k, v = (_rows(s, rows, 2, 64, DT.get(fmt, torch.bfloat16)) for s in (1, 2))
        store, k64, v64 = _make(pkg, fmt, k, v)
        q = torch.randn((n, 2, 64), generator=_gen(3)).to(DT[q_dtype]).cuda()
        out = torch.empty_like(q)
        kw = {} if n == 1 else {"cu_q": _i32([0, n]), "max_q": n}
        store.cross_attend(q, _i64([rows - length]), _i32([length]), out, max_len=length, **kw)
        want = ref.attend(q.double().cpu().numpy(), k64[rows - length:], v64[rows - length:], [length] * n,
                          float(np.float32(1 / math.sqrt(64))), fmt, q_dtype)
        ref.compare(out, want[0], want[2], "out")

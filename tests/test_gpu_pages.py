"""Rotary positions, appending to a paged cache and attention over it, on a B200 against 64-bit references."""
import math

import numpy as np
import pytest
import torch

import pages_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _randn(seed, *shape):
    return torch.randn(shape, generator=_gen(seed))


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _sums(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(int).tolist()


# ---------------------------------------------------------------------------------------------------------------
# Rotation
# ---------------------------------------------------------------------------------------------------------------
def _frequencies(rotary_dim, base=10000.0):
    return [base ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]


def _axis_of(half, axes, seed=0):
    a = torch.randint(0, axes, (half,), generator=_gen(seed)).numpy()
    a[-1] = axes - 1
    return a


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("dim,rotary_dim,axes", [(8, 2, 1), (8, 8, 1), (64, 64, 1), (64, 16, 2), (72, 72, 2), (80, 20, 1), (128, 128, 3),
                                                 (128, 96, 1), (128, 6, 2), (256, 64, 8), (512, 512, 3), (504, 504, 1)])
@pytest.mark.parametrize("tokens,heads", [(1, 1), (3, 5), (130, 3)])
def test_rotation(pkg, dtype, pairs, dim, rotary_dim, axes, tokens, heads):
    axis, freq = _axis_of(rotary_dim // 2, axes), _frequencies(rotary_dim)
    r = pkg.H2ORotary(dim, rotary_dim=rotary_dim, frequencies=freq, axes=None if axes == 1 else axis, pairs=pairs)
    x = (_randn(1, tokens, heads, dim) * 3).to(DT[dtype])
    pos = torch.randint(0, 5000, (axes, tokens), generator=_gen(2))
    pos[:, 0] = 0
    pos[0, -1] = 4000000
    for inverse in (False, True):
        want, tol = ref.rotate(x.double().numpy(), pos.numpy(), freq, np.minimum(axis, axes - 1), pairs == "halves", dtype, inverse)
        out = torch.full((tokens + 1, heads, dim), 7.0, dtype=DT[dtype], device="cuda")
        r.apply(x.cuda(), pos.cuda(), out[:tokens], inverse=inverse)
        ref.compare(out[:tokens], want, tol, "rotated")
        assert (out[tokens:] == 7.0).all()
        here = x.cuda()
        r.apply(here, pos.cuda() if axes > 1 else pos.cuda()[0], here, inverse=inverse)  # in place
        assert torch.equal(here, out[:tokens])
        if rotary_dim < dim:
            assert torch.equal(here[..., rotary_dim:].cpu(), x[..., rotary_dim:])


@pytest.mark.parametrize("position", [0, -1, -70000, 2 ** 20 + 1, 2 ** 31 + 12345, -2 ** 33])
def test_far_positions_keep_their_angle(pkg, position):
    freq = _frequencies(128)
    r = pkg.H2ORotary(128, frequencies=freq)
    x = _randn(1, 2, 2, 128)
    pos = torch.tensor([[position, position + 1]])
    out = torch.empty((2, 2, 128), device="cuda")
    r.apply(x.cuda(), pos.cuda(), out)
    ref.compare(out, *ref.rotate(x.double().numpy(), pos.numpy(), freq, [0] * 64, True, "f32"), "far")


def test_default_frequencies(pkg):
    x, pos = _randn(1, 5, 2, 64), torch.arange(5)
    out = torch.empty((5, 2, 64), device="cuda")
    pkg.H2ORotary(64, rotary_dim=32, base=500.0, pairs="neighbours").apply(x.cuda(), pos.cuda(), out)
    ref.compare(out, *ref.rotate(x.double().numpy(), pos.numpy()[None], _frequencies(32, 500.0), [0] * 16, False, "f32"), "base 500")


def test_rotation_of_strided_heads_and_empty_calls(pkg):
    packed = _randn(1, 9, 7, 64).to(torch.bfloat16).cuda()  # queries, keys and values of one projection
    r = pkg.H2ORotary(64)
    pos = torch.arange(9, device="cuda") * 1000
    out = torch.full((9, 5, 64), 3.0, dtype=torch.bfloat16, device="cuda")
    r.apply(packed[:, 4:6], pos, out[:, 1:3])
    want, tol = ref.rotate(packed[:, 4:6].double().cpu().numpy(), pos.cpu().numpy()[None], _frequencies(64), [0] * 32, True, "bf16")
    ref.compare(out[:, 1:3], want, tol, "strided")
    assert (out[:, 0] == 3.0).all() and (out[:, 3:] == 3.0).all()
    before = packed.clone()
    r.apply(packed[:, 4:6], pos, packed[:, 4:6])
    assert torch.equal(packed[:, 4:6], out[:, 1:3]) and torch.equal(packed[:, :4], before[:, :4]) and torch.equal(packed[:, 6], before[:, 6])
    r.apply(packed[:0, :2], pos[:0], out[:0, :2])
    many = torch.zeros((2, 20), dtype=torch.int64, device="cuda")  # positions that lie in a larger array
    many[:, 3:12] = pos
    two = pkg.H2ORotary(64, axes=[0, 1] * 16)
    two.apply(before[:, 4:6], many[:, 3:12], out[:, 1:3])
    ref.compare(out[:, 1:3], want, tol, "positions of a larger array")


def test_infinities_and_nan_stay_in_their_pair(pkg):
    x = torch.ones((1, 1, 64))
    x[0, 0, 3], x[0, 0, 40] = math.nan, math.inf
    out = torch.empty((1, 1, 64), device="cuda")
    pkg.H2ORotary(64).apply(x.cuda(), torch.tensor([5], device="cuda"), out)
    bad = ~torch.isfinite(out.cpu()[0, 0])
    assert bad.nonzero().flatten().tolist() == [3, 8, 35, 40]


def test_the_inverse_is_the_gradient(pkg):
    """<g, R(x + h e) - R(x - h e)> / 2h against (R^-1 g)_e, and against the formula's own derivative."""
    dim, tokens, heads = 64, 3, 2
    freq, axis = _frequencies(dim), _axis_of(dim // 2, 3)
    r = pkg.H2ORotary(dim, frequencies=freq, axes=axis, pairs="neighbours")
    pos = torch.tensor([[3, 70, 900], [5, 5, 6], [1, 2, 40]], device="cuda")
    x, g = _randn(1, tokens, heads, dim).cuda(), _randn(2, tokens, heads, dim).cuda()
    grad, up, down = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    r.apply(g, pos, grad, inverse=True)
    want, tol = ref.rotate(g.double().cpu().numpy(), pos.cpu().numpy(), freq, axis, False, "f32", inverse=True)
    ref.compare(grad, want, tol, "gradient")
    h = 0.5  # the map is linear: a difference is exact up to rounding, (2^-21.6 + 2^-24) times values below 10, over 2h
    for c in range(0, dim, 7):
        e = torch.zeros_like(x)
        e[..., c] = h
        r.apply(x + e, pos, up)
        r.apply(x - e, pos, down)
        change = ((up.double() - down.double()) * g.double()).sum(-1)
        assert (change / (2 * h) - grad[..., c].double()).abs().max() < dim * 10 * 10 * 2.0 ** -21
    back = torch.empty_like(x)
    r.apply(x, pos, up)
    r.apply(up, pos, back, inverse=True)
    assert (back - x).abs().max() < 2 * 5 * 2.0 ** -20  # two rotations of values below 5


# ---------------------------------------------------------------------------------------------------------------
# A paged cache on the host
# ---------------------------------------------------------------------------------------------------------------
class Pool:
    """Pages in one of several layouts, K and V in 64 bits by sequence and row, and a shuffled table."""

    def __init__(self, pkg, dtype, heads, dim, page, rows, layout="rows", seed=0, spare=3, fill=math.nan, width=0):
        per = [(n + page - 1) // page for n in rows]
        pages = sum(per) + spare
        t = DT[dtype]
        shape = {"rows": (pages, page, heads, dim), "heads": (pages, heads, page, dim), "both": (pages, 2, page, heads, dim),
                 "wide": (pages, page + 8, heads + 1, dim)}[layout]
        def one():
            return torch.full(shape, fill, dtype=t, device="cuda")
        if layout == "both":
            x = one()
            self.k, self.v = x[:, 0], x[:, 1]
        elif layout == "heads":
            self.k, self.v = one().transpose(1, 2), one().transpose(1, 2)
        elif layout == "wide":
            self.k, self.v = one()[:, 8:, 1:], one()[:, 8:, 1:]
        else:
            self.k, self.v = one(), one()
        order = torch.randperm(pages, generator=_gen(seed + 11)).tolist()
        self.width = max(max(per + [1]), width)
        self.table = [[-1] * self.width for _ in rows]
        at = 0
        for b, n in enumerate(per):
            self.table[b][:n] = order[at:at + n]
            at += n
        self.page, self.rows = page, rows
        self.pages = pkg.H2OPages(self.k, self.v)

    def fill(self, b, k, v, first=0):
        """Rows first, first + 1, .. of sequence b from [n, heads, dim]."""
        for x in range(k.shape[0]):
            e = self.table[b][(first + x) // self.page]
            self.k[e, (first + x) % self.page] = k[x].to(self.k)
            self.v[e, (first + x) % self.page] = v[x].to(self.v)


# ---------------------------------------------------------------------------------------------------------------
# Append
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["rows", "heads", "both", "wide"])
@pytest.mark.parametrize("heads,group,dim,page,new,held,rotary_dim,pairs,axes", [
    (1, 1, 64, 8, [1], [0], 64, "halves", 1),
    (3, 2, 128, 16, [1, 1, 1, 1], [0, 15, 16, 100], 128, "halves", 1),
    (2, 4, 128, 24, [5, 0, 77, 1, 24], [3, 9, 0, 23, 24], 32, "neighbours", 3),
    (8, 1, 64, 64, [130, 1, 63], [1, 64, 2], 12, "halves", 2),
    (5, 3, 64, 16, [33] * 40, list(range(40)), 64, "neighbours", 1),
])
def test_append(pkg, dtype, layout, heads, group, dim, page, new, held, rotary_dim, pairs, axes):
    rows = [a + b for a, b in zip(new, held)]
    pool = Pool(pkg, dtype, heads, dim, page, rows, layout, fill=5.0)
    tokens, hq, cu = sum(new), heads * group, _sums(new)
    freq, axis = _frequencies(rotary_dim), _axis_of(rotary_dim // 2, axes)
    r = pkg.H2ORotary(dim, rotary_dim=rotary_dim, frequencies=freq, axes=axis if axes > 1 else None, pairs=pairs)
    k, v, q = (_randn(s, tokens + 2, h, dim).to(DT[dtype]).cuda() for s, h in ((1, heads), (2, heads), (3, hq)))
    q_out = torch.full_like(q, 9.0)
    pos = torch.randint(0, 100000, (axes, tokens + 2), generator=_gen(4))
    own_pos = np.array([[m - n + i for n, m in zip(new, rows) for i in range(n)] + [0, 0]] * axes)
    kw = {} if all(n == 1 for n in new) else {"cu": _i32(cu)}
    want_k, want_v = pool.k.double().cpu().numpy(), pool.v.double().cpu().numpy()
    tol_k = np.zeros_like(want_k)
    for positions in (None, pos.cuda()):
        p = own_pos if positions is None else pos.numpy()
        pool.pages.append(k, v, _i32(pool.table), _i32(rows), rotary=r, positions=positions, q=q, q_out=q_out, **kw)
        kr, kt = ref.rotate(k.double().cpu().numpy(), p, freq, np.minimum(axis, axes - 1), pairs == "halves", dtype)
        for b in range(len(new)):
            for i in range(new[b]):
                x = held[b] + i
                e, o = pool.table[b][x // page], x % page
                want_k[e, o], tol_k[e, o], want_v[e, o] = kr[cu[b] + i], kt[cu[b] + i], v[cu[b] + i].double().cpu().numpy()
        ref.compare(pool.k, want_k, tol_k, "K")
        np.testing.assert_array_equal(pool.v.double().cpu().numpy(), want_v)
        qr, qt = ref.rotate(q.double().cpu().numpy(), p, freq, np.minimum(axis, axes - 1), pairs == "halves", dtype)
        ref.compare(q_out[:tokens], qr[:tokens], qt[:tokens], "q")
        assert (q_out[tokens:] == 9.0).all()  # tokens of no sequence
    plain = pool.k.clone()
    pool.pages.append(k, v, _i32(pool.table), _i32(rows), **kw)  # as they are
    for b in range(len(new)):
        for i in range(new[b]):
            x = held[b] + i
            plain[pool.table[b][x // page], x % page] = k[cu[b] + i]
    assert torch.equal(pool.k, plain)


def test_append_leaves_out_rows_that_do_not_exist(pkg):
    heads, dim, page = 2, 64, 8
    pool = Pool(pkg, "bf16", heads, dim, page, [40], fill=5.0)
    table = _i32([[0, -1, 7, 2, 99999], [1, 1 << 30, 3, -5, 4]])
    n_pages = pool.pages.n_pages
    assert n_pages == 8
    before = pool.k.clone()
    k, v, q = (_randn(s, 24, heads, dim).to(torch.bfloat16).cuda() for s in (1, 2, 3))
    out = torch.zeros_like(q)
    r = pkg.H2ORotary(dim)
    # sequence 0: rows 4 .. 15 (page 0, no page); sequence 1: rows -5 .. 6, of which the first five do not exist
    pool.pages.append(k, v, table, _i32([16, 7]), cu=_i32([0, 12, 24]), rotary=r, q=q, q_out=out)
    want = before.clone()
    want_v = before.clone()
    pos = list(range(4, 16)) + list(range(-5, 7))
    turned, tol = ref.rotate(k.double().cpu().numpy(), np.array([pos]), _frequencies(dim), [0] * 32, True, "bf16")
    got_k, got_v = pool.k.clone(), pool.v.clone()
    for t, x in enumerate(pos):
        if (t < 12 and x < 8) or (t >= 12 and x >= 0):
            e = 0 if t < 12 else 1
            ref.compare(got_k[e, x], turned[t], tol[t], "token %d" % t)
            assert torch.equal(got_v[e, x], v[t])
            got_k[e, x], got_v[e, x] = 5.0, 5.0
    assert torch.equal(got_k, want) and torch.equal(got_v, want_v)
    ref.compare(out, *ref.rotate(q.double().cpu().numpy(), np.array([pos]), _frequencies(dim), [0] * 32, True, "bf16"), "queries")
    # beyond the table, entries outside the pool, empty and broken cu arrays: nothing moves
    pool.k.fill_(5.0), pool.v.fill_(5.0)
    for length, cu in (([48, 0], [0, 8, 8]), ([40, 40], [0, 1, 2]), ([2 ** 31 - 1, -7], [0, 2, 24]), ([16, 16], [30, 40, 50]), ([16, 16], [24, 0, 0])):
        pool.pages.append(k, v, table[:, :5], _i32(length), cu=_i32(cu), rotary=r)
        if (length, cu) == ([40, 40], [0, 1, 2]):
            assert torch.equal(pool.v[4, 7], v[1])
            pool.k[4, 7], pool.v[4, 7] = 5.0, 5.0
        assert (pool.k == 5.0).all() and (pool.v == 5.0).all(), (length, cu)
    assert pool.pages.status() == 0


def test_append_in_place_queries_and_strides(pkg):
    heads, group, dim, n = 2, 2, 64, 19
    packed = _randn(1, n, 2 * heads + heads * group, dim).to(torch.bfloat16).cuda()
    q, k, v = packed[:, :4], packed[:, 4:6], packed[:, 6:]
    pool = Pool(pkg, "bf16", heads, dim, 8, [n], fill=0.0)
    r = pkg.H2ORotary(dim)
    want, tol = ref.rotate(q.double().cpu().numpy(), np.arange(n)[None], _frequencies(dim), [0] * 32, True, "bf16")
    keep = packed[:, 4:].clone()
    pool.pages.append(k, v, _i32(pool.table), _i32([n]), cu=_i32([0, n]), rotary=r, q=q, q_out=q)
    ref.compare(q, want, tol, "q in place")
    assert torch.equal(packed[:, 4:], keep)
    pool.pages.append(k[:0], v[:0], _i32(pool.table)[:0], _i32([n])[:0])
    pool.pages.append(k[:0], v[:0], _i32(pool.table), _i32([n]), cu=_i32([0, 0]))
    assert torch.equal(pool.v[pool.table[0][0]], v[:8])


# ---------------------------------------------------------------------------------------------------------------
# Attention
# ---------------------------------------------------------------------------------------------------------------
def _one_bf16(tokens, group):
    return tokens * group > 16


def _check_attend(pkg, dtype, heads, group, dim, page, new, rows, window=0, sinks=0, layout="rows", seed=0, max_len=None, scale=0.0, q_pad=0,
                  stream=None, lse=True, freed=True, width=0, most=None):
    """Rows that no query sees hold NaN (their pages, where whole, belong to nobody); rows of q behind the last sequence stay."""
    pool = Pool(pkg, dtype, heads, dim, page, rows, layout, seed, width=width)
    tokens, hq, extra = sum(new), heads * group, 2
    k, v = ([(_randn(seed + s + 10 * b, m, heads, dim) * (1.0 if s == 3 else 1.3)).to(DT[dtype]) for b, m in enumerate(rows)] for s in (2, 3))
    for b, m in enumerate(rows):
        pool.fill(b, k[b], v[b])
        seen = ref.visible(new[b], m, window, sinks).any(0) if 0 < new[b] <= m else np.ones(m, bool)
        if window and freed:
            for x in range(m):
                if not seen[x]:
                    e = pool.table[b][x // page]
                    pool.k[e, x % page], pool.v[e, x % page] = math.nan, math.inf
            for i in range((m + page - 1) // page):
                if not seen[i * page:(i + 1) * page].any():
                    pool.table[b][i] = [-1, 1 << 30, 0][i % 3]
    q = (_randn(seed + 4, tokens + extra, hq * dim + q_pad) * 1.5).to(DT[dtype]).cuda()[:, :hq * dim].view(tokens + extra, hq, dim)
    out = torch.full((tokens + extra, hq * dim + q_pad), 5.0, dtype=DT[dtype], device="cuda")[:, :hq * dim].view(tokens + extra, hq, dim)
    sums = torch.full((tokens + extra, hq), 5.0, dtype=torch.float32, device="cuda") if lse else None
    cu = _sums(new)
    table, length = _i32(pool.table), _i32(rows)
    torch.cuda.synchronize()
    kw = {} if all(n == 1 for n in new) else {"cu": _i32(cu), "max_q": max(new + [1])}
    pool.pages.attend(q, table, length, out, max_len=max(rows) if max_len is None else max_len, window=window, sinks=sinks, lse=sums,
                      softmax_scale=scale, stream=stream, **kw)
    torch.cuda.synchronize()
    assert pool.pages.status() == 0
    for b, n in enumerate(new):
        if n == 0:
            continue
        sl = slice(cu[b], cu[b] + n)
        m = rows[b]
        if n <= m:
            seen = ref.visible(n, m, window, sinks)
        else:  # more tokens than rows: the first ones see nothing
            seen = np.zeros((n, m), bool)
            seen[n - m:] = ref.visible(m, m, window, sinks)
        want = ref.attend(q[sl].double().cpu().numpy(), k[b].double().numpy(), v[b].double().numpy(), seen, ref.scale_of(dim, scale), dtype,
                          _one_bf16(max(new), group))
        ref.compare(out[sl], want[0], want[2], "out of sequence %d" % b)
        if lse:
            ref.compare(sums[sl], want[1], want[3], "lse of sequence %d" % b)
    assert (out[tokens:] == 5.0).all() and (sums is None or (sums[tokens:] == 5.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [8, 16, 24, 32, 64, 200])
@pytest.mark.parametrize("group", [1, 4])
def test_one_token(pkg, dtype, dim, page, group):
    _check_attend(pkg, dtype, 3, group, dim, page, [1] * 9, [1, 2, 7, 8, 31, 32, 33, 130, 517])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("layout", ["heads", "both", "wide"])
@pytest.mark.parametrize("new", [1, 7, 50])
def test_layouts(pkg, dtype, layout, new):
    _check_attend(pkg, dtype, 3, 2, 128, 16, [new] * 3, [60, 50, 333], layout=layout)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,group,dim,page", [(1, 1, 128, 16), (2, 3, 64, 32), (2, 8, 128, 64), (1, 32, 64, 8)])
@pytest.mark.parametrize("rows", [[3000], [5000, 1, 700]])
def test_long_sequences_are_cut_and_joined(pkg, dtype, heads, group, dim, page, rows):
    _check_attend(pkg, dtype, heads, group, dim, page, [1] * len(rows), rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,group,dim,page", [(8, 1, 128, 16), (8, 2, 64, 32), (8, 16, 128, 64), (12, 1, 64, 16), (37, 1, 128, 16), (38, 1, 128, 16)])
@pytest.mark.parametrize("rows", [[5003], [4100, 1, 2500]])
def test_few_heads_of_long_sequences(pkg, dtype, heads, group, dim, page, rows):
    _check_attend(pkg, dtype, heads, group, dim, page, [1] * len(rows), rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 64), (64, 24), (128, 8)])
@pytest.mark.parametrize("new,rows,group", [
    ([2, 1, 5], [2, 1, 90], 1), ([16, 0, 3], [300, 40, 3], 1), ([17, 1], [17, 260], 1), ([100, 128, 129], [100, 500, 129], 1),
    ([40, 7], [333, 7], 4), ([300, 257], [300, 1000], 2), ([5, 9, 70], [1, 0, 3], 1), ([600], [600], 1),
])
def test_prompts(pkg, dtype, dim, page, new, rows, group):
    _check_attend(pkg, dtype, 2, group, dim, page, new, rows)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 32), (128, 24), (64, 128)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (5, 4), (31, 0), (32, 40), (100, 4), (64, 16), (1000, 4), (2 ** 31 - 1, 3), (7, 2 ** 31 - 1)])
@pytest.mark.parametrize("group", [1, 5])
def test_window_steps(pkg, dtype, dim, page, window, sinks, group):
    _check_attend(pkg, dtype, 2, group, dim, page, [1] * 6, [1, 6, 40, 200, 333, 700], window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 16), (128, 64), (128, 24)])
@pytest.mark.parametrize("window,sinks", [(1, 0), (3, 2), (20, 4), (100, 0), (130, 70), (500, 4), (2 ** 31 - 1, 0)])
@pytest.mark.parametrize("new,rows,group", [([3, 1, 9], [3, 200, 600], 1), ([130, 2], [400, 700], 1), ([300, 40], [300, 900], 2)])
def test_window_prompts(pkg, dtype, dim, page, window, sinks, new, rows, group):
    _check_attend(pkg, dtype, 2, group, dim, page, new, rows, window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (900, 4), (2500, 100)])
@pytest.mark.parametrize("new", [1, 12, 33, 140])
def test_long_windows_are_cut_and_joined(pkg, dtype, window, sinks, new):
    _check_attend(pkg, dtype, 1, 1, 128, 16, [new, 1], [6000, 2900], window, sinks)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 20])
def test_strides_scales_bounds_and_no_lse(pkg, dtype, new):
    _check_attend(pkg, dtype, 2, 2, 64, 16, [new] * 3, [200, 99, 40], q_pad=64, scale=0.3, max_len=5000, width=40)
    _check_attend(pkg, dtype, 2, 2, 64, 16, [new] * 3, [200, 99, 40], lse=False, window=50, sinks=1)
    s = torch.cuda.Stream()
    _check_attend(pkg, dtype, 2, 2, 64, 16, [new] * 3, [200, 99, 4000], stream=s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 3, 40])
@pytest.mark.parametrize("window", [0, 20])
def test_empty_sequences(pkg, dtype, new, window):
    _check_attend(pkg, dtype, 2, 1, 64, 16, [new] * 3, [0, 100, 0], window, 2)
    pool = Pool(pkg, dtype, 2, 64, 16, [30])
    q = torch.zeros((0, 2, 64), dtype=DT[dtype], device="cuda")
    pool.pages.attend(q, _i32(pool.table)[:0], _i32([]), q.clone(), max_len=30)
    out = torch.full((1, 2, 64), 5.0, dtype=DT[dtype], device="cuda")
    pool.pages.attend(torch.zeros_like(out), torch.zeros((1, 0), dtype=torch.int32, device="cuda"), _i32([30]), out, max_len=30)
    assert (out == 0.0).all()  # no page at all: no row


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 40])
def test_rows_of_no_page_read_as_zeros(pkg, dtype, new):
    heads, dim, page, m = 2, 64, 16, 100
    pool = Pool(pkg, dtype, heads, dim, page, [m])
    k, v = _randn(1, m, heads, dim).to(DT[dtype]), _randn(2, m, heads, dim).to(DT[dtype])
    pool.fill(0, k, v)
    for i, e in ((0, -1), (2, pool.pages.n_pages), (3, -2 ** 31), (4, 2 ** 31 - 1)):
        pool.table[0][i] = e
        k[i * page:(i + 1) * page], v[i * page:(i + 1) * page] = 0, 0
    q = _randn(3, new, heads, dim).to(DT[dtype]).cuda()
    out = torch.empty_like(q)
    lse = torch.empty((new, heads), device="cuda")
    kw = {} if new == 1 else {"cu": _i32([0, new]), "max_q": new}
    pool.pages.attend(q, _i32(pool.table), _i32([m]), out, max_len=m, lse=lse, **kw)
    want = ref.attend(q.double().cpu().numpy(), k.double().numpy(), v.double().numpy(), ref.visible(new, m, 0, 0), ref.scale_of(dim), dtype, new > 16)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("new", [1, 5, 40, 200])
def test_arrays_that_hold_anything_stay_in_bounds(pkg, dtype, new):
    """Whatever table, length and cu hold, nothing outside q's and out's rows changes and the call ends."""
    heads, dim, page = 2, 64, 16
    pool = Pool(pkg, dtype, heads, dim, page, [300, 200, 50], fill=1.0)
    q = torch.ones((3 * new, heads, dim), dtype=DT[dtype], device="cuda")
    guard = torch.full((3 * new + 64, heads, dim), 5.0, dtype=DT[dtype], device="cuda")
    out = guard[32:32 + 3 * new]
    r = pkg.H2ORotary(dim)
    for s in range(6):
        g = _gen(s)
        table = torch.randint(-2 ** 31, 2 ** 31 - 1, (3, 19), generator=g, dtype=torch.int64).to(torch.int32)
        if s % 2:
            table %= 40
        length = torch.randint(-2 ** 31, 2 ** 31 - 1, (3,), generator=g, dtype=torch.int64).to(torch.int32)
        cu = torch.randint(-2 ** 31, 2 ** 31 - 1, (4,), generator=g, dtype=torch.int64).to(torch.int32)
        if s >= 3:
            cu = torch.randint(-1, 3 * new + 2, (4,), generator=g).to(torch.int32)
            length = torch.randint(-1, 400, (3,), generator=g).to(torch.int32)
        kw = {"cu": cu.cuda(), "max_q": new} if new > 1 else {}
        pool.pages.attend(q, table.cuda(), length.cuda(), out, max_len=304, window=[0, 7, 100][s % 3], sinks=s, **kw)
        kw.pop("max_q", None)
        pool.pages.append(q.clone(), q.clone(), table.cuda(), length.cuda(), rotary=r, **kw)
        torch.cuda.synchronize()
        assert (guard[:32] == 5.0).all() and (guard[32 + 3 * new:] == 5.0).all()
    assert pool.pages.status() == 0


# ---------------------------------------------------------------------------------------------------------------
# Together, as a decoding loop uses them
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (37, 4)])
def test_prompt_and_captured_steps(pkg, dtype, window, sinks):
    heads, group, dim, page, steps = 2, 2, 64, 16, 9
    prompt = [50, 33, 1]
    final = [n + steps for n in prompt]
    pool = Pool(pkg, dtype, heads, dim, page, final)
    freq, axis = _frequencies(dim), _axis_of(dim // 2, 3)
    r = pkg.H2ORotary(dim, frequencies=freq, axes=axis)
    batch, hq = len(prompt), heads * group
    table, length = _i32(pool.table), _i32(prompt)
    ks, vs, qs = ([_randn(100 * s + b, m, h, dim).to(DT[dtype]) for b, m in enumerate(final)] for s, h in ((1, heads), (2, heads), (3, hq)))
    pos = [torch.stack([torch.arange(m) + 7, torch.arange(m) // 5, torch.arange(m) % 5 + 100]) for m in final]
    cat = lambda xs: torch.cat([x[:n] for x, n in zip(xs, prompt)]).cuda()
    q, k, v = cat(qs), cat(ks), cat(vs)
    p0 = torch.cat([x[:, :n] for x, n in zip(pos, prompt)], 1).contiguous().cuda()
    cu = _i32(_sums(prompt))
    out = torch.empty_like(q)
    pool.pages.append(k, v, table, length, cu=cu, rotary=r, positions=p0, q=q, q_out=q)
    pool.pages.attend(q, table, length, out, max_len=max(final), window=window, sinks=sinks, cu=cu, max_q=max(prompt))
    got = [[out[a:b]] for a, b in zip(_sums(prompt), _sums(prompt)[1:])]
    # one step, captured; what a replay reads is copied into place before it
    q1, o1 = torch.zeros((batch, hq, dim), dtype=DT[dtype], device="cuda"), torch.zeros((batch, hq, dim), dtype=DT[dtype], device="cuda")
    k1, v1 = (torch.zeros((batch, heads, dim), dtype=DT[dtype], device="cuda") for _ in range(2))
    p1 = torch.zeros((3, batch), dtype=torch.int64, device="cuda")
    scratch_table = torch.full_like(table, -1)

    def step(t, o):
        pool.pages.append(k1, v1, t, length, rotary=r, positions=p1, q=q1, q_out=q1)
        pool.pages.attend(q1, t, length, o, max_len=max(final), window=window, sinks=sinks)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(scratch_table, torch.empty_like(o1))  # warm-up on a table without pages
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(table, o1)
    for i in range(steps):
        take = lambda xs: torch.stack([x[n + i] for x, n in zip(xs, prompt)])
        q1.copy_(take(qs)), k1.copy_(take(ks)), v1.copy_(take(vs))
        p1.copy_(torch.stack([x[:, n + i] for x, n in zip(pos, prompt)], 1))
        length += 1
        graph.replay()
        for b in range(batch):
            got[b].append(o1[b:b + 1].clone())
    torch.cuda.synchronize()
    for b, m in enumerate(final):
        turn = lambda x: ref.rotate(x[b].double().numpy(), pos[b].numpy(), freq, axis, True, dtype)[0]
        # rotated values as the cache and the queries hold them
        rounded = [torch.from_numpy(turn(x)).to(DT[dtype]).double().numpy() for x in (qs, ks)]
        want = ref.attend(rounded[0], rounded[1], vs[b].double().numpy(), ref.visible(m, m, window, sinks), ref.scale_of(dim), dtype, True)
        # a value next to a rounding border may be rounded the other way, by a whole step: 2^-7 of one product in 64 for
        # bfloat16, in q or k; allowed for one value in a hundred of them (2^-7 / 100 of the sum of |q k|), twice
        a = np.abs(rounded[0]).max() * np.abs(rounded[1]).sum(-1).max() * ref.scale_of(dim)
        extra = 2 * a * (2.0 ** -7 / 100 if dtype == "bf16" else 2.0 ** -21) * np.abs(vs[b].double().numpy()).max()
        ref.compare(torch.cat(got[b]), want[0], want[2] + extra, "sequence %d" % b)


def test_two_graphs_and_two_streams_share_a_cache(pkg):
    pool = Pool(pkg, "bf16", 2, 64, 16, [4000, 3000])
    for b, m in enumerate(pool.rows):
        pool.fill(b, _randn(b, m, 2, 64), _randn(b + 7, m, 2, 64))
    table, length = _i32(pool.table), _i32(pool.rows)
    q = [_randn(s, 2, 2, 64).to(torch.bfloat16).cuda() for s in (1, 2)]
    alone = [torch.empty_like(x) for x in q]
    for x, o in zip(q, alone):
        pool.pages.attend(x, table, length, o, max_len=4000)
    torch.cuda.synchronize()
    graphs, outs = [], [torch.empty_like(x) for x in q]
    for x, o in zip(q, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            pool.pages.attend(x, table, length, o, max_len=4000)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in q]
    for s, g in zip(streams, graphs):
        with torch.cuda.stream(s):
            g.replay()
            g.replay()
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    for x, o, s in zip(q, outs, streams):
        pool.pages.attend(x, table, length, o, max_len=4000, stream=s)
    torch.cuda.synchronize()
    for a, b in zip(alone, outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("new,rows", [([300, 40], [700, 40]), ([20, 0], [900, 5])])
def test_captured_prompts_follow_the_arrays(pkg, new, rows):
    """A captured prompt, replayed with other lengths, token counts and tables: the results of calls of their own."""
    heads, dim, page = 2, 128, 16
    pool = Pool(pkg, "bf16", heads, dim, page, [1000, 1000])
    for b in range(2):
        pool.fill(b, _randn(b, 1000, heads, dim), _randn(b + 7, 1000, heads, dim))
    q = _randn(3, 400, heads, dim).to(torch.bfloat16).cuda()
    table, length, cu = _i32(pool.table), _i32(rows), _i32(_sums(new))
    out, want = torch.full_like(q, 5.0), torch.full_like(q, 5.0)
    args = dict(max_len=1000, window=333, sinks=3, max_q=300)
    pool.pages.attend(q, table, length, out, cu=cu, **args)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        pool.pages.attend(q, table, length, out, cu=cu, **args)
    for new2, rows2, swap in ((new, rows, False), (new[::-1], rows[::-1], True), ([1, 1], [1000, 999], False), ([0, 300], [0, 300], True), ([0, 0], [9, 9], False)):
        table.copy_(_i32(pool.table[::-1] if swap else pool.table)), length.copy_(_i32(rows2)), cu.copy_(_i32(_sums(new2)))
        out.fill_(5.0), want.fill_(5.0)
        pool.pages.attend(q, table, length, want, cu=cu, **args)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert (out[sum(new2):] == 5.0).all()
    assert pool.pages.status() == 0


def test_many_places_without_work(pkg):
    """Thousands of sequences with one token beside one with 2000: almost no tile of query rows exists."""
    batch, heads, dim, page, n = 3000, 2, 64, 16, 2000
    g = torch.Generator(device="cuda").manual_seed(3)
    pages = batch - 1 + n // page
    k, v = (torch.randn((pages, page, heads, dim), generator=g, device="cuda").bfloat16() for _ in range(2))
    table = torch.full((batch, n // page), -1, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(batch, dtype=torch.int32, device="cuda")
    table[1234] = torch.cat([table[1234, :1], torch.arange(batch, pages + 0, dtype=torch.int32, device="cuda"), torch.full((n // page,), 7, dtype=torch.int32, device="cuda")])[:n // page]
    new = torch.ones(batch, dtype=torch.int64)
    new[1234] = n
    length = new.int().cuda()
    length[:1234] = 9
    cu = torch.cat([torch.zeros(1, dtype=torch.int64), new.cumsum(0)]).int().cuda()
    tokens = int(new.sum())
    q = torch.randn((tokens, heads, dim), generator=g, device="cuda").bfloat16()
    out = torch.full_like(q, 5.0)
    h = pkg.H2OPages(k, v)
    h.attend(q, table, length, out, max_len=n, cu=cu, max_q=n)
    torch.cuda.synchronize()
    assert h.status() == 0
    at = int(cu[1234])
    for b, first, count, m in ((5, 5, 1, 9), (1234, at, n, n), (2500, 2500 + n - 1, 1, 1)):
        rows = [x[table[b].clamp(min=0).long()].flatten(0, 1)[:m].double().cpu().numpy() for x in (k, v)]
        want = ref.attend(q[first:first + count].double().cpu().numpy(), *rows, ref.visible(count, m, 0, 0), ref.scale_of(dim), "bf16", True)
        ref.compare(out[first:first + count], want[0], want[2], "sequence %d" % b)

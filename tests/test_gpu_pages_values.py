"""Values at which attention over a paged cache can go wrong, and sizes beyond the ordinary, on a B200."""
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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _one(pkg, dtype, k, v, q, page=16, window=0, sinks=0, scale=0.0, max_len=None, max_q=None):
    """One sequence of k, v [rows, heads, dim] on shuffled pages; its last q tokens' results."""
    rows, heads, dim = k.shape
    n = (rows + page - 1) // page
    order = torch.randperm(n, generator=torch.Generator().manual_seed(rows)).cuda()
    pools = []
    for x in (k, v):
        whole = torch.full((n * page, heads, dim), math.nan, dtype=DT[dtype], device="cuda")
        whole[:rows] = x.to(DT[dtype])
        pool = torch.empty((n, page, heads, dim), dtype=DT[dtype], device="cuda")
        pool[order] = whole.view(n, page, heads, dim)
        pools.append(pool)
    pages = pkg.H2OPages(*pools)
    q = q.to(DT[dtype]).cuda()
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], dtype=torch.float32, device="cuda")
    pages.attend(q, order.int().view(1, n), _i32([rows]), out, max_len=max_len or rows, window=window, sinks=sinks, cu=_i32([0, q.shape[0]]),
                 max_q=max_q or q.shape[0], lse=lse, softmax_scale=scale)
    torch.cuda.synchronize()
    assert pages.status() == 0
    return out, lse


def _randn(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 9, 40, 300])
@pytest.mark.parametrize("window,sinks", [(0, 0), (400, 4)])
@pytest.mark.parametrize("direction", [1, -1])
def test_logits_that_keep_growing_or_falling(pkg, dtype, n, window, sinks, direction):
    """Each tile's logits lie far above (below) the one's before: the reference maximum has to follow (stay)."""
    rows, heads, dim = 1300, 2, 64
    q, k, v = _randn(1, n, heads, dim), _randn(2, rows, heads, dim) * 0.2, _randn(3, rows, heads, dim)
    level = torch.arange(rows)[:, None] / rows * 60 * direction  # 60 in exponents over the length
    unit = torch.ones(dim) / 8
    q = (q * 0.3 + 4 * unit).to(DT[dtype])
    k = (k + level[..., None] * unit * 2).to(DT[dtype])
    v = v.to(DT[dtype])
    out, lse = _one(pkg, dtype, k, v, q, window=window, sinks=sinks)
    want = ref.attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), ref.visible(n, rows, window, sinks), ref.scale_of(dim), dtype, n > 16)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
def test_sinks_that_take_everything(pkg, dtype, n):
    """The first rows' logits lie 80 above all others: later tiles add nothing, and nothing underflows into NaN."""
    rows, heads, dim = 900, 1, 128
    q, k, v = torch.ones(n, heads, dim), _randn(2, rows, heads, dim) * 0.01, _randn(3, rows, heads, dim)
    k[:4] += 80 / math.sqrt(dim)
    q, k, v = (x.to(DT[dtype]) for x in (q, k, v))
    for window, sinks in ((0, 0), (200, 4), (200, 0)):
        out, lse = _one(pkg, dtype, k, v, q, window=window, sinks=sinks)
        want = ref.attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), ref.visible(n, rows, window, sinks), ref.scale_of(dim), dtype, n > 16)
        ref.compare(out, want[0], want[2], "out")
        ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 8, 40])
def test_infinite_and_nan_rows(pkg, dtype, n):
    """-infinity in a key: its weight is 0.  All of them: no row counts.  NaN in a visible key or value: NaN.  Infinity in a value
    that all the tokens see: infinity."""
    rows, heads, dim = 200, 2, 64
    base = [x.to(DT[dtype]) for x in (_randn(1, n, heads, dim), _randn(2, rows, heads, dim), _randn(3, rows, heads, dim))]
    q = base[0].clone()
    q[..., 0] = 1.0
    k, v = base[1].clone(), base[2].clone()
    k[5, :, 0] = k[100, :, 0] = -math.inf
    out, lse = _one(pkg, dtype, k, v, q)
    kk = k.double().numpy().copy()
    kk[5], kk[100] = 0.0, 0.0
    seen = ref.visible(n, rows, 0, 0)
    seen[:, [5, 100]] = False
    want = ref.attend(q.double().numpy(), kk, v.double().numpy(), seen, ref.scale_of(dim), dtype, n > 16)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")
    k[:, 1, 0] = -math.inf
    out, lse = _one(pkg, dtype, k, v, q)
    assert (out[:, 1] == 0).all() and (lse[:, 1] == -math.inf).all() and torch.isfinite(out[:, 0].float()).all()
    k, v = base[1].clone(), base[2].clone()
    v[3, 0, 7] = math.inf
    v[4, 1, 9] = math.nan
    out, lse = _one(pkg, dtype, k, v, q)
    assert (out[:, 0, 7] == math.inf).all() and torch.isnan(out[:, 1, 9].float()).all() and torch.isfinite(lse).all()
    bad = ~torch.isfinite(out.float())
    assert bad.sum() == 2 * n
    k[3, 0, 2] = math.nan
    out, lse = _one(pkg, dtype, k, base[2], q)
    assert torch.isnan(out[:, 0].float()).all() and torch.isnan(lse[:, 0]).all()
    assert torch.isfinite(out[:, 1].float()).all() and torch.isfinite(lse[:, 1]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
@pytest.mark.parametrize("scale", [1e-30, 1e-3, 30.0, 2e38])
def test_softmax_scales(pkg, dtype, n, scale):
    rows, heads, dim = 130, 1, 64
    tiny = 1e-19 if scale == 2e38 else 1.0  # (products of 1e-38 times the scale: logits about 1)
    q, k, v = (_randn(1, n, heads, dim) * tiny).to(DT[dtype]), (_randn(2, rows, heads, dim) * tiny).to(DT[dtype]), _randn(3, rows, heads, dim).to(DT[dtype])
    out, lse = _one(pkg, dtype, k, v, q, scale=scale)
    want = ref.attend(q.double().numpy(), k.double().numpy(), v.double().numpy(), ref.visible(n, rows, 0, 0), float(np.float32(scale)), dtype, n > 16)
    tol = want[2]
    if scale == 2e38:
        # fp32 products of 1e-38 and below lose bits below 2^-149 (flushed below 2^-126): d of them, times the scale, twice
        tol = tol + 2 * dim * 2.0 ** -126 * 2e38 * np.abs(v.double().numpy()).max()
        ref.compare(lse, want[1], want[3] + dim * 2.0 ** -126 * 2e38, "lse")
    else:
        ref.compare(lse, want[1], want[3], "lse")
    ref.compare(out, want[0], tol, "out")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 40])
def test_upper_bounds_cut(pkg, dtype, n):
    """A length beyond max_len counts as max_len."""
    rows, heads, dim, cut = 300, 2, 64, 170
    q, k, v = (_randn(s, m, heads, dim).to(DT[dtype]) for s, m in ((1, n), (2, rows), (3, rows)))
    out, lse = _one(pkg, dtype, k, v, q, max_len=cut, window=100, sinks=3)
    want = ref.attend(q.double().numpy(), k[:cut].double().numpy(), v[:cut].double().numpy(), ref.visible(n, cut, 100, 3), ref.scale_of(dim), dtype, n > 16)
    ref.compare(out, want[0], want[2], "out")
    ref.compare(lse, want[1], want[3], "lse")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_offsets_past_32_bits(pkg, dtype):
    """A pool of more than 2^32 elements: its last pages are appended to and attended."""
    heads, dim, page = 8, 128, 16
    pages = 2 ** 32 // (page * heads * dim) + 40
    k, v = (torch.empty((pages, page, heads, dim), dtype=DT[dtype], device="cuda") for _ in range(2))
    h = pkg.H2OPages(k, v)
    rows = 300
    table = torch.arange(pages - 19, pages, dtype=torch.int32, device="cuda").flip(0).contiguous().view(1, 19)
    kk, vv, q = (_randn(s, rows, heads, dim).to(DT[dtype]).cuda() for s in (1, 2, 3))
    cu = _i32([0, rows])
    h.append(kk, vv, table, _i32([rows]), cu=cu)
    for x, y in ((k, kk), (v, vv)):
        assert torch.equal(x[table[0].long()].flatten(0, 1)[:rows], y)
    for n in (1, 100):
        qq = q[:n].contiguous()
        out = torch.empty_like(qq)
        h.attend(qq, table, _i32([rows]), out, max_len=rows, cu=_i32([0, n]), max_q=n)
        want = ref.attend(qq.double().cpu().numpy(), kk.double().cpu().numpy(), vv.double().cpu().numpy(), ref.visible(n, rows, 0, 0), ref.scale_of(dim),
                          dtype, n > 16)
        ref.compare(out, want[0], want[2], "out of %d" % n)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,window,sinks", [(1, 0, 0), (30, 0, 0), (30, 100000, 1000)])
def test_a_sequence_of_200000_rows(pkg, dtype, n, window, sinks):
    rows, heads, dim = 200003, 1, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((rows, heads, dim), generator=g, device="cuda").to(DT[dtype]) for _ in range(2))
    q = (torch.randn((n, heads, dim), generator=g, device="cuda") * 2).to(DT[dtype])
    out, lse = _one(pkg, dtype, k, v, q, window=window, sinks=sinks)
    seen = torch.from_numpy(ref.visible(n, rows, window, sinks)).cuda()
    x = (q[:, 0].double() @ k[:, 0].double().T / 8).masked_fill(~seen, -math.inf)
    want_lse, p = x.logsumexp(-1), x.softmax(-1)
    want = p @ v[:, 0].double()
    # as in pages_reference.attend: rounding of the type, of P, fp32 sums over the rows (in chunks), logits
    a = p @ v[:, 0].double().abs()
    ds = (dim + 4) * 2.0 ** -23 * (q[:, 0].double().abs() @ k[:, 0].double().abs().T / 8).max() + x[seen].abs().max() * 2.0 ** -22
    p_err = 0.0 if dtype == "f32" else 2.0 ** -8 if n > 16 else 2.0 ** -15
    tol = ref.EPS2[dtype] * want.abs() + (p_err + 2 * ds + 2 * rows * 2.0 ** -24 + 2.0 ** -20) * a
    assert ((out[:, 0].double() - want).abs() <= tol).all()
    assert ((lse[:, 0].double() - want_lse).abs() <= ds + rows * 2.0 ** -24 + 2.0 ** -20 + 2.0 ** -23 * want_lse.abs()).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_thousands_of_short_sequences(pkg, dtype):
    batch, heads, dim, page = 3001, 1, 64, 8
    g = torch.Generator(device="cuda").manual_seed(6)
    length = torch.randint(0, 17, (batch,), generator=g, device="cuda", dtype=torch.int32)
    table = torch.randperm(2 * batch, generator=g, device="cuda").int().view(batch, 2).contiguous()
    k, v = (torch.zeros((2 * batch, page, heads, dim), dtype=DT[dtype], device="cuda") for _ in range(2))
    h = pkg.H2OPages(k, v)
    rows = torch.randn((2, batch, 16, heads, dim), generator=g, device="cuda").to(DT[dtype])
    for i in range(16):  # one token after the other; a sequence that has enough rows keeps still (its token has no page)
        here = torch.where((length > i)[:, None], table, -1)
        h.append(rows[0, :, i].contiguous(), rows[1, :, i].contiguous(), here, torch.full_like(length, i + 1))
    q = torch.randn((batch, heads, dim), generator=g, device="cuda").to(DT[dtype])
    out = torch.full_like(q, 5.0)
    h.attend(q, table, length, out, max_len=16)
    x = torch.einsum("bhd,brhd->bhr", q.double(), rows[0].double()) / 8
    x = x.masked_fill((torch.arange(16, device="cuda") >= length[:, None])[:, None], -math.inf)
    p = torch.where(length[:, None, None] > 0, x.softmax(-1), 0.0)
    want = torch.einsum("bhr,brhd->bhd", p.nan_to_num(0.0), rows[1].double())
    # 16 rows: the type's rounding of values below 5, and 2^-15 (2^-20) of sums of p |v| below 5
    assert ((out.double() - want).abs() <= ref.EPS2[dtype] * want.abs() + 5 * (2.0 ** -14 if dtype == "bf16" else 2.0 ** -18)).all()
    assert (out[length == 0] == 0).all()

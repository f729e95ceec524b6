"""How exact the K/V store's attention is on each of its paths (needs a B200): the general tests allow every path the roundings of
the coarsest one; these allow each its own.

  up to 16 bfloat16 rows   P = bf16 hi + bf16 lo: 2^-15 of a probability
  more bfloat16 rows       P = one bf16: 2^-8
  float32 queries          P, queries and values in fp32, on 8-bit rows too
"""
import math

import numpy as np
import pytest
import torch

import store_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


def _bf16(x):
    return torch.from_numpy(np.asarray(x)).bfloat16().double().numpy()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,length", [(1, 8), (8, 8), (16, 8), (17, 8), (150, 8), (1, 3000), (16, 3000), (17, 3000)])
def test_probabilities_of_few_rows_keep_what_one_bf16_would_lose(pkg, dim, n, length):
    """Few keys that weigh (the others' logits are -200) and values that cancel, so that the output's own rounding is small.

    Queries are unit vectors and the scale is 1: logits are exact.  Tolerance: half a step of the output, 2^-15 (one bf16: 2^-8)
    of a = sum p |v| for P, 2^-20 for exp2 and its argument (of 8 at most), 2^-21 for fp32 sums of so few terms.  That the first bound
    tells the two apart is shown on the CPU: with P in one bf16 it is broken."""
    g = np.random.default_rng(dim + n + length)
    batch, keys = 24, 4
    k = np.zeros((batch, length, dim))
    v = np.zeros((batch, length, dim))
    k[:, :, 0] = -200.0
    want, a, coarse = (np.zeros((batch, dim)) for _ in range(3))
    for b in range(batch):
        at = int(g.integers(0, length - keys + 1))
        x = _bf16(g.uniform(-2.5, 2.5, keys))
        e = np.exp(x - x.max())
        p = e / e.sum()
        vv = _bf16(g.normal(size=(keys, dim)))
        vv[0] = _bf16(-(p[1:] @ vv[1:]) / p[0])
        k[b, at:at + keys, 0], v[b, at:at + keys] = x, vv
        want[b], a[b], coarse[b] = p @ vv, p @ np.abs(vv), _bf16(e.astype(np.float32)) @ vv / e.sum()
    tol = lambda p_err: 2.0 ** -8 * np.abs(want) + (p_err + 2.0 ** -20 + 2.0 ** -21) * a + 1e-30
    fine, one = tol(2.0 ** -15), tol(2.0 ** -8)
    assert (np.abs(coarse - want) > fine).mean() > 0.5 and (np.abs(coarse - want) <= one).all()
    rows = lambda t: torch.from_numpy(t.reshape(batch * length, 1, dim)).bfloat16().cuda()
    store = pkg.H2OStore(rows(k), rows(v))
    q = torch.zeros((batch * n, 1, dim), dtype=torch.bfloat16, device="cuda")
    q[:, 0, 0] = 1.0
    out = torch.empty_like(q)
    kw = {} if n == 1 else {"cu_q": torch.arange(0, batch * n + 1, n, dtype=torch.int32, device="cuda"), "max_q": n}
    store.cross_attend(q, torch.arange(0, batch * length, length, device="cuda"),
                       torch.full((batch,), length, dtype=torch.int32, device="cuda"), out, max_len=length, softmax_scale=1.0, **kw)
    assert store.status() == 0
    err = np.abs(out.view(batch, n, dim).double().cpu().numpy() - want[:, None])
    assert (err <= (fine if n <= 16 else one)[:, None]).all(), (err / a[:, None]).max()


@pytest.mark.parametrize("fmt", ["kv8", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n,group,length", [(1, 1, 30), (1, 4, 60), (3, 1, 50), (3, 1, 2100), (1, 12, 40), (20, 1, 33), (70, 2, 64), (70, 2, 700)])
def test_float32_queries_lose_nothing_to_16_bits(pkg, fmt, dim, n, group, length):
    """8-bit rows too: their values are exact in fp32, and so are queries and probabilities.  The tolerance is that of float32
    rows; on the CPU, f16 probabilities break it where the keys are few (the bound of the fp32 sums grows with them)."""
    g = torch.Generator().manual_seed(n + group + length)
    k, v = (torch.randn((2 * length, 1, dim), generator=g) for _ in range(2))
    if fmt == "kv8":
        (ck, sk), (cv, sv) = ref.quantise(k), ref.quantise(v)
        store = pkg.H2OStore(*[torch.from_numpy(x).cuda() for x in (ck, cv, sk, sv)])
        k64, v64 = ref.values(ck, sk).transpose(1, 0, 2), ref.values(cv, sv).transpose(1, 0, 2)
    else:
        store, k64, v64 = pkg.H2OStore(k.cuda(), v.cuda()), k.double().numpy(), v.double().numpy()
    q = (torch.randn((2 * n, group, dim), generator=g) * 0.1).cuda()
    out, lse = torch.empty_like(q), torch.empty((2 * n, group), dtype=torch.float32, device="cuda")
    kw = {} if n == 1 else {"cu_q": torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda"), "max_q": n}
    store.cross_attend(q, torch.tensor([0, length], device="cuda"), torch.tensor([length, length - 5], dtype=torch.int32, device="cuda"), out,
                       max_len=length, lse=lse, **kw)
    assert store.status() == 0
    scale = float(np.float32(1 / math.sqrt(dim)))
    for b, m in enumerate((length, length - 5)):
        sl, at = slice(b * n, b * n + n), slice(b * length, b * length + m)
        qq = q[sl].double().cpu().numpy()
        want, wl, tol, ltol = ref.attend(qq, k64[at], v64[at], [m] * n, scale, "f32", "f32")
        p = np.exp(scale * (qq[0, 0] @ k64[at, 0].T))
        p /= p.max()
        coarse = (p.astype(np.float16).astype(np.float64) @ v64[at, 0]) / p.sum()
        assert length > 100 or (np.abs(coarse - want[0, 0]) > tol[0, 0]).any()
        ref.compare(out[sl], want, tol, "out of sequence %d" % b)
        ref.compare(lse[sl], wl, ltol, "lse of sequence %d" % b)

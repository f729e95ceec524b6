"""Device arrays that the host never sees, holding anything: the K/V store's attention stays inside its arrays (needs a B200).

Around out, lse and the scratch lie guards; the scratch starts as NaN, so a chunk that is read and was never written shows
in the outputs.  tests/store_bounds_cases.py runs this file on the checked build as well, where every index is verified."""
import math
import random

import numpy as np
import pytest
import torch

import store_reference as ref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
FORMATS = [("f32", "f32"), ("bf16", "bf16"), ("kv8", "bf16"), ("kv8", "f32")]
GUARD = 64  # rows
# (query tokens of the sequences, their own rows, sequences of the groups, their prefixes): few rows and keys in one launch;
# few rows in chunks; many rows of a group and few of a sequence; many of both, the prefix in one piece and in several
SHAPES = [
    ([2, 4, 0, 3], [2, 70, 9, 33], [2, 2], [33, 440]),
    ([1, 3, 2, 4], [1, 64, 2, 300], [2, 2], [2100, 31]),
    ([1] * 40, list(range(40)), [25, 15], [1500, 700]),
    ([40, 17, 64, 33], [40, 20, 200, 33], [3, 1], [96, 65]),
    ([60, 130, 33], [200, 130, 40], [3], [5000]),
]


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


class Case:
    """Tensors of a call, with guards; `run` gives out and lse."""

    def __init__(self, pkg, fmt, q_dtype, dim, shape, heads=2):
        self.q_len, own, self.members, pre = shape
        self.fmt, self.q_dtype, self.dim = fmt, q_dtype, dim
        lengths = pre + own
        self.begin = [sum(lengths[:i]) + 3 * i for i in range(len(lengths))]
        self.rows = sum(lengths) + 3 * len(lengths)
        g = torch.Generator().manual_seed(len(own) + dim)
        k, v = (torch.randn((self.rows, heads, dim), generator=g).to(DT.get(fmt, torch.bfloat16)) for _ in range(2))
        if fmt == "kv8":
            (ck, sk), (cv, sv) = ref.quantise(k), ref.quantise(v)
            self.store = pkg.H2OStore(*[torch.from_numpy(x).cuda() for x in (ck, cv, sk, sv)])
            self.k64, self.v64 = (ref.values(*x).transpose(1, 0, 2) for x in ((ck, sk), (cv, sv)))
        else:
            self.store = pkg.H2OStore(k.cuda(), v.cuda())
            self.k64, self.v64 = k.double().numpy(), v.double().numpy()
        self.tokens = sum(self.q_len)
        self.q = torch.randn((self.tokens, heads, dim), generator=g).to(DT[q_dtype]).cuda()
        self.arena = torch.empty((self.tokens + 2 * GUARD, heads, dim), dtype=self.q.dtype, device="cuda")
        self.lse_arena = torch.empty((self.tokens + 2 * GUARD, heads), dtype=torch.float32, device="cuda")
        self.out, self.lse = self.arena[GUARD:-GUARD], self.lse_arena[GUARD:-GUARD]
        self.scratch = None

        def scratch(nbytes, stream):
            if self.scratch is None or self.scratch.numel() != nbytes + 2 * 65536:
                self.scratch = torch.empty(nbytes + 2 * 65536, dtype=torch.uint8, device="cuda")
            self.scratch.fill_(0xFF)
            return self.scratch[65536:65536 + nbytes]

        self.store._scratch = scratch
        sums = lambda x: np.concatenate([[0], np.cumsum(x)]).tolist()
        n = len(pre)
        self.arrays = dict(cu_q=sums(self.q_len), cu_group=sums(self.members), prefix_begin=self.begin[:n], prefix_len=list(pre),
                           own_begin=self.begin[n:], own_len=list(own))
        self.most = dict(max_prefix=max(pre), max_own=max(own))

    def run(self, cross, **changed):
        a = {k: torch.tensor(changed.get(k, v), dtype=torch.int64 if k.endswith("begin") else torch.int32, device="cuda")
             for k, v in self.arrays.items()}
        self.arena.fill_(5.0), self.lse_arena.fill_(5.0)
        if cross:
            self.store.cross_attend(self.q, a["own_begin"], a["own_len"], self.out, max_len=self.most["max_own"], lse=self.lse, cu_q=a["cu_q"],
                                    max_q=max(self.q_len))
        else:
            self.store.prefix_attend(self.q, a["prefix_begin"], a["prefix_len"], a["own_begin"], a["own_len"], self.out, lse=self.lse,
                                     cu_q=a["cu_q"], max_q=max(self.q_len), cu_group=a["cu_group"], max_group=max(self.members), **self.most)
        torch.cuda.synchronize()
        assert self.store.status() == 0
        for x in (self.arena, self.lse_arena):
            assert (x[:GUARD] == 5.0).all() and (x[-GUARD:] == 5.0).all()
        if self.scratch is not None:
            assert (self.scratch[:65536] == 0xFF).all() and (self.scratch[-65536:] == 0xFF).all()
        assert not torch.isnan(self.out).any() and not torch.isnan(self.lse).any()
        return self.out.clone(), self.lse.clone()

    def cut(self, begin, length, most):
        begin = max(0, min(begin, self.rows))
        return begin, max(0, min(length, most, self.rows - begin))

    def check(self, cross, out, lse, prefix_begin, prefix_len, own_begin, own_len):
        cu, which = self.arrays["cu_q"], np.repeat(np.arange(len(self.members)), self.members)
        for b, n in enumerate(self.q_len):
            o, m = self.cut(own_begin[b], own_len[b], self.most["max_own"])
            kk, vv, seen = self.k64[o:o + m], self.v64[o:o + m], [m] * n
            if not cross:
                p, r = self.cut(prefix_begin[which[b]], prefix_len[which[b]], self.most["max_prefix"])
                kk, vv = (np.concatenate([x[p:p + r], y]) for x, y in ((self.k64, kk), (self.v64, vv)))
                seen = [r + max(0, m - (n - 1 - i)) for i in range(n)]
            sl = slice(cu[b], cu[b] + n)
            want = ref.attend(self.q[sl].double().cpu().numpy(), kk, vv, seen, float(np.float32(1 / math.sqrt(self.dim))), self.fmt, self.q_dtype)
            ref.compare(out[sl], want[0], want[2], "out of sequence %d" % b)
            ref.compare(lse[sl], want[1], want[3], "lse of sequence %d" % b)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("cross", [True, False])
def test_ranges_that_point_anywhere_are_cut(pkg, fmt, q_dtype, dim, shape, cross):
    c = Case(pkg, fmt, q_dtype, dim, SHAPES[shape])
    r = random.Random(shape)
    begins = [-1, -2 ** 62, -2 ** 63, 2 ** 62, 2 ** 63 - 1, 2 ** 31, -2 ** 31, 2 ** 32 + 5, c.rows, c.rows - 1, c.rows - 17, c.rows + 1, 0, 7]
    lengths = [-1, -2 ** 31, 2 ** 31 - 1, 0, 1, c.rows, c.rows + 1, 77]
    good = c.run(cross)
    for _ in range(3):
        a = {k: [r.choice(begins if k.endswith("begin") else lengths) if r.random() < 0.5 else x for x in v]
             for k, v in c.arrays.items() if k.startswith(("prefix", "own"))}
        c.check(cross, *c.run(cross, **a), **a)
    for x, y in zip(good, c.run(cross)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("fmt,q_dtype", FORMATS)
@pytest.mark.parametrize("shape", range(len(SHAPES)))
@pytest.mark.parametrize("cross", [True, False])
def test_offsets_of_sequences_and_groups_that_hold_anything(pkg, fmt, q_dtype, shape, cross):
    """Negative, decreasing, oversized and equal cu_q and cu_group, with ranges of both kinds: nothing outside is touched and no
    chunk that nobody has written is joined.  Then the same call with proper ones gives the same bits as before."""
    c = Case(pkg, fmt, q_dtype, 128, SHAPES[shape])
    r = random.Random(shape + 50)
    good = c.run(cross)
    many = lambda limit: [-1, -2 ** 31, 2 ** 31 - 1, 0, 1, limit, limit + 1, limit - 1, limit // 2]
    for i in range(24):
        odds = (0.2, 0.6, 1.0)[i % 3]
        a = {"cu_q": [r.choice(many(c.tokens)) if r.random() < odds else x for x in c.arrays["cu_q"]],
             "cu_group": [r.choice(many(len(c.q_len))) if r.random() < odds else x for x in c.arrays["cu_group"]]}
        if i % 2:
            a["own_begin"] = [r.randrange(-50, c.rows + 50) for _ in c.arrays["own_begin"]]
            a["own_len"] = [r.randrange(-5, 300) for _ in c.arrays["own_len"]]
        if i == 5:
            a["cu_q"] = a["cu_q"][::-1]
        if i == 7:
            a["cu_group"] = c.arrays["cu_group"][::-1]
        c.run(cross, **a)
    for x, y in zip(good, c.run(cross)):
        assert torch.equal(x, y)

"""Bounded waits of the K/V store's attention kernels that give up: a status code, not the context (needs a B200).

h2o_debug_store_set_polls makes the waits of a store give up after a few polls, or at once.  Everything they wait for does
arrive, so nothing hangs: the kernels wind down while copies and products are under way, as after a real time-out, and the
same call with the ordinary limit gives the same bits as before."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


def _store(pkg, fmt, rows, heads, dim):
    g = torch.Generator().manual_seed(rows)
    k, v = (torch.randn((rows, heads, dim), generator=g).bfloat16().cuda() for _ in range(2))
    if fmt == "bf16":
        return pkg.H2OStore(k, v)
    store = pkg.H2OStore.empty_kv8(rows, heads, dim)
    store.write(k, v)
    return store


def _i64(x):
    return torch.tensor(x, dtype=torch.int64, device="cuda")


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _try_all(pkg, store, q, call):
    """`call(out, lse)` with the ordinary limit, then with short ones, then with the ordinary one again."""
    def run():
        store._status.zero_()
        out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, dtype=torch.float32, device="cuda")
        call(out, lse)
        torch.cuda.synchronize()
        return store.status(), out, lse

    code, out, lse = run()
    assert code == 0
    seen = []
    for polls in (0, 0, 1, 2, 3, 5, 10, 30, 100, 300, 1000):
        assert pkg.lib.h2o_debug_store_set_polls(store._h, polls) == 0
        code, o, s = run()
        assert code in (0, pkg.H2O_ERR_TIMEOUT)
        if code == 0:
            assert torch.equal(o, out) and torch.equal(s, lse)
        seen.append(code)
    assert seen[0] == seen[1] == pkg.H2O_ERR_TIMEOUT
    assert pkg.lib.h2o_debug_store_set_polls(store._h, -1) == 0
    code, o, s = run()
    assert code == 0 and torch.equal(o, out) and torch.equal(s, lse)


@pytest.mark.parametrize("fmt", ["bf16", "kv8"])
@pytest.mark.parametrize("dim", [64, 128])
# few rows in blocks of 8, 16 and (8-bit) 32; many in one group, in turn, in two groups; keys in one piece and in several
@pytest.mark.parametrize("n,length", [(1, 40), (1, 5000), (12, 700), (30, 700), (30, 5000), (100, 300), (100, 2000), (200, 300), (300, 3000)])
def test_cross_waits_that_give_up(pkg, fmt, dim, n, length):
    store = _store(pkg, fmt, 2 * length, 2, dim)
    q = torch.randn((2 * n, 2, dim), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    kw = dict(cu_q=_i32([0, n, 2 * n]), max_q=n)
    _try_all(pkg, store, q, lambda out, lse: store.cross_attend(q, _i64([0, length]), _i32([length, length - 7]), out, max_len=length,
                                                               lse=lse, **kw))


@pytest.mark.parametrize("fmt", ["bf16", "kv8"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("batch,n,prefix", [(3, 1, 100), (3, 1, 3000), (40, 1, 3000), (5, 20, 90), (5, 40, 3000), (3, 150, 6000)])
def test_prefix_waits_that_give_up(pkg, fmt, dim, batch, n, prefix):
    own = n + 30
    store = _store(pkg, fmt, prefix + batch * own, 2, dim)
    q = torch.randn((batch * n, 2, dim), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    begin = [prefix + own * b for b in range(batch)]
    kw = dict(cu_q=_i32([n * b for b in range(batch + 1)]), max_q=n)
    _try_all(pkg, store, q, lambda out, lse: store.prefix_attend(q, _i64([0]), _i32([prefix]), _i64(begin), _i32([own] * batch), out,
                                                                max_prefix=prefix, max_own=own, lse=lse, **kw))

"""Bounded waits of the paged cache's attention kernels that give up: a status code, not the context (needs a B200).

h2o_debug_pages_set_polls makes the waits give up after a few polls, or at once.  Everything they wait for does arrive, so
nothing hangs: the kernels wind down while copies and products are under way, as after a real time-out, and the same call with
the ordinary limit gives the same bits as before."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("page", [16, 64])
# few rows in blocks of 8 and 16; prompts of one tile and of several; keys in one piece and in several; a window with sinks
@pytest.mark.parametrize("n,length,window", [(1, 40, 0), (1, 5000, 0), (12, 700, 0), (30, 700, 0), (30, 5000, 0), (100, 300, 0), (300, 3000, 0),
                                             (1, 3000, 500), (300, 3000, 500)])
def test_waits_that_give_up(pkg, dim, page, n, length, window):
    g = torch.Generator().manual_seed(length)
    per = (length + page - 1) // page
    k, v = (torch.randn((2 * per, page, 2, dim), generator=g).bfloat16().cuda() for _ in range(2))
    pages = pkg.H2OPages(k, v)
    table = torch.randperm(2 * per, generator=g).int().view(2, per).cuda()
    rows = torch.tensor([length, length - 7], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, n, 2 * n], dtype=torch.int32, device="cuda")
    q = torch.randn((2 * n, 2, dim), generator=g).bfloat16().cuda()

    def run():
        pages._status.zero_()
        out, lse = torch.full_like(q, 5.0), torch.full(q.shape[:2], 5.0, dtype=torch.float32, device="cuda")
        pages.attend(q, table, rows, out, max_len=length, window=window, sinks=4, cu=cu, max_q=n, lse=lse)
        torch.cuda.synchronize()
        return pages.status(), out, lse

    code, out, lse = run()
    assert code == 0
    seen = []
    for polls in (0, 0, 1, 2, 3, 5, 10, 30, 100, 300, 1000):
        assert pkg.lib.h2o_debug_pages_set_polls(pages._h, polls) == 0
        code, o, s = run()
        assert code in (0, pkg.H2O_ERR_TIMEOUT)
        if code == 0:
            assert torch.equal(o, out) and torch.equal(s, lse)
        seen.append(code)
    assert seen[0] == seen[1] == pkg.H2O_ERR_TIMEOUT
    assert pkg.lib.h2o_debug_pages_set_polls(pages._h, -1) == 0
    code, o, s = run()
    assert code == 0 and torch.equal(o, out) and torch.equal(s, lse)

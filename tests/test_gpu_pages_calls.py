"""Calls of H2ORotary and H2OPages beside the ordinary ones: refusals that need a device, objects that go away, streams."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def pkg():
    import paper_2306_14048_b200 as p

    assert torch.cuda.is_available(), "these tests need a CUDA device; there is no CPU fallback"
    return p


@pytest.mark.parametrize("shape", [(50, 16, 2, 128), (1, 16, 2, 128)])
def test_a_broadcast_pool_is_refused(pkg, shape):
    x = torch.zeros(128, dtype=torch.bfloat16, device="cuda").expand(shape)
    with pytest.raises(ValueError):
        pkg.H2OPages(x, x)


def _waiting(stream):
    """Something that keeps `stream` busy for some milliseconds."""
    with torch.cuda.stream(stream):
        torch.cuda._sleep(20_000_000)


def _taken(n):
    """Small pieces of memory of the current stream, full of other numbers: what has just been given back is among them."""
    return [torch.full((n,), 1e30, dtype=torch.float64, device="cuda") for _ in range(64)]


@pytest.mark.parametrize("how", ["argument", "current"])
@pytest.mark.parametrize("call", ["apply", "append"])
def test_a_rotary_may_go_before_its_call_has_run(pkg, how, call):
    """Its tables were made on one stream; the call that reads them waits on another when the object goes."""
    tokens, heads, dim = 40, 2, 64
    x = torch.randn((tokens, heads, dim), device="cuda")
    pos = torch.arange(tokens, device="cuda") * 3
    pool = [torch.zeros((5, 8, heads, dim), device="cuda") for _ in range(2)]
    table, length = torch.arange(5, dtype=torch.int32, device="cuda").view(1, 5), torch.tensor([tokens], dtype=torch.int32, device="cuda")
    cu = torch.tensor([0, tokens], dtype=torch.int32, device="cuda")
    pages = pkg.H2OPages(*pool)
    axes = [i % 2 for i in range(32)]
    two = torch.stack([pos, pos + 5])
    want, out = torch.empty_like(x), torch.zeros_like(x)

    def run(to, stream):
        r = pkg.H2ORotary(dim, axes=axes)  # (goes when run returns)
        kw = {"stream": stream} if how == "argument" else {}
        with torch.cuda.stream(stream if how == "current" else torch.cuda.current_stream()):
            if call == "apply":
                r.apply(x, two, to, **kw)
            else:
                pages.append(x, x, table, length, cu=cu, rotary=r, positions=two, q=x, q_out=to, **kw)

    run(want, torch.cuda.current_stream())
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    _waiting(side)
    run(out, side)
    others = _taken(32), [torch.full((32,), 255, dtype=torch.uint8, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    del others


def test_streams_of_another_library_are_left_alone(pkg):
    """Such a stream may be gone before the object: nothing is recorded on it."""
    raw = torch.cuda.Stream().cuda_stream
    outside = torch.cuda.ExternalStream(raw)
    r = pkg.H2ORotary(64)
    x, pos = torch.randn((3, 1, 64), device="cuda"), torch.arange(3, device="cuda")
    want, out = torch.empty_like(x), torch.empty_like(x)
    r.apply(x, pos, want)
    noted = []
    r._kept = [type("T", (), {"record_stream": lambda self, s: noted.append(s)})()]
    torch.cuda.synchronize()
    r.apply(x, pos, out, stream=outside)
    torch.cuda.synchronize()
    assert torch.equal(out, want) and not noted
    with torch.cuda.stream(torch.cuda.ExternalStream(torch.cuda.Stream().cuda_stream)):
        r.apply(x, pos, out)
    assert not noted
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(2):
        r.apply(x, pos, out, stream=s)
    assert noted == [s]
    torch.cuda.synchronize()


def test_the_status_word_may_go_before_its_call_has_run(pkg):
    """A wait that gives up writes into the status word, whose memory is nobody else's yet."""
    k, v = (torch.randn((8, 16, 2, 128), device="cuda").bfloat16() for _ in range(2))
    q = torch.randn((40, 2, 128), device="cuda").bfloat16()
    table, length, cu = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([list(range(8))], [120], [0, 40]))
    out, side = torch.empty_like(q), torch.cuda.Stream()
    torch.cuda.synchronize()
    _waiting(side)

    def run():
        pages = pkg.H2OPages(k, v)
        pkg.lib.h2o_debug_pages_set_polls(pages._h, 0)  # every wait gives up at once
        pages.attend(q, table, length, out, max_len=120, cu=cu, max_q=40, stream=side)

    run()
    others = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    assert all(int(x) == 0 for x in others)


def test_captured_calls_and_objects_that_go_later(pkg):
    """What a capture notes about its stream does no harm when the object goes, before or after the graph."""
    x, pos = torch.randn((5, 2, 64), device="cuda"), torch.arange(5, device="cuda")
    want, out = torch.empty_like(x), torch.empty_like(x)
    r = pkg.H2ORotary(64)
    r.apply(x, pos, want)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        r.apply(x, pos, out)
    other = pkg.H2ORotary(64)
    other.apply(x, pos, out, stream=torch.cuda.Stream())
    torch.cuda.synchronize()
    out.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    del g
    h = torch.cuda.CUDAGraph()
    with torch.cuda.graph(h):
        r.apply(x, pos, out)
        del other  # (given back while a capture is under way)
    h.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    del r, h
    torch.cuda.synchronize()

"""Rotary positions of many tokens, where a block takes several of them, on a B200 against 64-bit references (tolerances:
pages_reference.rotate)."""
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


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pairs", ["halves", "neighbours"])
@pytest.mark.parametrize("heads,dim,rotary_dim,axes", [
    (1, 8, 8, 1), (1, 8, 2, 1), (1, 16, 16, 2), (1, 16, 4, 1),  # one or two items to a token
    (1, 64, 64, 1), (3, 72, 72, 2), (2, 80, 20, 1), (5, 128, 128, 3), (1, 512, 512, 2), (7, 24, 6, 3)])
@pytest.mark.parametrize("tokens", [1185, 5003])  # (not multiples of 8, the most tokens of a block)
def test_many_tokens(pkg, dtype, pairs, heads, dim, rotary_dim, axes, tokens):
    g = torch.Generator().manual_seed(tokens + dim)
    freq = [10000.0 ** (-2.0 * i / rotary_dim) for i in range(rotary_dim // 2)]
    axis = [i % axes for i in range(rotary_dim // 2)]
    r = pkg.H2ORotary(dim, rotary_dim=rotary_dim, frequencies=freq, axes=None if max(axis) == 0 else axis, pairs=pairs)
    x = (torch.randn((tokens, heads, dim), generator=g) * 3).to(DT[dtype])
    pos = torch.randint(0, 100000, (max(axis) + 1, tokens), generator=g)
    for inverse in (False, True):
        want, tol = ref.rotate(x.double().numpy(), pos.numpy(), freq, axis, pairs == "halves", dtype, inverse)
        guard = torch.full((tokens + 16, heads, dim), 7.0, dtype=DT[dtype], device="cuda")
        out = guard[8:8 + tokens]
        r.apply(x.cuda(), pos.cuda(), out, inverse=inverse)
        ref.compare(out, want, tol, "rotated")
        assert (guard[:8] == 7.0).all() and (guard[8 + tokens:] == 7.0).all()
        here = x.cuda()
        r.apply(here, pos.cuda(), here, inverse=inverse)  # in place
        assert torch.equal(here, out)
        if rotary_dim < dim:
            assert torch.equal(here[..., rotary_dim:].cpu(), x[..., rotary_dim:])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_tokens_of_strided_heads(pkg, dtype):
    """A head of a packed projection, written into another one: what lies between stays."""
    tokens, dim = 3001, 16
    g = torch.Generator().manual_seed(4)
    packed = torch.randn((tokens, 3, dim), generator=g).to(DT[dtype]).cuda()
    out = torch.full((tokens, 2, dim), 5.0, dtype=DT[dtype], device="cuda")
    pos = torch.arange(tokens, device="cuda") * 7
    freq = [10000.0 ** (-i / 8) for i in range(8)]
    pkg.H2ORotary(dim, frequencies=freq).apply(packed[:, 1:2], pos, out[:, 1:])
    want, tol = ref.rotate(packed[:, 1:2].double().cpu().numpy(), pos.cpu().numpy()[None], freq, np.zeros(8, int), True, dtype)
    ref.compare(out[:, 1:], want, tol, "strided")
    assert (out[:, 0] == 5.0).all()

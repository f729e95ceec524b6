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

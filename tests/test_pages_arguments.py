"""What H2OPages and H2ORotary refuse or accept, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def b():
    import __graft_entry__

    __graft_entry__.build()
    from paper_2306_14048_b200 import binding

    return binding


# ---- pools ----
@pytest.mark.parametrize("shape", [(50, 16, 2, 128), (1, 16, 2, 128), (50, 16, 1, 64), (1, 8, 1, 64)])
def test_a_broadcast_pool_is_refused(b, shape):
    """Three strides of 0 mean dense to the library, so that rows would be written and read far behind the tensor."""
    one = torch.zeros(shape[3])
    for lead in ((1, 1, 1), (shape[0], 1, 1), (1, shape[1], 1), (1, 1, shape[2])):
        x = one.expand(*lead, shape[3]).contiguous().expand(shape)
        if all(s != 0 for s, n in zip(x.stride(), shape) if n > 1):
            continue
        with pytest.raises(ValueError):
            b._pool_strides(x, x)


def test_strides_of_pools(b):
    z = torch.zeros
    assert b._pool_strides(z(5, 16, 2, 64), z(5, 16, 2, 64)) == [2048, 128, 64, 1]
    heads = z(5, 2, 16, 64).transpose(1, 2)
    assert b._pool_strides(heads, heads) == [2048, 64, 1024, 1]
    both = z(5, 2, 16, 2, 64)
    assert b._pool_strides(both[:, 0], both[:, 1]) == [4096, 128, 64, 1]
    # strides that say nothing: one head, one page
    assert b._pool_strides(z(5, 16, 1, 64), z(5, 16, 1, 64)) == [1024, 64, 64, 1]
    assert b._pool_strides(z(1, 16, 2, 64), z(1, 16, 2, 64)) == [2048, 128, 64, 1]
    page = z(16, 2, 64)
    assert b._pool_strides(page.expand(1, 16, 2, 64), z(1, 16, 2, 64)) == [2048, 128, 64, 1]
    head = z(5, 16, 64).unsqueeze(2).expand(5, 16, 1, 64)
    assert b._pool_strides(head, head) == [1024, 64, 64, 1]
    for k, v in ((z(5, 16, 2, 64), heads), (z(5, 16, 2, 128)[..., ::2], z(5, 16, 2, 128)[..., ::2])):
        with pytest.raises(ValueError):
            b._pool_strides(k, v)

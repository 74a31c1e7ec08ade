"""What the paged cache and its attention say of their memory and their launches, without a GPU."""
import numpy as np
import pytest

from paper_2309_15531_amd import binding as B


@pytest.mark.parametrize("pages,page,heads,dim", [(1 << 25, 64, 1, 64), (1 << 26, 32, 1, 64), (2 ** 31 - 1, 32, 8, 128), (1 << 15, 1 << 16, 1, 256),
                                                  (2 ** 31 - 1, 65536, 1024, 256)])
def test_a_pool_of_2_31_positions_has_no_size(pages, page, heads, dim):
    """No other call takes one, and the largest product of these numbers passes 64 bits."""
    assert B.load_library().adadim_mx4_cache_bytes(pages, page, heads, dim) == 0


def test_the_largest_pools_have_their_size():
    for pages, page, heads, dim in (((1 << 26) - 1, 32, 1024, 256), ((1 << 15) - 1, 1 << 16, 1024, 256)):
        assert B.load_library().adadim_mx4_cache_bytes(pages, page, heads, dim) == int(np.prod(B.mx4_cache_shape(pages, page, heads, dim), dtype=object))

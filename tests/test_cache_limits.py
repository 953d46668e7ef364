"""libbscache.so at the ends of what it takes (no GPU): every call below fails
validation, has nothing to do or is described only."""
import ctypes

from paper_1810_11066_amd import cache as kc
from tests.test_cache_abi import (A, B, C, D, E, INVALID, attend, lib, pages,
                                  params, workspace)

assert lib      # (a fixture)


def test_an_empty_batch_needs_no_workspace(lib):
    """Also where a batch of one would be shared."""
    one, none = (params(batch=n, max_pages=100, max_len=1600) for n in (1, 0))
    assert workspace(lib, p=one)[1] > 0
    assert workspace(lib, p=none) == (kc.OK, 0)
    assert lib.bscache_attend(pages(), none, A, B, C, D, E, None, 0,
                              None) == kc.OK
    assert attend(lib, p=one, space=0) == INVALID

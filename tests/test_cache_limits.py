"""libbscache.so at the ends of what it takes (no GPU): every call below fails
validation, has nothing to do or is described only."""
import types

import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests.test_cache_abi import (A, B, C, D, E, INVALID, KC, UNSUPPORTED,
                                  attend, lib, pages, params, read, workspace,
                                  write)

assert lib      # (a fixture)


def test_an_empty_batch_needs_no_workspace(lib):
    """Also where a batch of one would be shared."""
    one, none = (params(batch=n, max_pages=100, max_len=1600) for n in (1, 0))
    assert workspace(lib, p=one)[1] > 0
    assert workspace(lib, p=none) == (kc.OK, 0)
    assert lib.bscache_attend(pages(), none, A, B, C, D, E, None, 0,
                              None) == kc.OK
    assert attend(lib, p=one, space=0) == INVALID


@pytest.mark.parametrize("dim,lanes", [(256, 32), (144, 32), (128, 16),
                                       (80, 16), (64, 8), (16, 2)])
@pytest.mark.parametrize("heads", [1, 8])
def test_rows_of_a_launch(lib, dim, lanes, heads):
    """As many as its lanes, two rows to a lane, and no more than 2^31 - 1: what
    fits gets to the check of overlaps (and is refused there)."""
    cache = pages(heads=heads, dim=dim)
    most = min((2 ** 31 - 1) // (2 * heads),
               (2 ** 26 - 4) // (2 * heads) * (128 // lanes))
    assert abs(most * 2 * heads * lanes / min(2 ** 33, 2 ** 31 * lanes) - 1) \
        < 1e-6
    stride = heads * dim
    for tokens, status in ((most, INVALID), (most + 1, UNSUPPORTED)):
        assert read(lib, cache, tokens=tokens, v=KC) == status
        assert write(lib, cache, tokens=tokens, ks=stride, vs=stride,
                     slots=KC) == status
    assert b"rows" in lib.bscache_last_error()


def test_pairs_of_a_launch(lib):
    """Whole pairs are a workgroup each, and so are those of the join: 2^24 of a
    sequence and up to 16 heads of a key-value head are too many."""
    def status(batch, kv_heads, group, length):
        heads = kv_heads * group
        return workspace(lib, pages(heads=kv_heads), params(
            batch=batch, heads=heads, stride=64 * heads, max_len=length,
            max_pages=100))[0]
    assert status(2 ** 22 - 1, 4, 16, 512) == kc.OK
    assert status(2 ** 22, 4, 16, 512) == UNSUPPORTED
    assert status(2 ** 21 - 1, 4, 17, 16) == kc.OK          # two tiles each
    assert status(2 ** 21, 4, 17, 16) == UNSUPPORTED
    assert status(2 ** 24 - 1, 1, 1, 1024) == kc.OK
    assert status(2 ** 24, 1, 1, 1024) == UNSUPPORTED
    assert b"pairs" in lib.bscache_last_error()


def test_a_stream_of_another_device_is_refused():
    """Its handle would not be used: the call would go to the current stream of
    the cache's device."""
    class OnSecond(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 1
    cache = kc.Pages(*(torch.zeros((2, 1, 16, n), dtype=t).as_subclass(
        OnSecond) for n, t in ((64, torch.uint8), (2, torch.bfloat16)) * 2))
    x, slots = torch.zeros((3, 1, 64)), torch.zeros(3, dtype=torch.int32)
    stream = types.SimpleNamespace(device=torch.device("cuda", 0))
    for call in (lambda: kc.write(x, x, slots, cache, stream=stream),
                 lambda: kc.read(slots, cache, 64, stream=stream),
                 lambda: kc.attend(x, cache, slots.view(3, 1), slots,
                                   stream=stream)):
        with pytest.raises(ValueError, match="cuda:0, the cache on cuda:1"):
            call()


def test_describe_refuses_as_a_call_does():
    sizes = dict(pages=4, kv_heads=1, page_tokens=16, dim=64, batch=1, heads=4,
                 max_len=16)
    assert kc.describe(**sizes).startswith("attend_kernel<64")
    for change, error in ((dict(page_tokens=0), kc.CacheError),
                          (dict(page_tokens=-16), kc.CacheError),
                          (dict(dim=24), kc.CacheError),
                          (dict(dtype=torch.float64), TypeError),
                          (dict(kv_heads=1 << 31), ValueError),
                          (dict(pages=1 << 63), ValueError),
                          (dict(dim=64.0), ValueError)):
        with pytest.raises(error):
            kc.describe(**{**sizes, **change})


@pytest.mark.parametrize("dim,dtype,ways", [
    (64, torch.bfloat16, "whole shared wide wide whole shared whole shared"),
    (128, torch.float16, "whole shared wide wide whole whole whole shared"),
    (256, torch.bfloat16, "whole shared wide shared whole whole whole shared"),
    (96, torch.float32, "whole shared wide shared whole whole whole shared")])
def test_ways_at_the_bounds_of_the_plan(dim, dtype, ways):
    """Those that test_gpu_cache.test_attend_on_both_sides_of_the_plan is made
    for (256 compute units)."""
    calls = ((1, 500), (1, 700), (12, 700), (20, 1500), (50, 1000), (60, 1100),
             (70, 2000), (70, 2100))
    assert [kc.describe(200, 8, 32, dim, batch, 16, longest, 8, 4,
                        dtype=dtype).split()[4]
            for batch, longest in calls] == ways.split()

"""GPU: what the cache's Python binding makes of its arguments."""
import numpy as np
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests.test_gpu_cache import Filled, queries

pytestmark = pytest.mark.gpu


def test_bounds_in_objects_that_change():
    """max_len and window of any integer kind count as what they are at the
    call, a tensor's that is written between two calls as well."""
    rng = np.random.default_rng(1)
    f = Filled(rng, 8, 1, 16, 64, 8, 4)
    q = queries(rng, 2, 4, 64, "bf16")
    table = torch.from_numpy(rng.integers(0, 8, (2, 100)).astype(np.int32))
    args = f.cache, table.cuda(), torch.tensor([40, 1500], dtype=torch.int32,
                                               device="cuda")
    most, window = torch.tensor(64), torch.tensor(0)
    for m, w in ((64, 0), (1600, 0), (1600, 33), (300, 0)):
        most.fill_(m)
        window.fill_(w)
        want = kc.attend(q, *args, max_len=m, window=w)
        for a, b in ((most, window), (np.int64(m), np.int32(w))):
            got = kc.attend(q, *args, max_len=a, window=b)
            assert torch.equal(got[0], want[0])
            assert torch.equal(got[1], want[1])
    for kw in ({"window": 1.5}, {"max_len": 64.0}, {"max_len": 1 << 31},
               {"window": "1"}):
        with pytest.raises(ValueError, match="32-bit"):
            kc.attend(q, *args, **kw)

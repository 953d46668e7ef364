"""GPU: the cache's attention where numbers are far apart or near a type's
ends, against float64 (tests/cache_reference.py)."""
import numpy as np
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests import cache_reference as ref
from tests.test_gpu_cache import DTYPE, Filled, host, queries, rounded, say

pytestmark = pytest.mark.gpu


def on(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ---- bfloat16 calls keep a weight in both terms ------------------------------

@pytest.mark.parametrize("vbits", [8, 4])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_bfloat16_outputs_are_the_result_rounded_once(dim, vbits):
    """Half a step of bfloat16 at the result, and what binary32 sums and
    weights of 22 bits may add: ref.attention's bound of float16 calls without
    their output's own rounding.  Logits are small, so that they add next to
    nothing."""
    say(dim, vbits)
    rng = np.random.default_rng(dim + vbits)
    batch, heads, n = 24, 16, 24
    f = Filled(rng, 30, 2, 16, dim, 8, vbits)
    table = rng.integers(0, 30, (batch, 2)).astype(np.int32)
    q = queries(rng, batch, heads, dim, "bf16")
    out, _ = kc.attend(q, f.cache, torch.from_numpy(table).cuda(),
                       on([n] * batch), scale=1e-4)
    got, qh = host(out).astype(np.float64), host(q)
    t = np.arange(n)
    for b in range(batch):
        slot = table[b, t // 16].astype(np.int64) * 16 + t % 16
        for h in range(heads):
            g = h // 8
            (ck, sk, zk), (cv, sv, zv) = f.held
            o, _, tol, _ = ref.attention(
                qh[b, h], ck[slot, g], sk[slot, g], zk[slot, g], cv[slot, g],
                sv[slot, g], zv[slot, g], 1e-4, 8, vbits, "f16")
            more = tol - ref.STEP["f16"] * np.abs(o)
            half = 2.0 ** (np.floor(np.log2(np.abs(o) + more)) - 8)
            off = np.abs(got[b, h] - o)
            assert (off <= half + more).all(), (b, h, (off - half).max())

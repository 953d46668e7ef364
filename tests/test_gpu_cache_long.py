"""GPU: attention over sequences next to 2^31 tokens, the pages of which a table
names again and again."""
import numpy as np
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests import cache_reference as ref
from tests.test_gpu_cache import Filled, host, queries, say

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("window", [1, 130, 300, 1500])
@pytest.mark.parametrize("dim", [16, 128])
def test_windows_at_the_end(window, dim):
    """The last tokens of sequences that end where a unit passes 2^31."""
    say(window, dim)
    rng = np.random.default_rng(window)
    lengths = [MOST, MOST - 15, MOST - 16, MOST - 127, MOST - 128, MOST - 700,
               5]
    f = Filled(rng, 3, 1, 2 ** 11, dim, 4, 8)
    table = np.zeros((len(lengths), 2 ** 20), np.int32)
    table[:, -2:] = [1, 2]
    table[3, -1] = -1
    f.check(queries(rng, len(lengths), 2, dim, "bf16"),
            torch.from_numpy(table).cuda(),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            window=window, kind="bf16")


@pytest.mark.parametrize("length", [MOST, MOST - 127, MOST - 128])
def test_all_tokens(length):
    """A wave of the 768 workgroups takes 2^31 / (4 * 768 * 32) = 21846 steps:
    a lane adds 8 terms in each, so its sums of p and of p z are off by 174763
    roundings of 2^-24 at most, and the products' by 21846 of 2^-22 (see
    ref.error_terms), beside what a short call may be off by."""
    say(length)
    rng = np.random.default_rng(1)
    page = 2 ** 17
    f = Filled(rng, 1, 1, page, 16, 4, 4)
    q = queries(rng, 1, 1, 16, "bf16")
    table = torch.zeros((1, 2 ** 31 // page), dtype=torch.int32, device="cuda")
    out, lse = kc.attend(q, f.cache, table, torch.tensor(
        [length], dtype=torch.int32, device="cuda"))
    (ck, sk, zk), (cv, sv, zv) = ((c[:, 0], s[:, 0], z[:, 0])
                                  for c, s, z in f.held)
    k = zk[:, None] + sk[:, None] * ck.astype(np.float64)
    v = zv[:, None] + sv[:, None] * cv.astype(np.float64)
    x = k @ host(q)[0, 0].astype(np.float64) / 4
    often = np.full(page, 2.0 ** 31 / page)
    often[length - 2 ** 31:] -= 1
    p = often * np.exp(x)
    want = p @ v / p.sum()
    *_, tol, ltol = ref.attention(host(q)[0, 0], ck, sk, zk, cv, sv, zv, 0.25,
                                  4, 4, "bf16")
    add, products = 174763 * 2.0 ** -24, 21846 * 2.0 ** -22
    spread = p @ (sv[:, None] * cv + np.abs(zv)[:, None]) / p.sum()
    assert abs(float(lse) - np.log(p.sum())) <= ltol + add
    assert (np.abs(host(out)[0, 0] - want) <=
            tol + spread * (2 * add + products)).all()

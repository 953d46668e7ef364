"""GPU: every way in which the cache's attention shares a call out, with more
than 16 query heads to a key-value head, windows, and joins of every shape,
against float64 on the GPU; each call's way is asserted."""
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests import cache_reference as ref
from tests.test_gpu_cache import DTYPE, say

pytestmark = pytest.mark.gpu


def check(way, batch, kv, group, dim, kind, longest, window=0, page=32,
          pages=200, kbits=8, vbits=4):
    """attend of random lengths up to the longest, one of them empty; the bounds
    are those of ref.error_terms."""
    say(way, batch, kv, group, dim, kind, longest, window)
    assert " %s " % way in kc.describe(pages, kv, page, dim, batch, kv * group,
                                       longest, kbits, vbits, window,
                                       DTYPE[kind])
    gen = torch.Generator(device="cuda").manual_seed(batch + longest + group)
    cache = kc.empty(pages, kv, page, dim, kbits, vbits)
    k, v = (torch.randn((pages * page, kv, dim), generator=gen, device="cuda")
            for _ in range(2))
    slots = torch.arange(pages * page, dtype=torch.int32, device="cuda")
    kc.write(k, v, slots, cache)
    # rows as offset and rest: value = s c' + z', both float64
    rest, offset = [], []
    for x, steps, bits in zip(kc.read(slots, cache, dim),
                              (cache.k_steps, cache.v_steps), (kbits, vbits)):
        s, z = steps.double().transpose(1, 2).reshape(-1, kv, 2).unbind(-1)
        offset.append((z + ref.centre(kind, bits) * s)[..., None])
        rest.append(x.double() - offset[-1])
    table = torch.randint(pages, (batch, -(-longest // page)), generator=gen,
                          device="cuda", dtype=torch.int32)
    lengths = torch.randint(longest + 1, (batch,), generator=gen,
                            device="cuda", dtype=torch.int32)
    lengths[0] = longest
    if batch > 1:
        lengths[1] = 0
    q = torch.randn((batch, kv * group, dim), generator=gen,
                    device="cuda").to(DTYPE[kind])
    out, lse = kc.attend(q, cache, table, lengths, window=window,
                         max_len=longest)
    for b in range(batch):
        n = int(lengths[b])
        t = torch.arange(max(0, n - window) if window else 0, n, device="cuda")
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -torch.inf).all()
            continue
        slot = table[b].long()[t // page] * page + t % page
        # (n, kv, dim) -> (kv, dim, n) and (kv, n, dim), contiguous
        kr, kz = (x[0][slot].permute(1, 2, 0).contiguous()
                  for x in (rest, offset))
        vr, vz = (x[1][slot].permute(1, 0, 2).contiguous()
                  for x in (rest, offset))
        qb = q[b].double().view(kv, group, dim)
        x = torch.matmul(qb, kr + kz) * dim ** -0.5
        p = torch.softmax(x, -1)
        want = torch.matmul(p, vr + vz).view(kv * group, dim)
        size = dim ** -0.5 * (torch.matmul(qb.abs(), kr.abs()) +
                              qb.abs().sum(-1, keepdim=True) * kz.abs())
        by_logit, by_weight, by_sum = ref.error_terms(kind, dim, len(t))
        d = float(size.max() * by_logit + x.abs().max() * 2.0 ** -21)
        spread = torch.matmul(p, vr.abs() + vz.abs()).view(kv * group, dim)
        tol = ref.STEP[kind] * want.abs() + \
            spread * (by_weight + 2 * d + by_sum)
        assert ((out[b].double() - want).abs() <= tol).all(), (b, n)
        total = torch.logsumexp(x, -1).view(-1)
        far = (lse[b].double() - total).abs()
        assert (far <= d + by_sum + 2.0 ** -22 * total.abs()).all(), (b, n)


@pytest.mark.parametrize("group,dim,kind", [(17, 64, "bf16"), (24, 128, "f16"),
                                            (40, 256, "bf16"), (33, 80, "f32")])
@pytest.mark.parametrize("longest", [600, 3000])
def test_shared_head_tiles(group, dim, kind, longest):
    """More than one tile of 16 heads, the last one short, joined all heads
    together (600 tokens of narrow rows) and one by one."""
    check("shared", 2, 2, group, dim, kind, longest)


@pytest.mark.parametrize("group", [16, 19])
@pytest.mark.parametrize("dim,kind,batch,kv,longest", [
    (64, "f16", 34, 8, 1100), (128, "bf16", 34, 8, 1100),
    (96, "f32", 32, 8, 2100), (256, "f16", 32, 8, 2100)])
def test_join_of_many_columns(group, dim, kind, batch, kv, longest):
    """A pair for every CU and 16 heads: the join's threads are one row of 256
    to 1024 columns, the last round of which may be short."""
    if group > 16:
        batch //= 2                  # as many pairs
    check("shared", batch, kv, group, dim, kind, longest)


@pytest.mark.parametrize("dim,kind", [(64, "bf16"), (128, "f16"),
                                      (256, "bf16"), (112, "f32")])
def test_wide_with_a_window(dim, kind):
    check("wide", 12, 8, 3, dim, kind, 5000, window=600)


@pytest.mark.parametrize("group,dim,kind", [(20, 64, "bf16"), (32, 128, "f32"),
                                            (17, 256, "f16")])
def test_wide_head_tiles(group, dim, kind):
    check("wide", 8, 4, group, dim, kind, 700)


@pytest.mark.parametrize("group,dim,kind", [(20, 64, "f32"), (40, 256, "f32"),
                                            (17, 128, "bf16")])
def test_whole_head_tiles_and_windows(group, dim, kind):
    check("whole", 5, 2, group, dim, kind, 500)
    check("whole", 5, 2, group, dim, kind, 3000, window=300)
    check("shared", 5, 2, group, dim, kind, 3000, window=1000)

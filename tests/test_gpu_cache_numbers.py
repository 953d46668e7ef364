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


# ---- rows of one sequence far apart in size ----------------------------------

@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("vbits", [8, 4])
@pytest.mark.parametrize("size", [2.0 ** 15, 2.0 ** 22, 2.0 ** 30, np.inf])
def test_a_wide_row_that_nobody_attends_to(kind, vbits, size):
    """One token of 40 with a logit 100 lower and values `size` times larger
    (an infinity is kept as 2^126) leaves the others' weights as they are, at
    each place in a wave's tile, among the first tokens and the last."""
    say(kind, vbits, size)
    rng = np.random.default_rng(7)
    n, dim = 48, 64
    q = rounded(np.ones((6, 1, dim)) * 0.5, kind)[1]
    k = rng.standard_normal((6 * n, 1, dim)) * 0.05
    v = rng.standard_normal((6 * n, 1, dim))
    for b, at in enumerate((0, 5, 17, 31, 33, 39)):
        k[b * n + at] = -25.0                   # 0.5 * 64 * 25 / 8 = 100
        if np.isinf(size):
            v[b * n + at, 0, 3] = np.inf
        else:
            v[b * n + at] *= size
    with np.errstate(all="ignore"):
        f = Filled(rng, 18, 1, 16, dim, 8, vbits, rows=[k, v])
    f.check(q, on(np.arange(18).reshape(6, 3)), on([40] * 6), kind=kind)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_wide_rows_in_other_waves_and_workgroups(kind):
    """The same in a sequence that several workgroups share: waves and partial
    results of different references are joined."""
    say(kind)
    rng = np.random.default_rng(8)
    n, dim = 3000, 64
    q = rounded(np.ones((1, 2, dim)) * 0.5, kind)[1]
    k = rng.standard_normal((n + 8, 1, dim)) * 0.05
    v = rng.standard_normal((n + 8, 1, dim))
    for at, size in ((10, 2.0 ** 26), (700, 2.0 ** 40), (1500, 2.0 ** 100),
                     (2999, 2.0 ** 30)):
        k[at] = -30.0
        v[at] *= size
    f = Filled(rng, 188, 1, 16, dim, 8, 8, rows=[k, v])
    assert " shared " in kc.describe(188, 1, 16, dim, 1, 2, 188 * 16,
                                     dtype=DTYPE[kind])
    f.check(q, on(np.arange(188)[None]), on([n]), kind=kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("n", [7, 300, 3000])
def test_values_at_the_ends(kind, n):
    """Rows of the largest values attended to beside ordinary ones, nothing but
    the largest, constant rows (steps of 2^-60) of large, alternating and tiny
    values: outputs are the mean, and lse knows nothing of the values."""
    say(kind, n)
    rng = np.random.default_rng(n)
    dim, pages = 64, -(-n // 16)
    k = rng.standard_normal((16 * pages, 1, dim))
    q = queries(rng, 1, 3, dim, kind)
    table, lengths = on(np.arange(pages)[None]), on([n])
    lse = []
    some = rng.standard_normal((16 * pages, 1, dim))
    one = some.copy()
    one[n // 2] = np.inf
    sign = np.where(np.arange(16 * pages) % 2, 1.0, -1.0)[:, None, None]
    for v in (some, one, np.full_like(some, np.inf), np.full_like(some, 1e30),
              sign * np.full_like(some, 1e30), np.full_like(some, 1e-30),
              some * 1e34, some * 1e-15,
              np.where(np.arange(16 * pages)[:, None, None] < n // 2, 1e36,
                       some)):
        with np.errstate(all="ignore"):
            f = Filled(rng, pages, 1, 16, dim, 8, 8, rows=[k, v])
        lse.append(f.check(q, table, lengths, kind=kind)[1])
    for other in lse[1:]:
        assert np.array_equal(lse[0], other)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_logits_that_rise_and_wide_rows_that_fade(kind):
    """Logits rise by up to 300 along the sequence while the steps fall and
    rise: a reference that was set by a token long past does not last."""
    say(kind)
    rng = np.random.default_rng(9)
    n, dim = 480, 64
    rise = np.linspace(0, 1, n)
    q = rounded(np.ones((1, 4, dim)) * np.array([0.0, 0.1, 0.5, -0.5])
                [None, :, None], kind)[1]
    k = rng.standard_normal((n, 1, dim)) * 0.01 + 75 * rise[:, None, None]
    for power in (np.linspace(60, -40, n), np.linspace(-40, 60, n),
                  30 * np.cos(np.arange(n))):
        v = rng.standard_normal((n, 1, dim)) * (2.0 ** power)[:, None, None]
        f = Filled(rng, 30, 1, 16, dim, 8, 8, rows=[k, v])
        f.check(q, on(np.arange(30)[None]), on([n]), kind=kind)


# ---- queries ----------------------------------------------------------------

@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("batch,longest", [(2, 64), (3, 3000), (64, 700)])
def test_nothing_visible_with_a_query_that_is_no_number(bad, kind, batch,
                                                        longest):
    """A padded place of a batch (length 0, or a table without a page, and
    whatever its query holds) gives 0 and -inf however the call is shared; a
    head with visible tokens gives NaN, the others what they are."""
    say(bad, kind, batch, longest)
    rng = np.random.default_rng(batch)
    f = Filled(rng, 40, 2, 16, 64, 8, 4)
    per = -(-longest // 16)
    table = rng.integers(0, 40, (batch, per)).astype(np.int32)
    lengths = rng.integers(1, longest, batch).astype(np.int32)
    lengths[0], lengths[batch - 1] = 0, longest
    table[1] = -1
    q = queries(rng, batch, 4, 64, kind)
    args = f.cache, torch.from_numpy(table).cuda(), on(lengths)
    want, want_lse = (host(t) for t in kc.attend(q, *args))
    q[0], q[1, 2] = bad, bad
    q[batch - 1, 3, 5] = bad
    out, lse = (host(t) for t in kc.attend(q, *args))
    assert (out[:2] == 0).all() and (lse[:2] == -np.inf).all()
    if batch > 2:
        assert np.isnan(out[-1, 3]).all() and np.isnan(lse[-1, 3])
        out[-1, 3], lse[-1, 3] = want[-1, 3], want_lse[-1, 3]
    assert np.array_equal(out, want) and np.array_equal(lse, want_lse)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("kbits", [8, 4])
@pytest.mark.parametrize("size", [1e-36, 1e36, 2.5e36])
def test_queries_far_from_one(kind, kbits, size):
    """The scale brings the logits back to a few units."""
    say(kind, kbits, size)
    rng = np.random.default_rng(11)
    f = Filled(rng, 8, 1, 32, 64, kbits, 8)
    q = rounded(rng.uniform(-1, 1, (2, 4, 64)) * size, kind)[1]
    scale = float(np.float32(4.0 / size)) if size > 1 else 1e35
    f.check(q, on(np.arange(8).reshape(2, 4)), on([100, 128]), scale=scale,
            kind=kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("kbits", [8, 4])
@pytest.mark.parametrize("size", [2e37, 3e38])
def test_queries_whose_sum_is_beyond_binary32(kind, kbits, size):
    """Finite queries of one sign, the sum of which is none."""
    say(kind, kbits, size)
    rng = np.random.default_rng(12)
    f = Filled(rng, 8, 1, 32, 64, kbits, 8)
    q = rounded(rng.uniform(0.25, 1, (2, 4, 64)) * size, kind)[1]
    f.check(q, on(np.arange(8).reshape(2, 4)), on([100, 128]),
            scale=float(np.float32(4.0 / size)), kind=kind)


def small_scale(kind, scale, size, keys, kbits=8):
    say(kind, scale, size, keys)
    rng = np.random.default_rng(12)
    k = rng.standard_normal((128, 1, 64)) * keys
    v = rng.standard_normal((128, 1, 64))
    f = Filled(rng, 8, 1, 16, 64, kbits, 8, rows=[k, v])
    q = rounded(rng.standard_normal((2, 4, 64)) * size, kind)[1]
    f.check(q, on(np.arange(8).reshape(2, 4)), on([60, 64]),
            scale=float(np.float32(scale)), kind=kind)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("scale,size,keys", [
    (0.0, 1.0, 1e30), (-0.0, 1e-30, 1.0), (1e-32, 1.0, 1e31),
    (0.1, 1e-30, 1e30), (1e-12, 1e-18, 1e30), (1.0, 1e-37, 1e31)])
def test_small_scales_of_large_keys(kind, scale, size, keys):
    """scale * q far below 1 with keys far above: logits of 0 or of a few
    units."""
    small_scale(kind, scale, size, keys)


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("kbits", [8, 4])
@pytest.mark.parametrize("scale,size,keys", [
    (0.0, 1e30, 1e36), (1e-20, 1e-18, 1e37), (0.1, 1e-35, 1e35)])
def test_keys_far_from_one(kind, kbits, scale, size, keys):
    """The same of keys next to the largest that a cache keeps."""
    small_scale(kind, scale, size, keys, kbits)


@pytest.mark.parametrize("kind", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("kbits", [8, 4])
def test_keys_at_the_ends(kind, kbits):
    """Keys up to 2^126 (what infinities are kept as) in every channel, with
    queries of one sign, and a scale that brings the logits back."""
    say(kind, kbits)
    rng = np.random.default_rng(13)
    n, dim = 64, 256
    k = rng.standard_normal((n, 1, dim)) * 1e37
    k[3, 0, 1:] = np.inf
    k[3, 0, 0] = -np.inf
    k[9] = -np.inf
    k[9, 0, 77] = np.inf
    k[11] = np.inf
    v = rng.standard_normal((n, 1, dim))
    with np.errstate(all="ignore"):
        f = Filled(rng, 4, 1, 16, dim, kbits, 8, rows=[k, v])
    # (the largest logit: 256 * 2^126 * scale * q = 20)
    q = np.ones((1, 2, dim)) * np.array([255 / 128, -1.5])[None, :, None] / 1024
    q[0, :, 0] *= -1                # as the key's: nothing cancels
    q = rounded(q, kind)[1]
    f.check(q, on([[0, 1, 2, 3]]), on([n]), scale=20 * 2.0 ** -125, kind=kind)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("scale", [1 + i / 64 for i in range(24)])
def test_logits_that_binary32_has_in_steps_of_128(kind, scale):
    """Logits of 2^30 and the next number in binary32: only the largest count.
    (Two thirds of a shared sequence hold keys of 1, the rest keys of 1 + 2^-23,
    every product and sum exact.)"""
    say(kind, scale)
    rng = np.random.default_rng(14)
    n, dim, first = 3000, 64, 2000
    f = Filled(rng, 188, 1, 16, dim, 8, 8)
    kc_, ks = f.cache.k_codes, f.cache.k_steps
    kc_.zero_()
    kc_.view(-1, dim)[first:] = 1
    ks[..., 0], ks[..., 1] = 2.0 ** -23, 1.0
    q = torch.full((1, 1, dim), 2.0 ** 10, dtype=DTYPE[kind], device="cuda")
    assert " shared " in kc.describe(188, 1, 16, dim, 1, 1, 188 * 16,
                                     dtype=DTYPE[kind])
    out, lse = kc.attend(q, f.cache, on(np.arange(188)[None]), on([n]),
                         scale=scale * 2.0 ** 14)
    cv, sv, zv = (t[first:n, 0] for t in f.held[1])
    v = zv[:, None] + sv[:, None] * cv.astype(np.float64)
    # (sums of 1000 tokens: ref.error_terms)
    _, by_weight, by_sum = ref.error_terms(kind, dim, n - first)
    tol = ref.STEP[kind] * np.abs(v.mean(0)) + \
        np.abs(v).mean(0) * (by_weight + by_sum) * 3
    assert (np.abs(host(out)[0, 0] - v.mean(0)) <= tol).all()
    # half a step of the logit, and of its product with log2 e and ln 2
    want = scale * 2.0 ** 30 * (1 + 2.0 ** -23)
    assert abs(float(lse) - want) <= 4 * 2.0 ** -24 * want


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n", [200, 3000])
def test_heads_know_nothing_of_each_other(kind, n):
    """A head's bits are the same whatever the other heads of its tile hold;
    the rows' sizes and the logits are far enough apart for references to move
    all the time."""
    say(kind, n)
    rng = np.random.default_rng(n)
    dim, pages = 64, -(-n // 16)
    k = rng.standard_normal((16 * pages, 1, dim)) * 4
    v = rng.standard_normal((16 * pages, 1, dim)) * \
        2.0 ** rng.uniform(-30, 10, (16 * pages, 1, 1))
    f = Filled(rng, pages, 1, 16, dim, 8, 8, rows=[k, v])
    q = queries(rng, 1, 12, dim, kind)
    args = f.cache, on(np.arange(pages)[None]), on([n])
    out, lse = f.check(q, *args[1:], kind=kind)
    for other in (0.0, 1e3, float("nan"), float("inf")):
        for keep in (0, 7, 11):
            p = torch.full_like(q, other)
            p[:, keep] = q[:, keep]
            got, got_lse = (host(t) for t in kc.attend(p, *args))
            assert np.array_equal(got[:, keep], out[:, keep]), (other, keep)
            assert np.array_equal(got_lse[:, keep], lse[:, keep])


def test_small_weights_beside_a_head_that_is_no_number():
    """Weights 2^-24 of a wave's largest, which came within what a reference may
    lag: what float16 holds of them does not depend on another head."""
    rng = np.random.default_rng(15)
    n, dim = 500, 64
    k = rng.standard_normal((512, 1, dim)) * 0.01
    v = rng.standard_normal((512, 1, dim)) * 2.0 ** -16
    v[0], v[128] = rng.standard_normal((2, 1, dim)) * [[[1.0]], [[180.0]]]
    f = Filled(rng, 32, 1, 16, dim, 8, 8, rows=[k, v])
    q = queries(rng, 1, 12, dim, "f32")
    args = f.cache, on(np.arange(32)[None]), on([n])
    out, lse = f.check(q, *args[1:], kind="f32")
    q[0, 5] = float("nan")
    got, got_lse = (host(t) for t in kc.attend(q, *args))
    rest = np.arange(12) != 5
    assert np.array_equal(got[:, rest], out[:, rest])
    assert np.array_equal(got_lse[:, rest], lse[:, rest])


@pytest.mark.parametrize("kind", ["f16", "bf16"])
@pytest.mark.parametrize("kbits,vbits", [(8, 4), (4, 8)])
@pytest.mark.parametrize("window", [0, 1])
def test_one_visible_token_is_its_value(kind, kbits, vbits, window):
    """Bit for bit what a read gives: values of 4 bits and a step of 8 lie on
    ties of the output's type, where any rounding of the weight shows."""
    say(kind, kbits, vbits, window)
    rng = np.random.default_rng(16)
    dim, batch = 128, 48
    f = Filled(rng, batch, 2, 16, dim, kbits, vbits)
    n = np.ones(batch) if not window else np.r_[rng.integers(1, 17, batch - 1),
                                                16]
    q = queries(rng, batch, 6, dim, kind) * 3
    out, _ = kc.attend(q, f.cache, on(np.arange(batch)[:, None]), on(n),
                       window=window)
    _, v = kc.read(on(np.arange(batch) * 16 + n - 1), f.cache, dim, DTYPE[kind])
    assert torch.equal(out, v.repeat_interleave(3, 1))


@pytest.mark.parametrize("kind", ["f32", "bf16"])
def test_lse_of_equal_logits_is_the_logarithm_of_their_number(kind):
    """Sums of equal weights are exact; the logarithm of the fraction, the sum
    with the exponent and the product with ln 2 (and ln 2 itself) are a rounding
    each."""
    rng = np.random.default_rng(17)
    n = np.r_[1:40, rng.integers(40, 3000, 60)]
    f = Filled(rng, 188, 1, 16, 64, 8, 8)
    table = np.broadcast_to(np.arange(188), (len(n), 188)).copy()
    q = torch.zeros((len(n), 2, 64), dtype=DTYPE[kind], device="cuda")
    _, lse = kc.attend(q, f.cache, on(table), on(n))
    want = np.log(n)[:, None]
    off = np.abs(host(lse).astype(np.float64) - want)
    assert (off <= 4 * 2.0 ** -24 * np.maximum(want, 0.5)).all(), off.max()

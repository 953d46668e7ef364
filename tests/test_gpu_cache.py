"""GPU: the quantized key-value cache (write, read) and the attention over its
pages, against the definition in plain numpy (tests/cache_reference.py)."""
import numpy as np
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests import cache_reference as ref

pytestmark = pytest.mark.gpu

DTYPE = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def gpu():
    assert torch.cuda.is_available(), "GPU tests need the MI355X"
    kc.load_library()
    yield


def say(*a):
    print(*a, flush=True)


def rounded(x, kind):
    """float32 numpy rows as the type holds them, and the GPU tensor."""
    t = torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(DTYPE[kind])
    return t.float().numpy(), t.cuda()


def host(t):
    return t.float().cpu().numpy()


class Filled:
    """A cache filled through write, with what numpy says it holds."""

    def __init__(self, rng, pages, kv_heads, page, dim, kbits, vbits,
                 kind="f32", rows=None):
        self.page, self.dim, self.bits = page, dim, (kbits, vbits)
        self.cache = kc.empty(pages, kv_heads, page, dim, kbits, vbits)
        for t in self.cache:                # rows nobody wrote: NaN steps
            t.view(torch.uint8).fill_(0xFF)
        n = pages * page
        if rows is None:
            rows = [rng.standard_normal((n, kv_heads, dim)) *
                    np.where(np.arange(dim) % 16 == 0, 3.0, 1.0),
                    rng.standard_normal((n, kv_heads, dim))]
        (kh, k), (vh, v) = (rounded(r, kind) for r in rows)
        kc.write(k, v, torch.arange(n, dtype=torch.int32, device="cuda"),
                 self.cache)
        self.held = [ref.quantize(kh, kbits), ref.quantize(vh, vbits)]

    def check(self, q, table, lengths, scale=None, window=0, max_len=None,
              kind="f32"):
        """attend's result against the reference, every element."""
        qh = host(q)
        tb, ln = table.cpu().numpy(), lengths.cpu().numpy()
        out, lse = kc.attend(q, self.cache, table, lengths, scale=scale,
                             window=window, max_len=max_len)
        torch.cuda.synchronize()
        out, lse = host(out), host(lse)
        batch, heads, dim = qh.shape
        kv = self.cache.k_codes.shape[1]
        pages = self.cache.k_codes.shape[0]
        scale = dim ** -0.5 if scale is None else scale
        most = tb.shape[1] * self.page if max_len is None else max_len
        worst = 0.0
        for b in range(batch):
            n = min(max(int(ln[b]), 0), most)
            t = np.arange(max(0, n - window) if window else 0, n)
            at = tb[b, t // self.page].astype(np.int64)
            ok = (at >= 0) & (at < pages)
            slot = at[ok] * self.page + t[ok] % self.page
            for h in range(heads):
                g = h // (heads // kv)
                (ck, sk, zk), (cv, sv, zv) = self.held
                o, l, tol, ltol = ref.attention(
                    qh[b, h], ck[slot, g], sk[slot, g], zk[slot, g],
                    cv[slot, g], sv[slot, g], zv[slot, g], scale,
                    self.bits[0], self.bits[1], kind)
                if len(slot) == 0:
                    assert (out[b, h] == 0).all() and lse[b, h] == -np.inf
                    continue
                off = np.abs(out[b, h] - o)
                worst = max(worst, float((off / np.maximum(tol, 1e-300)).max()))
                assert (off <= tol).all(), (b, h, n, off.max(), tol.min())
                assert abs(lse[b, h] - l) <= ltol, (b, h, n, lse[b, h], l)
        say("largest share of the tolerance: %.2f" % worst)
        return out, lse


def spread_tables(rng, lengths, page, pages, max_pages):
    """Tables of distinct pages in no order; places behind the last page hold
    a number that is no page."""
    table = np.full((len(lengths), max_pages), 10 ** 9, np.int32)
    free = list(rng.permutation(pages))
    for b, n in enumerate(lengths):
        for i in range(-(-n // page)):
            table[b, i] = free.pop()
    return torch.from_numpy(table).cuda()


def queries(rng, batch, heads, dim, kind):
    return rounded(rng.standard_normal((batch, heads, dim)), kind)[1]


# ---- write and read ---------------------------------------------------------

@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("dim", [16, 48, 64, 80, 128, 208, 256])
@pytest.mark.parametrize("kbits,vbits", [(8, 4), (4, 8)])
def test_write_bytes(kind, dim, kbits, vbits):
    """Codes and steps bit for bit; other rows keep their bytes."""
    say(kind, dim, kbits, vbits)
    rng = np.random.default_rng(dim + kbits)
    heads, page, pages, tokens = 3, 48, 5, 101
    cache = kc.empty(pages, heads, page, dim, kbits, vbits)
    for t in cache:
        t.view(torch.uint8).fill_(0xA5)
    x = [rng.standard_normal((tokens, heads, dim)) *
         np.exp(rng.uniform(-8, 8, (tokens, heads, 1))) +
         rng.choice([0, 0, 100, -3], (tokens, heads, 1)) for _ in range(2)]
    for a in x:
        a[1] = 0.0                                  # constant rows
        a[2] = 1.7
        a[3] = -1.7
        a[4] = np.round(a[4])                       # ties
        a[5, :, 0] = np.inf                         # what nobody wants
        a[6, :, 1] = -np.inf
        a[7, :, 2] = np.nan
        a[8] = 1e-30
        a[9] *= 1e-33
    (kh, k), (vh, v) = (rounded(a, kind) for a in x)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int32)
    slots[11:14] = [-1, pages * page, -2 ** 31]     # left out
    kc.write(k, v, torch.from_numpy(slots).cuda(), cache)
    torch.cuda.synchronize()
    at = (slots >= 0) & (slots < pages * page)
    for codes, steps, rows, bits in ((cache[0], cache[1], kh, kbits),
                                     (cache[2], cache[3], vh, vbits)):
        with np.errstate(all="ignore"):
            c, s, z = ref.quantize(rows, bits)
        want_c = np.full(codes.shape, 0xA5, np.uint8)
        want_s = np.full(steps.shape, 0xA5A5, np.uint16)
        p, o = slots[at] // page, slots[at] % page
        want_c[p, :, o] = ref.join_codes(c, bits)[at]
        want_s[p, :, o, 0] = (s[at].view(np.uint32) >> 16).astype(np.uint16)
        # (-0 and 0 are the same offset)
        want_s[p, :, o, 1] = ((z[at] + np.float32(0)).view(np.uint32) >>
                              16).astype(np.uint16)
        got_s = steps.view(torch.int16).cpu().numpy().view(np.uint16).copy()
        got_s[..., 1][got_s[..., 1] == 0x8000] = 0
        assert np.array_equal(codes.cpu().numpy(), want_c)
        assert np.array_equal(got_s, want_s)


@pytest.mark.parametrize("tokens", [1, 2, 63, 257, 5000])
@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_read_values(tokens, kind):
    """z + s c rounded once; any order, twice the same slot, none."""
    rng = np.random.default_rng(tokens)
    f = Filled(rng, 7, 3, 32, 80, 8, 4)
    slots = rng.integers(0, 7 * 32, tokens).astype(np.int32)
    if tokens > 2:
        slots[1], slots[2] = -1, 7 * 32
    k, v = kc.read(torch.from_numpy(slots).cuda(), f.cache, 80, DTYPE[kind])
    torch.cuda.synchronize()
    ok = (slots >= 0) & (slots < 7 * 32)
    for got, (c, s, z) in ((k, f.held[0]), (v, f.held[1])):
        want = np.zeros((tokens, 3, 80), np.float32)
        at = slots[ok]
        want[ok] = z[at][..., None] + s[at][..., None] * c[at].astype(
            np.float32)
        want = torch.from_numpy(want).to(DTYPE[kind])
        assert got.shape == want.shape and got.dtype == want.dtype
        assert torch.equal(got.cpu(), want)


def same_bytes(cache, x, bits):
    """The cache, its slots 0.. written with rows x, holds the definition's
    codes, steps and offsets (-0 and 0 are the same offset)."""
    with np.errstate(all="ignore"):
        c, s, z = ref.quantize(x, bits)
    n = len(x)
    for codes, steps in (cache[:2], cache[2:]):
        got = codes.transpose(1, 2).flatten(0, 1)[:n].cpu().numpy()
        assert np.array_equal(got, ref.join_codes(c, bits))
        got = steps.float().transpose(1, 2).flatten(0, 1)[:n].cpu().numpy()
        assert np.array_equal(got[..., 0], s)
        assert np.array_equal(got[..., 1], z)


@pytest.mark.parametrize("bits", [8, 4])
def test_write_every_step(bits):
    """Steps of every bfloat16 mantissa and of exponents from the smallest to
    the largest, with values next to the middle between two codes."""
    top = 2 ** bits - 1
    e = np.concatenate([np.arange(-60, -50), np.arange(-50, 110, 7),
                        np.arange(110, 118)])
    s = ((1 + np.arange(128) / 128) * 2.0 ** e[:, None]).ravel()
    part = (np.arange(14) + 0.5) * top / 14
    near = np.concatenate([[0.0, top - 0.25], np.floor(part) + 0.5 +
                           2.0 ** -18 * (np.arange(14) % 3 - 1)])
    x = (s[:, None] * near).astype(np.float32)[:, None]
    pages = len(x) // 64 + 1
    cache = kc.empty(pages, 1, 64, 16, bits, bits)
    k = torch.from_numpy(x).cuda()
    kc.write(k, k, torch.arange(len(x), dtype=torch.int32, device="cuda"),
             cache)
    same_bytes(cache, x, bits)
    assert len(np.unique(ref.quantize(x, bits)[1])) > 128 * (len(e) - 2)


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
def test_write_odd_values_among_others(kind):
    """NaN, infinities and the largest values, alone in a row of a wave, several
    that cancel in a sum, and rows whose sum overflows though none does."""
    rng = np.random.default_rng(3)
    big = 65504.0 if kind == "f16" else 3.0e38
    x = rng.standard_normal((60, 1, 48))
    x[3, 0, 40] = np.nan
    x[9, 0, 0], x[9, 0, 1] = np.inf, -np.inf
    x[14, 0, 7], x[14, 0, 6] = big, -big
    x[20] = big / 4
    x[25, 0, :24], x[25, 0, 24:] = big / 2, -big / 2
    x[33, 0, 47] = -np.inf
    x[41] = np.nan
    x[47] = np.inf
    xh, xd = rounded(x, kind)
    cache = kc.empty(4, 1, 16, 48, 8, 8)
    kc.write(xd, xd, torch.arange(60, dtype=torch.int32, device="cuda"), cache)
    same_bytes(cache, xh, 8)


@pytest.mark.parametrize("bits", [8, 4])
def test_values_within_half_a_step(bits):
    """A value is off by at most s / 2 and a few units of binary32 of the
    numbers added."""
    rng = np.random.default_rng(bits)
    x = rng.standard_normal((600, 2, 128)) * np.exp(
        rng.uniform(-20, 20, (600, 2, 1)))
    xh, xd = rounded(x, "f32")
    cache = kc.empty(10, 2, 64, 128, bits, bits)
    slots = torch.arange(600, dtype=torch.int32, device="cuda")
    kc.write(xd, xd, slots, cache)
    k, v = kc.read(slots, cache, 128)
    s = cache.k_steps[..., 0].float().transpose(1, 2).reshape(-1, 2, 1)[:600]
    big = np.abs(xh).max(-1, keepdims=True)
    off = np.abs(k.cpu().numpy().astype(np.float64) - xh)
    assert torch.equal(k, v)
    assert (off <= 0.5 * s.cpu().numpy() + 8 * 2.0 ** -24 * big).all()


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("tokens", [1, 40, 4100])
def test_write_from_slices_of_one_projection(kind, tokens):
    rng = np.random.default_rng(tokens)
    heads, dim = 4, 128
    x = rounded(rng.standard_normal((tokens, 4 + 2 * heads, dim)), kind)[1]
    q, k, v = x.split([4, heads, heads], 1)
    pages = tokens // 64 + 1
    a = kc.empty(pages, heads, 64, dim, 4, 8)
    b = kc.empty(pages, heads, 64, dim, 4, 8)
    for t in a + b:
        t.view(torch.uint8).zero_()
    slots = torch.randperm(pages * 64, device="cuda")[:tokens].int()
    kc.write(k, v, slots, a)
    kc.write(k.contiguous(), v.contiguous(), slots, b)
    for s, t in zip(a, b):
        assert torch.equal(s.view(torch.uint8), t.view(torch.uint8))


# ---- attention --------------------------------------------------------------

EDGES = [0, 1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 300, 513]


@pytest.mark.parametrize("kind", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("kbits,vbits", [(8, 8), (8, 4), (4, 8), (4, 4)])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_attend_lengths(kind, kbits, vbits, dim):
    """Lengths at the edges of halves, tiles, units and pages."""
    say(kind, kbits, vbits, dim)
    rng = np.random.default_rng(dim + 10 * kbits + vbits)
    pages = sum(-(-n // 48) for n in EDGES) + 2
    f = Filled(rng, pages, 2, 48, dim, kbits, vbits)
    table = spread_tables(rng, EDGES, 48, pages, 12)
    f.check(queries(rng, len(EDGES), 8, dim, kind), table,
            torch.tensor(EDGES, dtype=torch.int32, device="cuda"), kind=kind)


@pytest.mark.parametrize("dim", [16, 32, 48, 80, 96, 112, 144, 192, 208, 240])
@pytest.mark.parametrize("kbits,vbits", [(8, 4), (4, 8)])
@pytest.mark.parametrize("kind", ["f32", "f16"])
def test_attend_dims(dim, kbits, vbits, kind):
    say(dim, kbits, vbits, kind)
    rng = np.random.default_rng(dim + kbits)
    lengths = [5, 200, 37]
    f = Filled(rng, 20, 3, 16, dim, kbits, vbits)
    f.check(queries(rng, 3, 6, dim, kind),
            spread_tables(rng, lengths, 16, 20, 14),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            kind=kind)


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (3, 3), (7, 1), (15, 1),
                                            (16, 1), (17, 1), (40, 1),
                                            (34, 2), (64, 2), (12, 4)])
def test_attend_head_layouts(heads, kv_heads):
    """Shared heads: groups below, at and over the 16 columns of a tile."""
    say(heads, kv_heads)
    rng = np.random.default_rng(heads)
    lengths = [150, 20]
    f = Filled(rng, 8, kv_heads, 32, 64, 8, 4)
    f.check(queries(rng, 2, heads, 64, "bf16"),
            spread_tables(rng, lengths, 32, 8, 6),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            kind="bf16")


@pytest.mark.parametrize("window", [1, 5, 16, 17, 100, 128, 300, 1000])
@pytest.mark.parametrize("kbits,vbits", [(8, 8), (4, 4)])
def test_attend_window(window, kbits, vbits):
    rng = np.random.default_rng(window)
    lengths = [1, 16, 17, 100, 129, 333, 500]
    pages = sum(-(-n // 16) for n in lengths)
    f = Filled(rng, pages, 1, 16, 128, kbits, vbits)
    f.check(queries(rng, len(lengths), 4, 128, "f16"),
            spread_tables(rng, lengths, 16, pages, 32),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            window=window, kind="f16")


@pytest.mark.parametrize("kind", ["f32", "bf16"])
@pytest.mark.parametrize("batch,longest", [(1, 20000), (3, 7000), (40, 900)])
def test_attend_split_sequences(kind, batch, longest):
    """Long sequences beside short ones: ranges of units that begin and end
    inside sequences, and pages shared by sequences."""
    say(kind, batch, longest)
    rng = np.random.default_rng(batch)
    lengths = rng.integers(0, longest, batch)
    lengths[0] = longest
    pages = 120
    f = Filled(rng, pages, 2, 64, 64, 8, 8)
    table = rng.integers(0, pages, (batch, longest // 64 + 1)).astype(np.int32)
    f.check(queries(rng, batch, 4, 64, kind), torch.from_numpy(table).cuda(),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            kind=kind)


@pytest.mark.parametrize("kind", ["f32", "f16"])
@pytest.mark.parametrize("vbits", [8, 4])
def test_attend_weights_next_to_ties(kind, vbits):
    """96 Ki weights, some of which lie next to a tie of their first term's
    rounding: the two terms together are the weight all the same.  Logits are
    small, so that they add next to nothing to the bound."""
    say(kind, vbits)
    rng = np.random.default_rng(vbits)
    f = Filled(rng, 30, 2, 16, 64, 8, vbits)
    table = rng.integers(0, 30, (64, 3)).astype(np.int32)
    f.check(queries(rng, 64, 64, 64, kind), torch.from_numpy(table).cuda(),
            torch.full((64,), 24, dtype=torch.int32, device="cuda"),
            scale=2e-3, kind=kind)


@pytest.mark.parametrize("batch", [64, 65, 300, 4096, 4500])
def test_attend_many_sequences(batch):
    """More sequences than lanes of a wave, more than 64 for a lane; most of
    them short, some empty, one long enough for every way to be shared."""
    rng = np.random.default_rng(batch)
    lengths = rng.choice([0, 1, 7, 40, 200], batch)
    lengths[batch - 2] = 2600
    f = Filled(rng, 30, 1, 16, 16, 4, 4)
    table = rng.integers(0, 30, (batch, 163)).astype(np.int32)
    assert " shared " in kc.describe(30, 1, 16, 16, batch, 1, 163 * 16, 4, 4,
                                     dtype=torch.float16)
    f.check(queries(rng, batch, 1, 16, "f16"), torch.from_numpy(table).cuda(),
            torch.tensor(lengths, dtype=torch.int32, device="cuda"),
            kind="f16")


def test_attend_pages_and_lengths_out_of_range():
    """Tokens of entries that are no pages are not seen; lengths beyond
    max_len and below 0 count as the bounds."""
    rng = np.random.default_rng(8)
    f = Filled(rng, 9, 2, 16, 64, 8, 4)
    table = rng.integers(0, 9, (6, 20)).astype(np.int32)
    table[0, 3] = 9
    table[1, :] = -1
    table[2, 0], table[2, 1] = 2 ** 31 - 1, -2 ** 31
    table[3, 1::2] = 10 ** 6
    lengths = torch.tensor([300, 320, 40, 317, 10 ** 6, -5],
                           dtype=torch.int32, device="cuda")
    q = queries(rng, 6, 4, 64, "bf16")
    t = torch.from_numpy(table).cuda()
    f.check(q, t, lengths, kind="bf16")
    f.check(q, t, lengths, max_len=130, kind="bf16")
    f.check(q, t, lengths, max_len=100, window=33, kind="bf16")


def test_attend_values_that_are_hard():
    """Constant rows, huge and tiny rows, offsets far beyond the step, weights
    from one dominant token to thousands of equal ones."""
    rng = np.random.default_rng(10)
    n = 16 * 64
    k = rng.standard_normal((n, 1, 64))
    v = rng.standard_normal((n, 1, 64))
    v[:64] = 0.0
    v[64:128] = 3.25
    v[128:192] = 1000.0 + rng.standard_normal((64, 1, 64))
    v[192:256] *= 1e-12
    v[256:320] *= 1e9
    v[320:384] = 1e20
    k[384:448] = 0.0
    k[448:512] = 5.0
    k[512] *= 40.0
    f = Filled(rng, 64, 1, 16, 64, 8, 8, rows=[k, v])
    rows = [range(0, 4), range(4, 8), range(8, 12), range(12, 16),
            range(16, 20), range(20, 24), range(0, 12), range(24, 32),
            range(32, 64), range(12, 20), range(4, 24)]
    table = np.zeros((len(rows), 64), np.int32)
    for i, r in enumerate(rows):
        table[i, :len(r)] = list(r)
    lengths = torch.tensor([16 * len(r) for r in rows], dtype=torch.int32,
                           device="cuda")
    q = queries(rng, len(rows), 2, 64, "f32")
    q[:, 1] *= 30.0
    for kind in ("f32", "bf16"):
        f.check(q.to(DTYPE[kind]), torch.from_numpy(table).cuda(), lengths,
                kind=kind)


@pytest.mark.parametrize("kind,size", [("f32", 1e-30), ("f32", 1e25),
                                       ("bf16", 1e-30), ("bf16", 1e20),
                                       ("f16", 1e-4), ("f16", 3e4)])
def test_attend_query_sizes(kind, size):
    """Queries far from 1; the scale brings the logits back."""
    rng = np.random.default_rng(4)
    f = Filled(rng, 8, 1, 32, 64, 8, 8)
    q = rounded(rng.uniform(-1, 1, (2, 4, 64)) * size, kind)[1]
    table = torch.arange(8, dtype=torch.int32, device="cuda").view(2, 4)
    f.check(q, table, torch.tensor([100, 128], dtype=torch.int32,
                                   device="cuda"), scale=0.3 / size,
            kind=kind)


def test_attend_query_with_nan_or_infinity():
    """NaN for that head alone; a zero query gives the plain mean."""
    rng = np.random.default_rng(5)
    f = Filled(rng, 4, 2, 32, 64, 8, 4)
    q = queries(rng, 2, 8, 64, "bf16")
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    lengths = torch.tensor([50, 64], dtype=torch.int32, device="cuda")
    want, want_lse = f.check(q, table, lengths, kind="bf16")
    p = q.clone()
    p[0, 1, 3] = float("nan")
    p[1, 6, 0] = float("inf")
    out, lse = kc.attend(p, f.cache, table, lengths)
    out, lse = host(out), host(lse)
    bad = np.zeros((2, 8), bool)
    bad[0, 1] = bad[1, 6] = True
    assert np.isnan(out[bad]).all() and np.isnan(lse[bad]).all()
    assert np.array_equal(out[~bad], want[~bad])
    assert np.array_equal(lse[~bad], want_lse[~bad])
    q[1, 2] = 0.0
    f.check(q, table, lengths, kind="bf16")


def test_attend_strided_queries_scales_and_a_lone_row():
    rng = np.random.default_rng(6)
    f = Filled(rng, 6, 2, 32, 128, 4, 8)
    x = rounded(rng.standard_normal((3, 12, 128)), "f16")[1]
    table = torch.tensor([[0, 1], [2, 3], [4, 5]], dtype=torch.int32,
                         device="cuda")
    lengths = torch.tensor([64, 1, 40], dtype=torch.int32, device="cuda")
    for scale in (1.0, -0.2, 0.0):
        f.check(x[:, 4:8], table, lengths, scale=scale, kind="f16")
    f.check(x[1:2, 2:4], table[:1], lengths[:1], kind="f16")


def test_no_work_is_valid():
    f = Filled(np.random.default_rng(1), 2, 1, 16, 64, 8, 8)
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    empty = torch.empty((0, 1, 64), device="cuda")
    kc.write(empty, empty, none, f.cache)
    k, v = kc.read(none, f.cache, 64)
    assert k.shape == v.shape == (0, 1, 64)
    out, lse = kc.attend(empty, f.cache,
                         torch.empty((0, 0), dtype=torch.int32,
                                     device="cuda"), none)
    assert out.shape == (0, 1, 64) and lse.shape == (0, 1)


def test_rows_beyond_4_gib():
    """Slots and pages whose bytes lie over 2^32."""
    rng = np.random.default_rng(12)
    heads, page, dim = 4, 64, 256
    pages = (5 << 30) // (heads * page * dim)
    cache = kc.empty(pages, heads, page, dim, 8, 8)
    n = 3 * page
    kh, k = rounded(rng.standard_normal((n, heads, dim)), "bf16")
    vh, v = rounded(rng.standard_normal((n, heads, dim)), "bf16")
    use = [pages - 1, 0, pages // 2 + 3]
    slots = np.concatenate([p * page + np.arange(page) for p in use])
    dev = torch.from_numpy(slots.astype(np.int32)).cuda()
    kc.write(k, v, dev, cache)
    rk, rv = kc.read(dev, cache, dim)
    table = torch.tensor([use], dtype=torch.int32, device="cuda")
    q = queries(rng, 1, 8, dim, "bf16")
    out, lse = kc.attend(q, cache, table,
                         torch.tensor([n], dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    (ck, sk, zk), (cv, sv, zv) = ref.quantize(kh, 8), ref.quantize(vh, 8)
    assert np.array_equal(rk.cpu().numpy(), zk[..., None] + sk[..., None] *
                          ck.astype(np.float32))
    assert np.array_equal(rv.cpu().numpy(), zv[..., None] + sv[..., None] *
                          cv.astype(np.float32))
    out, lse = host(out), host(lse)
    for h in range(8):
        g = h // 2
        o, l, tol, ltol = ref.attention(host(q)[0, h], ck[:, g], sk[:, g],
                                        zk[:, g], cv[:, g], sv[:, g],
                                        zv[:, g], dim ** -0.5, 8, 8, "bf16")
        assert (np.abs(out[0, h] - o) <= tol).all()
        assert abs(lse[0, h] - l) <= ltol


# ---- together, streams, graphs ----------------------------------------------

def test_decoding_steps_together():
    """A prompt written in chunks, then tokens one by one: each step writes
    its rows and attends over all of them, itself included."""
    rng = np.random.default_rng(21)
    batch, heads, kv, dim, page, most = 3, 4, 2, 64, 16, 80
    cache = kc.empty(batch * (most // page), kv, page, dim, 8, 4)
    for t in cache:
        t.view(torch.uint8).fill_(0xFF)
    table_h = rng.permutation(batch * (most // page)).astype(np.int32)
    table_h = table_h.reshape(batch, -1)
    table = torch.from_numpy(table_h).cuda()
    kh, k = rounded(rng.standard_normal((batch, most, kv, dim)), "bf16")
    vh, v = rounded(rng.standard_normal((batch, most, kv, dim)), "bf16")
    held = [ref.quantize(kh, 8), ref.quantize(vh, 4)]
    prompt = [37, 5, 16]

    def slots_of(b, t):
        return table_h[b, t // page] * page + t % page

    for b, n in enumerate(prompt):
        for first in range(0, n, 20):
            t = np.arange(first, min(first + 20, n))
            kc.write(k[b, first:t[-1] + 1], v[b, first:t[-1] + 1],
                     torch.from_numpy(slots_of(b, t).astype(np.int32)).cuda(),
                     cache)
    for step in range(25):
        at = [n + step for n in prompt]
        slots = torch.tensor([slots_of(b, at[b]) for b in range(batch)],
                             dtype=torch.int32, device="cuda")
        row = torch.arange(batch, device="cuda")
        col = torch.tensor(at, device="cuda")
        kc.write(k[row, col], v[row, col], slots, cache)
        q = queries(rng, batch, heads, dim, "bf16")
        out, lse = kc.attend(q, cache, table, torch.tensor(
            [t + 1 for t in at], dtype=torch.int32, device="cuda"))
        out, lse, qh = host(out), host(lse), host(q)
        for b in range(batch):
            n = at[b] + 1
            for h in range(heads):
                g = h // 2
                (ck, sk, zk), (cv, sv, zv) = held
                o, l, tol, ltol = ref.attention(
                    qh[b, h], ck[b, :n, g], sk[b, :n, g], zk[b, :n, g],
                    cv[b, :n, g], sv[b, :n, g], zv[b, :n, g], dim ** -0.5, 8,
                    4, "bf16")
                assert (np.abs(out[b, h] - o) <= tol).all(), (step, b, h)
                assert abs(lse[b, h] - l) <= ltol


def test_repeated_calls_are_bit_identical():
    rng = np.random.default_rng(30)
    f = Filled(rng, 64, 2, 64, 128, 8, 8)
    table = torch.from_numpy(rng.integers(0, 64, (5, 64)).astype(np.int32))
    table = table.cuda()
    lengths = torch.tensor([4096, 3, 0, 1777, 640], dtype=torch.int32,
                           device="cuda")
    q = queries(rng, 5, 8, 128, "bf16")
    first = kc.attend(q, f.cache, table, lengths)
    for _ in range(5):
        again = kc.attend(q, f.cache, table, lengths)
        assert torch.equal(first[0], again[0])
        assert torch.equal(first[1], again[1])


def test_two_streams():
    """Calls in flight on two streams, each with outputs and workspace of its
    own."""
    rng = np.random.default_rng(31)
    f = Filled(rng, 64, 2, 64, 128, 4, 4)
    table = torch.from_numpy(rng.integers(0, 64, (2, 64)).astype(np.int32))
    table = table.cuda()
    lengths = [torch.tensor(n, dtype=torch.int32, device="cuda")
               for n in ([4096, 100], [2000, 4000])]
    q = [queries(rng, 2, 8, 128, "f16") for _ in range(2)]
    want = [kc.attend(q[i], f.cache, table, lengths[i]) for i in range(2)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = [kc.attend(q[i % 2], f.cache, table, lengths[i % 2],
                     stream=streams[i % 2]) for i in range(16)]
    torch.cuda.synchronize()
    for i, (out, lse) in enumerate(got):
        assert torch.equal(out, want[i % 2][0])
        assert torch.equal(lse, want[i % 2][1])


def test_steps_in_a_graph():
    """Write, attend and read captured and replayed with new rows, slots and
    lengths, eager calls in between; every replay against the eager result."""
    rng = np.random.default_rng(32)
    heads, kv, dim, page, batch, most = 8, 2, 128, 32, 4, 20
    f = Filled(rng, batch * most, kv, page, dim, 8, 4, kind="bf16")
    table = torch.from_numpy(rng.permutation(batch * most).reshape(
        batch, most).astype(np.int32)).cuda()
    k = torch.empty((batch, kv, dim), dtype=torch.bfloat16, device="cuda")
    v, q = torch.empty_like(k), queries(rng, batch, heads, dim, "bf16")
    slots = torch.zeros(batch, dtype=torch.int32, device="cuda")
    lengths = torch.zeros(batch, dtype=torch.int32, device="cuda")

    def fill(i):
        r = np.random.default_rng(100 + i)
        n = r.integers(1, most * page, batch)
        lengths.copy_(torch.from_numpy(n.astype(np.int32)))
        at = table.cpu().numpy()[np.arange(batch), (n - 1) // page]
        slots.copy_(torch.from_numpy((at * page + (n - 1) % page)
                                     .astype(np.int32)))
        for t in (k, v, q):
            t.copy_(torch.from_numpy(r.standard_normal(t.shape)))

    def step():
        kc.write(k, v, slots, f.cache)
        return kc.attend(q, f.cache, table, lengths) + kc.read(
            slots, f.cache, dim, torch.bfloat16)

    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(1, 6):
        fill(i)
        graph.replay()
        torch.cuda.synchronize()
        kept = [t.clone() for t in got]
        want = step()
        torch.cuda.synchronize()
        say("replay", i)
        for a, b in zip(kept, want):
            assert torch.equal(a, b)


def test_memory_around_the_outputs_stays():
    """The C entry points write their outputs and the workspace they asked for
    and nothing beside them."""
    import ctypes
    rng = np.random.default_rng(40)
    f = Filled(rng, 40, 3, 16, 80, 8, 4)
    batch, heads, dim = 5, 15, 80
    table = torch.from_numpy(rng.integers(0, 40, (batch, 30)).astype(
        np.int32)).cuda()
    lengths = torch.tensor([480, 0, 33, 129, 470], dtype=torch.int32,
                           device="cuda")
    q = queries(rng, batch, heads, dim, "f16")
    lib = kc.load_library()
    pages = kc._pages(f.cache, dim)[0]
    params = kc._PARAMS.pack(heads * dim, batch, heads, 30, 480, 0, 1,
                             dim ** -0.5)
    need = ctypes.c_int64()
    assert lib.bscache_attend_workspace(pages, params,
                                        ctypes.byref(need)) == kc.OK
    guard = 4096
    sizes = (batch * heads * dim * 2, batch * heads * 4, need.value)
    bufs = [torch.full((n + 2 * guard,), 0x5A, dtype=torch.uint8,
                       device="cuda") for n in sizes]
    at = [b.data_ptr() + guard for b in bufs]
    assert lib.bscache_attend(
        pages, params, q.data_ptr(), table.data_ptr(), lengths.data_ptr(),
        at[0], at[1], at[2], need.value,
        torch.cuda.current_stream().cuda_stream) == kc.OK
    torch.cuda.synchronize()
    for b, n in zip(bufs, sizes):
        assert (b[:guard] == 0x5A).all() and (b[guard + n:] == 0x5A).all()
    want, want_lse = f.check(q, table, lengths, kind="f16")
    got = bufs[0][guard:guard + sizes[0]].view(torch.float16)
    assert np.array_equal(host(got).reshape(want.shape), want)
    # without lse
    assert lib.bscache_attend(
        pages, params, q.data_ptr(), table.data_ptr(), lengths.data_ptr(),
        at[0], None, at[2], need.value,
        torch.cuda.current_stream().cuda_stream) == kc.OK
    torch.cuda.synchronize()
    assert np.array_equal(host(got).reshape(want.shape), want)


@pytest.mark.parametrize("batch,longest", [
    (1, 500), (1, 700),         # whole pairs of up to 4 units; shared ones
    (12, 700), (20, 1500),      # wide workgroups, and what is past their 4 steps
    (50, 1000), (60, 1100),     # pairs on every CU: whole up to 8 units
    (70, 2000), (70, 2100)])    # many pairs: whole up to 16
@pytest.mark.parametrize("dim,kind", [(64, "bf16"), (128, "f16"),
                                      (256, "bf16"), (96, "f32")])
def test_attend_on_both_sides_of_the_plan(batch, longest, dim, kind):
    """Ways of sharing a call out, each at its bounds: lengths up to the longest
    one, against float64 on the GPU."""
    say(batch, longest, dim, kind)
    gen = torch.Generator(device="cuda").manual_seed(batch + longest)
    kv, group, page = 8, 2, 32
    pages = 200
    cache = kc.empty(pages, kv, page, dim, 8, 4)
    k, v = (torch.randn((pages * page, kv, dim), generator=gen, device="cuda")
            for _ in range(2))
    kc.write(k, v, torch.arange(pages * page, dtype=torch.int32,
                                device="cuda"), cache)
    # rows as offset and rest: value = s c' + z', both float64
    rest, offset = [], []
    for x, steps, bits in zip(kc.read(torch.arange(
            pages * page, dtype=torch.int32, device="cuda"), cache, dim),
            (cache.k_steps, cache.v_steps), (8, 4)):
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
    out, lse = kc.attend(q, cache, table, lengths, max_len=longest)
    for b in range(batch):
        n = int(lengths[b])
        t = torch.arange(n, device="cuda")
        slot = table[b].long()[t // page] * page + t % page
        if n == 0:
            assert (out[b] == 0).all() and (lse[b] == -torch.inf).all()
            continue
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
        by_logit, by_weight, by_sum = ref.error_terms(kind, dim, n)
        d = float(size.max() * by_logit + x.abs().max() * 2.0 ** -21)
        spread = torch.matmul(p, vr.abs() + vz.abs()).view(kv * group, dim)
        tol = ref.STEP[kind] * want.abs() + \
            spread * (by_weight + 2 * d + by_sum)
        assert ((out[b].double() - want).abs() <= tol).all(), (b, n)
        total = torch.logsumexp(x, -1).view(-1)
        far = (lse[b].double() - total).abs()
        assert (far <= d + by_sum + 2.0 ** -22 * total.abs()).all(), (b, n)

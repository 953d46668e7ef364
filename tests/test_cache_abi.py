"""libbscache.so loads and validates arguments on the host (no GPU): every call
below fails validation or has nothing to do, so none reaches the HIP runtime;
the fake pointers are never dereferenced.  And the binding's own checks, and
the plain numpy definition that the GPU tests compare with."""
import ctypes
import os
import re
import types

import numpy as np
import pytest
import torch

from paper_1810_11066_amd import cache as kc
from tests import cache_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "bscache.h")

INVALID, UNSUPPORTED = kc.ERR_INVALID_ARG, kc.ERR_UNSUPPORTED
BASE = 1 << 40
# buffers far apart: keys' and values' codes and steps, then the others
KC, KS, VC, VS, A, B, C, D, E, F = (BASE + (i << 36) for i in range(10))


@pytest.fixture(scope="module")
def lib():
    return kc.load_library()


def pages(pages=10, heads=2, tokens=16, dim=64, kbits=8, vbits=4, kc_=KC,
          ks=KS, vc=VC, vs=VS):
    return kc._PAGES.pack(pages, heads, tokens, dim, kbits, vbits, kc_, ks,
                          vc, vs)


def params(stride=256, batch=3, heads=4, max_pages=5, max_len=80, window=0,
           dtype=1, scale=0.1):
    return kc._PARAMS.pack(stride, batch, heads, max_pages, max_len, window,
                           dtype, scale)


def write(lib, cache=None, k=A, v=B, ks=128, vs=128, dtype=1, slots=C,
          tokens=7):
    return lib.bscache_write(pages() if cache is None else cache, k, v, ks,
                             vs, dtype, slots, tokens, None)


def read(lib, cache=None, slots=A, tokens=7, k=B, v=C, dtype=1):
    return lib.bscache_read(pages() if cache is None else cache, slots,
                            tokens, k, v, dtype, None)


def attend(lib, cache=None, p=None, q=A, table=B, lengths=C, out=D, lse=E,
           space=F, size=1 << 30):
    return lib.bscache_attend(pages() if cache is None else cache,
                              params() if p is None else p, q, table, lengths,
                              out, lse, space, size, None)


def workspace(lib, cache=None, p=None):
    n = ctypes.c_int64(-1)
    st = lib.bscache_attend_workspace(pages() if cache is None else cache,
                                      params() if p is None else p,
                                      ctypes.byref(n))
    return st, n.value


def test_exports_every_declared_symbol(lib):
    text = re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)
    names = set(re.findall(r"\b(bscache_[a-z0-9_]+)\s*\(", text))
    assert names == set(kc.EXPORTED)
    for name in names:
        assert hasattr(lib, name), name
    assert lib.bscache_abi_version() == 100


CACHES = [
    (dict(pages=0), INVALID), (dict(pages=-1), INVALID),
    (dict(heads=0), INVALID), (dict(tokens=0), INVALID),
    (dict(dim=0), INVALID), (dict(dim=-16), INVALID),
    (dict(dim=24), UNSUPPORTED), (dict(dim=272), UNSUPPORTED),
    (dict(tokens=8), UNSUPPORTED), (dict(tokens=24), UNSUPPORTED),
    (dict(kbits=2), UNSUPPORTED), (dict(vbits=16), UNSUPPORTED),
    (dict(pages=1 << 28), UNSUPPORTED), (dict(heads=1 << 21), UNSUPPORTED),
]
POINTERS = [
    (dict(kc_=0), INVALID), (dict(ks=KS + 4), INVALID),
    (dict(vc=0), INVALID), (dict(vs=VS + 8), INVALID),
]


@pytest.mark.parametrize("change,status", CACHES + POINTERS)
def test_cache_validation(lib, change, status):
    cache = pages(**change)
    assert write(lib, cache) == status
    assert read(lib, cache) == status
    assert attend(lib, cache) == status
    assert lib.bscache_last_error() != b""
    if (change, status) in CACHES:
        assert workspace(lib, cache)[0] == status


def test_null_structs(lib):
    assert lib.bscache_write(None, A, B, 128, 128, 1, C, 1, None) == INVALID
    assert lib.bscache_read(None, A, 1, B, C, 1, None) == INVALID
    assert lib.bscache_attend(None, params(), A, B, C, D, E, F, 1 << 30,
                              None) == INVALID
    assert lib.bscache_attend(pages(), None, A, B, C, D, E, F, 1 << 30,
                              None) == INVALID
    assert lib.bscache_attend_workspace(pages(), params(), None) == INVALID


def test_write_validation(lib):
    for change in (dict(k=0), dict(v=0), dict(slots=0), dict(k=A + 2),
                   dict(slots=C + 4), dict(dtype=3), dict(dtype=-1),
                   dict(tokens=-1), dict(ks=127), dict(vs=120),
                   dict(ks=132), dict(ks=-128)):
        assert write(lib, **change) == INVALID, change
    assert write(lib, tokens=1 << 30) == UNSUPPORTED
    assert write(lib, ks=1 << 41) == UNSUPPORTED
    # k, v or the slots inside what is written; the cache over itself
    for at in (KC, KS, VC, VS):
        assert write(lib, k=at + 64) == INVALID
        assert write(lib, v=at + 64) == INVALID
        assert write(lib, slots=at + 64) == INVALID
    assert write(lib, k=KC - 128) == INVALID
    assert b"overlaps" in lib.bscache_last_error()
    assert write(lib, pages(vc=KC + 16)) == INVALID
    assert write(lib, tokens=0) == kc.OK
    assert lib.bscache_last_error() == b""


def test_read_validation(lib):
    for change in (dict(k=0), dict(v=0), dict(slots=0), dict(v=C + 2),
                   dict(dtype=3), dict(tokens=-1), dict(k=C), dict(k=A),
                   dict(v=KC), dict(k=VS + 16)):
        assert read(lib, **change) == INVALID, change
    assert read(lib, tokens=1 << 30) == UNSUPPORTED
    assert read(lib, tokens=0) == kc.OK


def test_attend_validation(lib):
    for change in (dict(batch=-1), dict(heads=0), dict(heads=3),
                   dict(max_pages=0), dict(max_len=0), dict(max_len=81),
                   dict(window=-1), dict(dtype=3), dict(stride=255),
                   dict(stride=260), dict(scale=float("inf")),
                   dict(scale=float("nan"))):
        assert attend(lib, p=params(**change)) == INVALID, change
        assert workspace(lib, p=params(**change))[0] == INVALID, change
    for change in (dict(q=0), dict(table=0), dict(lengths=0), dict(out=0),
                   dict(q=A + 8), dict(lse=E + 4), dict(out=A), dict(lse=D),
                   dict(out=KC), dict(lse=B), dict(out=C - 16)):
        assert attend(lib, **change) == INVALID, change
    big = params(batch=1 << 20, max_pages=1 << 16, max_len=1 << 20)
    assert workspace(lib, p=big)[0] == UNSUPPORTED
    assert workspace(lib, pages(heads=1), params(
        stride=1 << 18, batch=1 << 20, heads=1 << 12))[0] == UNSUPPORTED
    assert attend(lib, p=params(batch=0)) == kc.OK


def test_workspace(lib):
    """None where no sequence can be shared, otherwise as much as is said;
    too little is refused."""
    assert workspace(lib) == (kc.OK, 0)
    long = params(max_pages=100, max_len=1600)
    st, n = workspace(lib, p=long)
    assert st == kc.OK and n > 0
    assert attend(lib, p=long, size=n - 1) == INVALID
    assert attend(lib, p=long, space=0) == INVALID
    assert attend(lib, p=long, space=F + 8) == INVALID
    assert attend(lib, p=long, space=KC) == INVALID
    # it depends on what bounds the lengths, not on how long they may grow
    assert workspace(lib, p=params(max_pages=100, max_len=1600,
                                   window=100))[1] == 0
    most = [workspace(lib, p=params(batch=64, max_pages=m, max_len=16 * m))[1]
            for m in (1 << 10, 1 << 12, 1 << 13)]
    assert most[0] == most[1] == most[2]


# ---- the plan (256 compute units where there is no GPU) ---------------------

def plan(batch, max_len, kv_heads=8, dim=128, group=4, **kw):
    d = kc.describe(100, kv_heads, 32, dim, batch, kv_heads * group, max_len,
                    **kw)
    m = re.match(r"attend_kernel<(\d+), (\d), (\d), (\w+)> (\w+) grid=(\d+) "
                 r"waves=(\d+) workspace=(\d+)$", d)
    assert m, d
    return m.group(5), int(m.group(6)), int(m.group(7)), int(m.group(8))


@pytest.mark.parametrize("batch,max_len,way,grid,waves", [
    (1, 512, "whole", 8, 4), (1, 513, "shared", 40, 4),
    (1, 100000, "shared", 768, 4),
    # wide: pairs on a quarter of the CUs up to all, 5 units to 4 steps
    (7, 700, "shared", 336, 4), (8, 700, "wide", 64, 12),
    (8, 512, "whole", 64, 4), (8, 1536, "wide", 64, 12),
    (8, 1537, "shared", 768, 4), (32, 1024, "wide", 256, 12),
    # whole: 8 units with a pair for every CU, 16 with pairs for half of the
    # workgroups that run at once
    (33, 1024, "whole", 264, 4), (33, 1025, "shared", 768, 4),
    (47, 1025, "shared", 768, 4), (48, 1025, "whole", 384, 4),
    (48, 2048, "whole", 384, 4), (48, 2049, "shared", 768, 4)])
def test_plan_rules(batch, max_len, way, grid, waves):
    w, g, n, space = plan(batch, max_len)
    assert (w, g, n) == (way, grid, waves)
    # two partial results of 16 heads a workgroup, an entry for every pair
    assert space == (grid * 2 * 16 * (128 + 2) * 4 + 8 * 8 * batch
                     if way == "shared" else 0)


def test_plan_follows_registers_window_and_head_tiles():
    # waves of a wide workgroup are what the kernel's registers leave room for
    assert plan(16, 700, dim=64)[:3] == ("wide", 128, 16)
    assert plan(16, 700, dim=256)[:3] == ("wide", 128, 8)
    assert plan(16, 700, dtype=torch.float32)[:3] == ("wide", 128, 8)
    # (one workgroup of 4 waves is all that runs on a CU at once)
    assert plan(16, 700, dim=256, dtype=torch.float32)[:3] == ("whole", 128, 4)
    # a window bounds the span: its first token is taken down to a 16
    assert plan(1, 100000, window=497)[0] == "whole"
    assert plan(1, 100000, window=498)[0] == "shared"
    # 17 heads to a key-value head are two tiles
    assert plan(1, 512, group=16)[1] == 8
    assert plan(1, 512, group=17)[1] == 16


def test_describe_validation(lib):
    buf = ctypes.create_string_buffer(16)
    assert lib.bscache_attend_describe(pages(), params(), None, 16) == INVALID
    assert lib.bscache_attend_describe(pages(), params(), buf, 0) == INVALID
    assert lib.bscache_attend_describe(pages(dim=24), params(), buf,
                                       16) == UNSUPPORTED
    assert lib.bscache_attend_describe(pages(), params(), buf, 16) == kc.OK
    assert buf.value == b"attend_kernel<6"      # truncated


# ---- the binding ------------------------------------------------------------

def test_binding_refuses_host_tensors_and_types():
    host = kc.Pages(*(torch.zeros((2, 1, 16, n), dtype=t) for n, t in
                      ((64, torch.uint8), (2, torch.bfloat16)) * 2))
    x = torch.zeros((3, 1, 64))
    slots = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU tensor"):
        kc.write(x, x, slots, host)
    with pytest.raises(ValueError, match="GPU tensor"):
        kc.read(slots, host, 64)
    with pytest.raises(ValueError, match="GPU tensor"):
        kc.attend(x, host, slots.view(3, 1), slots)
    with pytest.raises(TypeError, match="dtype"):
        kc.read(slots, host, 64, torch.float64)
    with pytest.raises(ValueError, match="tokens, kv_heads, dim"):
        kc.write(x[0], x, slots, host)
    with pytest.raises(ValueError, match="batch, heads, dim"):
        kc.attend(x[0], host, slots, slots)
    with pytest.raises(ValueError, match="bits"):
        kc.empty(1, 1, 16, 64, 2, 8, "cpu")


def test_empty_shapes():
    c = kc.empty(3, 2, 32, 80, 8, 4, "cpu")
    assert c.k_codes.shape == (3, 2, 32, 80)
    assert c.v_codes.shape == (3, 2, 32, 40)
    assert c.k_steps.shape == c.v_steps.shape == (3, 2, 32, 2)
    assert c.k_codes.dtype == torch.uint8
    assert c.k_steps.dtype == torch.bfloat16


def fake(dtype=torch.float16, shape=(4, 2, 64), stride=None):
    """What _rows looks at, of a tensor on device 0."""
    t = torch.empty(shape, dtype=dtype)
    if stride is not None:
        t = torch.empty(10 ** 5, dtype=dtype).as_strided(shape, stride)

    class OnDevice(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 0
    return t.as_subclass(OnDevice)


def test_binding_strides():
    assert kc._rows(fake(), "k", 2, 64, 0) == (1, 128)
    assert kc._rows(fake(torch.bfloat16, stride=(512, 64, 1)), "k", 2, 64,
                    0) == (2, 512)
    # a lone token's stride says nothing
    assert kc._rows(fake(torch.float32, (1, 2, 64), (7, 64, 1)), "k", 2, 64,
                    0) == (0, 128)
    for stride in ((128, 65, 1), (128, 64, 2)):
        with pytest.raises(ValueError, match="lie together"):
            kc._rows(fake(stride=stride), "k", 2, 64, 0)
    with pytest.raises(ValueError, match="must be"):
        kc._rows(fake(), "k", 3, 64, 0)
    with pytest.raises(TypeError, match="float32"):
        kc._rows(fake(torch.float64), "k", 2, 64, 0)
    with pytest.raises(ValueError, match="cuda:1"):
        kc._rows(fake(), "k", 2, 64, 1)


def test_calls_run_on_the_tensors_device(monkeypatch):
    """A call for another device than the current one is made with that one
    current."""
    entered = []

    class Guard:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            entered.append(self.device)

        def __exit__(self, *a):
            entered.append("out")

    monkeypatch.setattr(kc, "_raw_device", lambda: 0)
    monkeypatch.setattr(kc, "_raw_stream", lambda d: 100 + d)
    monkeypatch.setattr(torch.cuda, "device", Guard)
    kc._call(0, lambda: kc.OK)
    assert entered == []
    kc._call(2, lambda: kc.OK)
    assert entered == [2, "out"]
    assert kc._stream(2) == 102
    monkeypatch.setattr(kc, "_raw_stream", None)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d:
                        types.SimpleNamespace(cuda_stream=1000 + d))
    assert kc._stream(3) == 1003


# ---- the numpy definition ---------------------------------------------------

def test_reference_rounds_to_bfloat16_towards_its_side():
    x = np.float32([1.0, 1.0 + 2.0 ** -8, -1.0 - 2.0 ** -20, 0.0, -0.0, 3e38,
                    1e-40])
    down, up = ref.bf16_down(x), ref.bf16_up(np.abs(x))
    assert (down <= x).all() and (up >= np.abs(x)).all()
    assert down[1] == 1.0 and up[1] == 1.0 + 2.0 ** -7
    assert down[2] == -1.0 - 2.0 ** -7
    for y in (down, up):
        assert (y.view(np.uint32) & 0xFFFF == 0).all()


@pytest.mark.parametrize("bits", [8, 4])
def test_reference_rows(bits):
    """Codes use their range, values stand within half a step."""
    rng = np.random.default_rng(bits)
    x = (rng.standard_normal((500, 64)) * np.exp(
        rng.uniform(-30, 30, (500, 1)))).astype(np.float32)
    x[0], x[1] = 0.0, -7.0
    c, s, z = ref.quantize(x, bits)
    v = z[:, None] + s[:, None] * c.astype(np.float64)
    off = np.abs(v - x)
    assert (off <= 0.5 * s[:, None] * (1 + 1e-5) +
            2.0 ** -22 * np.abs(x).max(-1, keepdims=True)).all()
    assert c[2:].max() == 2 ** bits - 1 or c[2:].max() == 2 ** bits - 2
    assert (ref.split_codes(ref.join_codes(c, bits), bits) == c).all()
    assert (v[0] == 0).all() and (v[1] == -7.0).all()


def test_reference_attention_is_the_softmax():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((40, 2, 16)).astype(np.float32)
    (ck, sk, zk), (cv, sv, zv) = (ref.quantize(x[:, i], 8) for i in (0, 1))
    q = rng.standard_normal(16)
    out, lse, tol, _ = ref.attention(q, ck, sk, zk, cv, sv, zv, 0.25, 8, 8,
                                     "f32")
    k = zk[:, None] + sk[:, None] * ck.astype(np.float64)
    v = zv[:, None] + sv[:, None] * cv.astype(np.float64)
    want = torch.softmax(torch.from_numpy(k @ q * 0.25), 0)
    assert np.allclose(out, want.numpy() @ v, rtol=1e-12, atol=1e-12)
    assert abs(lse - np.log(np.exp(k @ q * 0.25).sum())) < 1e-12
    assert (tol > 0).all() and (tol < 1e-4).all()


def test_binding_refuses_numbers_that_no_field_holds():
    for kw in ({"window": 1 << 40}, {"max_len": 1 << 31}, {"window": 1.5}):
        with pytest.raises(ValueError, match="32-bit"):
            kc.describe(4, 1, 16, 64, 1, 4, **{"max_len": 16, **kw})

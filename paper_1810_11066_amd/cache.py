"""Python binding of libbscache.so (include/bscache.h): a paged key-value
cache of 8- or 4-bit codes and the attention that reads it.

``write``, ``read`` and ``attend`` take torch tensors on the GPU, check them,
allocate the outputs (and the workspace) with torch and call the C entry point
on the current stream of the tensors' device, or on ``stream`` of that device
(which then owns the outputs' memory, as under ``torch.cuda.stream``).  Everything is
computed by the library's HIP kernels; there is no host fallback.

A cache is four tensors (``empty`` allocates them; any tuple of four does):

  k_codes, v_codes  uint8    [pages, kv_heads, page_tokens, dim * bits / 8]
  k_steps, v_steps  bfloat16 [pages, kv_heads, page_tokens, 2]

A row stands for z + s c with (s, z) its steps; the widths of keys and values
(8 or 4 bits each) are those of the last axes.  A token's slot is
page * page_tokens + its place in the page.
"""
from __future__ import annotations

import ctypes
import functools
import operator
import os
import struct
import threading
from typing import NamedTuple, Optional, Tuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
# BSCACHE_LIBRARY selects another build of the same library
LIB_PATH = os.environ.get("BSCACHE_LIBRARY",
                          os.path.join(_HERE, "libbscache.so"))

OK = 0
ERR_INVALID_ARG = 1
ERR_UNSUPPORTED = 2
ERR_HIP = 4

EXPORTED = ("bscache_write", "bscache_read", "bscache_attend",
            "bscache_attend_workspace", "bscache_attend_describe",
            "bscache_last_error", "bscache_abi_version")

# bscache_dtype
_DTYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}


class CacheError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("bscache status %d: %s" % (status, msg))
        self.status = status


class Pages(NamedTuple):
    """The four tensors of a cache."""
    k_codes: torch.Tensor
    k_steps: torch.Tensor
    v_codes: torch.Tensor
    v_steps: torch.Tensor


# bscache_pages and bscache_attend_params as bytes (natural alignment)
_PAGES = struct.Struct("@q5i4xPPPP")
_PARAMS = struct.Struct("@q6if4x")

_lock = threading.Lock()
_lib = None


def load_library():
    """Load libbscache.so (built in-tree by paper_1810_11066_amd.build)."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libbscache.so is not built (%s); run "
                "`python -m paper_1810_11066_amd.build`" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        P, S = ctypes.c_void_p, ctypes.c_char_p      # S: a packed struct
        i64, ci = ctypes.c_int64, ctypes.c_int
        sig = {
            "bscache_write": (ci, [S, P, P, i64, i64, ci, P, i64, P]),
            "bscache_read": (ci, [S, P, i64, P, P, ci, P]),
            "bscache_attend_workspace": (ci, [S, S, ctypes.POINTER(i64)]),
            "bscache_attend_describe": (ci, [S, S, P, ctypes.c_int32]),
            "bscache_attend": (ci, [S, S, P, P, P, P, P, P, i64, P]),
            "bscache_last_error": (ctypes.c_char_p, []),
            "bscache_abi_version": (ci, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def _refuse_numbers(values, e):
    raise ValueError("batch, heads, max_pages, max_len and window must be "
                     "32-bit integers, scale a binary32 number (got %s)"
                     % (values,)) from e


def _params(*values) -> bytes:
    """Packed bscache_attend_params."""
    try:
        return _PARAMS.pack(*values)
    except (struct.error, OverflowError) as e:
        _refuse_numbers(values[1:6] + values[7:], e)


def _integer(x) -> int:
    """An integer of any kind (a tensor's, say, as it is now) as an int."""
    try:
        return operator.index(x)
    except TypeError as e:
        _refuse_numbers(x, e)


def _check(status: int):
    if status != OK:
        raise CacheError(status, load_library().bscache_last_error().decode())


# ---- tensors ----------------------------------------------------------------

try:
    _raw_stream = torch._C._cuda_getCurrentRawStream
    _raw_device = torch._C._cuda_getDevice
except AttributeError:          # not public names: they may go
    _raw_stream = _raw_device = None


def _stream(device: int) -> int:
    """Handle of the device's current stream."""
    if _raw_stream is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device)


def _under(stream, cache):
    """The context in which `stream` is the current one, of the cache's device."""
    t = cache[0]
    device = t.get_device() if isinstance(t, torch.Tensor) else -1
    if device >= 0 and stream.device.index != device:
        raise ValueError("the stream is of %s, the cache on cuda:%d"
                         % (stream.device, device))
    return torch.cuda.stream(stream)


def _call(device: int, fn, *args) -> None:
    """The C call with the tensors' device as the current one."""
    current = torch.cuda.current_device() if _raw_device is None \
        else _raw_device()
    if current == device:
        status = fn(*args)
    else:
        with torch.cuda.device(device):
            status = fn(*args)
    if status != OK:
        _check(status)


def _refuse(t, name: str, dtype, dims: int, device: int):
    """Raises what is wrong with a tensor that should be a contiguous one of
    the given type and rank on `device`."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if not t.is_cuda:
        raise ValueError("%s must be a GPU tensor (got %s)" % (name, t.device))
    if t.get_device() != device:
        raise ValueError("%s is on %s, the cache on cuda:%d"
                         % (name, t.device, device))
    if t.dtype != dtype:
        raise TypeError("%s must be %s (got %s)" % (name, dtype, t.dtype))
    if t.dim() != dims:
        raise ValueError("%s must have %d axes (got %s)"
                         % (name, dims, tuple(t.shape)))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)


def _int32(t, name: str, dims: int, device: int):
    """Shape of a contiguous int32 tensor on `device`."""
    if not (isinstance(t, torch.Tensor) and t.dtype is torch.int32
            and t.get_device() == device and t.is_contiguous()
            and t.dim() == dims):
        _refuse(t, name, torch.int32, dims, device)
    return t.shape


def _rows(t, name: str, heads: int, dim: int, device: int):
    """(dtype number, token stride in elements) of [tokens][heads][dim] rows
    whose tokens may lie apart."""
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    kind = _DTYPES.get(t.dtype)
    if kind is None:
        raise TypeError("%s must be float32, float16 or bfloat16 (got %s)"
                        % (name, t.dtype))
    if t.get_device() != device:
        raise ValueError("%s is on %s, the cache on cuda:%d"
                         % (name, t.device, device))
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError("%s must be [tokens, %d, %d] (got %s)"
                         % (name, heads, dim, tuple(shape)))
    s0, s1, s2 = t.stride()
    if (s2 != 1 and dim > 1) or (s1 != dim and heads > 1):
        raise ValueError("%s: a token's heads and channels must lie together "
                         "(strides %s)" % (name, (s0, s1, s2)))
    # a lone token has no distance to a next one
    return kind, s0 if shape[0] > 1 else heads * dim


def _pages(cache, dim: int):
    """(packed bscache_pages, kv_heads, page_tokens, device) of a cache whose
    rows have `dim` channels."""
    kc, ks, vc, vs = cache
    # all of it at once; what is wrong is looked for only if something is
    try:
        device = kc.get_device()
        pages, heads, tokens, k_row = shape = kc.shape
        v_row = vc.shape[3]
        good = (device >= 0 and kc.dtype is torch.uint8
                and vc.dtype is torch.uint8 and ks.dtype is torch.bfloat16
                and vs.dtype is torch.bfloat16 and ks.get_device() == device
                and vc.get_device() == device and vs.get_device() == device
                and kc.is_contiguous() and ks.is_contiguous()
                and vc.is_contiguous() and vs.is_contiguous()
                and ks.shape == (pages, heads, tokens, 2) == vs.shape
                and (k_row == v_row and vc.shape == shape
                     or vc.shape == (pages, heads, tokens, v_row))
                and dim >= 1 and k_row * 8 % dim == 0 == v_row * 8 % dim)
    except (AttributeError, IndexError, ValueError):
        good = False
    if not good:
        _refuse_cache(cache, dim)
    return _PAGES.pack(pages, heads, tokens, dim, k_row * 8 // dim,
                       v_row * 8 // dim, kc.data_ptr(), ks.data_ptr(),
                       vc.data_ptr(), vs.data_ptr()), heads, tokens, device


def _refuse_cache(cache, dim: int):
    """Raises what is wrong with a cache."""
    device = cache[0].get_device() if isinstance(cache[0], torch.Tensor) else 0
    for t, name, dtype in zip(cache, Pages._fields,
                              (torch.uint8, torch.bfloat16) * 2):
        _refuse(t, name, dtype, 4, device)
    k_codes, k_steps, v_codes, v_steps = cache
    if (v_codes.shape[:3] != k_codes.shape[:3]
            or k_steps.shape != k_codes.shape[:3] + (2,)
            or v_steps.shape != k_steps.shape):
        raise ValueError("the cache's tensors differ in pages, heads or "
                         "tokens: %s" % [tuple(t.shape) for t in cache])
    raise ValueError("codes of %d and %d bytes do not hold rows of %d channels"
                     % (k_codes.shape[3], v_codes.shape[3], dim))


@functools.lru_cache(maxsize=1024)
def _workspace(device: int, pages: int, kv_heads: int, page_tokens: int,
               dim: int, batch: int, heads: int, max_pages: int, max_len: int,
               window: int, dtype: int) -> int:
    """Bytes that bscache_attend_workspace asks for: of the sizes alone, and
    the device's compute units."""
    need = ctypes.c_int64()
    cache = _PAGES.pack(pages, kv_heads, page_tokens, dim, 8, 8, 0, 0, 0, 0)
    params = _params(heads * dim, batch, heads, max_pages, max_len, window,
                     dtype, 1.0)
    _call(device, load_library().bscache_attend_workspace, cache, params,
          ctypes.byref(need))
    return need.value


# ---- the operators ----------------------------------------------------------

def empty(pages: int, kv_heads: int, page_tokens: int, dim: int,
          kbits: int = 8, vbits: int = 8, device="cuda") -> Pages:
    """An uninitialised cache of `pages` pages of `page_tokens` tokens."""
    def side(bits):
        if bits not in (4, 8):
            raise ValueError("bits must be 8 or 4 (got %s)" % (bits,))
        shape = (pages, kv_heads, page_tokens)
        return (torch.empty(shape + (dim * bits // 8,), dtype=torch.uint8,
                            device=device),
                torch.empty(shape + (2,), dtype=torch.bfloat16,
                            device=device))
    return Pages(*(side(kbits) + side(vbits)))


def write(k: torch.Tensor, v: torch.Tensor, slots: torch.Tensor, cache,
          stream: Optional[torch.cuda.Stream] = None) -> None:
    """Quantize the rows of new tokens into the cache (bscache_write).

    k, v: [tokens, kv_heads, dim] float32, float16 or bfloat16; tokens may lie
    apart (slices of a projection's output).  slots: [tokens] int32; a token
    whose slot is outside the cache (-1) is left out; no slot twice."""
    if stream is not None:
        with _under(stream, cache):
            return write(k, v, slots, cache)
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise ValueError("k must be a [tokens, kv_heads, dim] tensor")
    dim = k.shape[2]
    pages, heads, _, device = _pages(cache, dim)
    kind, k_stride = _rows(k, "k", heads, dim, device)
    v_kind, v_stride = _rows(v, "v", heads, dim, device)
    tokens, = _int32(slots, "slots", 1, device)
    if v_kind != kind:
        raise TypeError("k is %s, v %s" % (k.dtype, v.dtype))
    if k.shape[0] != tokens or v.shape[0] != tokens:
        raise ValueError("%d keys, %d values and %d slots"
                         % (k.shape[0], v.shape[0], tokens))
    if tokens == 0:
        return
    _call(device, (_lib or load_library()).bscache_write, pages, k.data_ptr(),
          v.data_ptr(), k_stride, v_stride, kind, slots.data_ptr(), tokens,
          _stream(device))


def read(slots: torch.Tensor, cache, dim: int, dtype=torch.float32,
         stream: Optional[torch.cuda.Stream] = None
         ) -> Tuple[torch.Tensor, torch.Tensor]:
    """The keys and values that the rows of `slots` stand for, each
    [tokens, kv_heads, dim] of `dtype` (bscache_read); zeros for a slot
    outside the cache."""
    if stream is not None:
        with _under(stream, cache):         # the outputs are this stream's
            return read(slots, cache, dim, dtype)
    kind = _DTYPES.get(dtype)
    if kind is None:
        raise TypeError("dtype must be float32, float16 or bfloat16 (got %s)"
                        % (dtype,))
    pages, heads, _, device = _pages(cache, dim)
    tokens, = _int32(slots, "slots", 1, device)
    k = torch.empty(tokens, heads, dim, dtype=dtype, device=slots.device)
    v = torch.empty_like(k)
    if tokens:
        _call(device, (_lib or load_library()).bscache_read, pages,
              slots.data_ptr(), tokens, k.data_ptr(), v.data_ptr(), kind,
              _stream(device))
    return k, v


def attend(q: torch.Tensor, cache, table: torch.Tensor, lengths: torch.Tensor,
           scale: Optional[float] = None, window: int = 0,
           max_len: Optional[int] = None,
           stream: Optional[torch.cuda.Stream] = None
           ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of one new token of each sequence over its cached tokens
    (bscache_attend): (out, lse).

    q: [batch, heads, dim]; table: [batch, max_pages] int32 page numbers;
    lengths: [batch] int32; scale: of the logits (default dim ** -0.5);
    window: only the last `window` tokens are visible (0: all); max_len: no
    sequence is longer (default: what the table has room for) -- a close bound
    saves workgroups that find nothing to do.  out is like q, lse float32
    [batch, heads]; a sequence without visible tokens gets 0 and -inf."""
    if stream is not None:
        with _under(stream, cache):         # outputs and workspace too
            return attend(q, cache, table, lengths, scale, window, max_len)
    if not isinstance(q, torch.Tensor) or q.dim() != 3:
        raise ValueError("q must be a [batch, heads, dim] tensor")
    batch, heads, dim = q.shape
    pages, kv_heads, page_tokens, device = _pages(cache, dim)
    kind, q_stride = _rows(q, "q", heads, dim, device)
    rows, max_pages = _int32(table, "table", 2, device)
    if rows != batch or _int32(lengths, "lengths", 1, device)[0] != batch:
        raise ValueError("%d queries, %d rows of the table and %d lengths"
                         % (batch, rows, lengths.shape[0]))
    out = torch.empty_like(q, memory_format=torch.contiguous_format)
    lse = torch.empty(batch, heads, dtype=torch.float32, device=q.device)
    if batch == 0:
        return out, lse
    if max_len is None:
        max_len = min(max_pages * page_tokens, 2 ** 31 - 1)
    elif type(max_len) is not int:
        max_len = _integer(max_len)
    if type(window) is not int:
        window = _integer(window)
    need = _workspace(device, cache[0].shape[0], kv_heads, page_tokens, dim,
                      batch, heads, max_pages, max_len, window, kind)
    space = torch.empty(need, dtype=torch.uint8, device=q.device) if need \
        else None
    _call(device, (_lib or load_library()).bscache_attend, pages,
          _params(q_stride, batch, heads, max_pages, max_len, window, kind,
                  dim ** -0.5 if scale is None else scale),
          q.data_ptr(), table.data_ptr(), lengths.data_ptr(), out.data_ptr(),
          lse.data_ptr(), space.data_ptr() if need else None, need,
          _stream(device))
    return out, lse


def describe(pages: int, kv_heads: int, page_tokens: int, dim: int,
             batch: int, heads: int, max_len: int, kbits: int = 8,
             vbits: int = 8, window: int = 0, dtype=torch.bfloat16) -> str:
    """Kernel and launch that attend would use for these sizes (host only)."""
    kind = _DTYPES.get(dtype)
    if kind is None:
        raise TypeError("dtype must be float32, float16 or bfloat16 (got %s)"
                        % (dtype,))
    numbers = pages, kv_heads, page_tokens, dim, kbits, vbits
    try:
        cache = _PAGES.pack(*numbers, 0, 0, 0, 0)
    except struct.error as e:
        raise ValueError("pages must be a 64-bit integer, kv_heads, page_tokens, "
                         "dim, kbits and vbits 32-bit ones (got %s)"
                         % (numbers,)) from e
    # (no page holds a token where page_tokens is none: refused below)
    max_pages = -(-max_len // page_tokens) if page_tokens else 1
    buf = ctypes.create_string_buffer(256)
    _check(load_library().bscache_attend_describe(
        cache, _params(heads * dim, batch, heads, max_pages, max_len, window,
                       kind, 1.0), buf, 256))
    return buf.value.decode()

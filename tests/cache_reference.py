"""The cache's definition in plain numpy: rows in binary32 steps as the header
fixes them, attention in 64 bits, and how far a call may be off it."""
import numpy as np

F32 = np.float32
STEP = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}


def bf16_down(x):
    b = np.ascontiguousarray(x, F32).view(np.uint32).astype(np.int64)
    cut = b & 0xFFFF0000
    cut = np.where((cut != b) & (b >> 31 == 1), cut + 0x10000, cut)
    return cut.astype(np.uint32).view(F32)


def bf16_up(x):                                  # of x >= 0
    b = np.ascontiguousarray(x, F32).view(np.uint32).astype(np.int64)
    cut = b & 0xFFFF0000
    return np.where(cut != b, cut + 0x10000, cut).astype(np.uint32).view(F32)


def quantize(x, bits):
    """(codes, s, z) of float32 rows x: codes one to a byte."""
    top = F32(2 ** bits - 1)
    x = np.asarray(x, F32)
    x = np.where(np.isnan(x), F32(0), x)
    x = np.clip(x, F32(-2.0 ** 126), F32(2.0 ** 126)).astype(F32)
    z = bf16_down(x.min(-1, keepdims=True))
    part = ((x.max(-1, keepdims=True) - z).astype(F32) * (F32(1) / top))
    s = np.maximum(bf16_up(part.astype(F32)), F32(2.0 ** -60))
    t = ((x - z).astype(F32) * (F32(1) / s)).astype(F32)
    c = np.minimum(np.rint(t), top).astype(np.uint8)
    return c, s[..., 0], z[..., 0]


def join_codes(c, bits):
    """Codes as the cache's bytes."""
    return c if bits == 8 else c[..., 0::2] | c[..., 1::2] << 4


def split_codes(b, bits):
    if bits == 8:
        return b
    return np.stack([b & 15, b >> 4], -1).reshape(b.shape[:-1] + (-1,))


def error_terms(kind, dim, tokens):
    """(binary32 roundings of a logit's magnitudes, relative error of a weight
    times s, relative error of a sum over tokens) that a call may have.

    A logit is s (q . c') + z' sum q, z' = z + centre s, with the codes c' = c -
    centre (centre 0 for 16-bit calls, 128 or 8 for float32).  Its dim products
    are added in binary32, in the matrix unit's order: at most dim roundings of
    2^-24 of the magnitudes added, and 16 for the rest of the expression;
    16-bit calls multiply subnormals of 8 bits, which lie up to 2 bits below
    what the unit aligns them as, so 4 times that.  A float32 query is kept to
    22 bits.  A weight times s is kept to 11 bits for bfloat16 calls, to 22 for
    the others.  Tokens accumulate in binary32: at most tokens / 32 + 64
    roundings in a row (again 4 times for subnormals), and what is below the
    smallest float16 of a weight, 2^-30 of the largest."""
    unit = 2.0 ** -24
    wide = 1 if kind == "f32" else 4
    logit = wide * unit * (dim + 16) + (2.0 ** -22 if kind == "f32" else 0.0)
    weight = 2.0 ** -11 if kind == "bf16" else 2.0 ** -22
    return logit, weight, wide * unit * (tokens / 32 + 64) + 2.0 ** -30


def centre(kind, bits):
    return 0 if kind != "f32" else 128 if bits == 8 else 8


def attention(q, c_k, s_k, z_k, c_v, s_v, z_v, scale, kbits, vbits, kind):
    """One head: q [dim], codes [tokens][dim], steps [tokens]; (out, lse, how
    far out may be off, how far lse may be off), all float64.  A logit off by d
    moves a weight by a factor e^d; both the sum and the total move."""
    q = q.astype(np.float64)
    dim = q.size
    if len(s_k) == 0:
        return np.zeros(dim), -np.inf, np.zeros(dim), 0.0
    ck, cv = c_k.astype(np.float64), c_v.astype(np.float64)
    s_k, z_k = s_k.astype(np.float64)[:, None], z_k.astype(np.float64)[:, None]
    s_v, z_v = s_v.astype(np.float64)[:, None], z_v.astype(np.float64)[:, None]
    mk, mv = centre(kind, kbits), centre(kind, vbits)
    k, v = z_k + s_k * ck, z_v + s_v * cv
    logit = scale * (k @ q)
    top = logit.max()
    p = np.exp(logit - top)
    total = p.sum()
    out = p @ v / total
    lse = top + np.log(total)
    size = abs(scale) * (s_k[:, 0] * (np.abs(ck - mk) @ np.abs(q)) +
                         np.abs(z_k + mk * s_k)[:, 0] * np.abs(q).sum())
    by_logit, by_weight, by_sum = error_terms(kind, dim, len(p))
    unit = 2.0 ** -24
    d = size.max() * by_logit + np.abs(logit).max() * 8 * unit
    spread = p @ (s_v * np.abs(cv - mv) + np.abs(z_v + mv * s_v)) / total
    tol = STEP[kind] * np.abs(out) + spread * (by_weight + 2 * d + by_sum)
    return out, lse, tol, d + by_sum + 4 * unit * abs(lse)

// extern "C" entry points of libbscache.so (declared in include/bscache.h)
// and the kernels that write a cache's rows and read them back.  Every check
// runs on the host before anything is enqueued.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>

#include "bscache.h"
#include "cache_internal.h"

namespace bscache {
namespace {

// ---------------------------------------------------------------------------
// Rows.  LPR lanes (a power of two, at least dim / 8) share a row, 8
// consecutive channels each, so a wave has 64 / LPR rows at a time: rows of
// consecutive tokens for one head of the keys or of the values.  Consecutive
// tokens of a prompt lie side by side in a page, so a wave's codes go to one
// stretch of memory (4-bit rows are narrower than a cache line).  STEPS such
// groups follow each other, with all their loads in flight first.

// Full reduction over the LPR lanes of a row with DPP moves: xor 1, xor 2,
// then mirrors of 8 and of 16 lanes, which reach the other half whatever the
// order in it, and one LDS permutation for 32.
template <int CTRL>
__device__ __forceinline__ float dpp(float v) {
    return __builtin_bit_cast(
        float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), CTRL, 0xF,
                                        0xF, true));
}
template <int LPR, class F>
__device__ __forceinline__ float reduce_row(float v, F f) {
    if constexpr (LPR >= 2) v = f(v, dpp<0xB1>(v));     // quad_perm 1,0,3,2
    if constexpr (LPR >= 4) v = f(v, dpp<0x4E>(v));     // quad_perm 2,3,0,1
    if constexpr (LPR >= 8) v = f(v, dpp<0x141>(v));    // row_half_mirror
    if constexpr (LPR >= 16) v = f(v, dpp<0x140>(v));   // row_mirror
    if constexpr (LPR >= 32) v = f(v, __shfl_xor(v, 16));
    return v;
}

// x as the quantizer takes it: 0 for NaN, within +-kBig.  The smaller and the
// larger of two such values as medians with a bound (v_med3_f32): after a DPP
// move fminf and fmaxf take an instruction more each, which quiets NaNs that
// are not there.
constexpr float kBig = 0x1p126f;
__device__ __forceinline__ float finite(float x) {
    return __builtin_amdgcn_fmed3f(x == x ? x : 0.0f, -kBig, kBig);
}
__device__ __forceinline__ float smaller(float a, float b) {
    return __builtin_amdgcn_fmed3f(a, b, -kBig);
}
__device__ __forceinline__ float larger(float a, float b) {
    return __builtin_amdgcn_fmed3f(a, b, kBig);
}

// 1 / s, rounded to nearest, of a bfloat16 s of 2^-60 to 2^124.  v_rcp_f32 is within
// an ulp, so e = 1 - s r is below 2^-22 and exact (8 bits times 24), and r + e r
// is 1 / s but for e^2, 2^-21 of an ulp, and its own rounding; 1 / s itself is
// a power of two or, s having 8 bits, 1/510 of an ulp or more from a tie.  (The
// division takes 10 instructions, this 3.)
__device__ __forceinline__ float reciprocal(float s) {
    const float r = __builtin_amdgcn_rcpf(s);
    return __builtin_fmaf(__builtin_fmaf(-s, r, 1.0f), r, r);
}

// Smallest and largest of 8 values.
__device__ __forceinline__ void extremes(const float (&x)[8], float& lo,
                                         float& hi) {
    lo = hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
    }
}

// Which rows a wave has: all tokens of a stretch for one (head, side).
struct RowsGrid {
    int64_t tokens;
    uint32_t groups;      // stretches of (64 / LPR) * STEPS tokens
    uint32_t waves;       // groups * kv_heads * 2
    FastDiv by_pairs;     // by kv_heads * 2
};

// The side (0 keys, 1 values), head and first token of a wave.
__device__ __forceinline__ bool wave_rows(const RowsGrid& g, int per,
                                          int& side, int& head,
                                          int64_t& first) {
    const uint32_t w = __builtin_amdgcn_readfirstlane(
        (blockIdx.x * kBlock + threadIdx.x) >> 6);
    if (w >= g.waves) return false;
    const uint32_t group = g.by_pairs.div(w);
    const uint32_t pair = w - group * g.by_pairs.d;
    side = pair & 1;
    head = pair >> 1;
    first = (int64_t)group * per;
    return true;
}

// Codes of 8 values: fl32(fl32(x - z) * inv) rounded half to even, as bytes
// (v_cvt_pk_u8_f32).  The clamp of the definition never binds: x >= z, and
// (x - z) inv <= (2^B - 1) (1 + 2^-21), which rounds to 2^B - 1.
__device__ __forceinline__ u32x2 codes8(const float (&x)[8], float z,
                                        float inv) {
    u32x2 d = {0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        d[i >> 2] = __builtin_amdgcn_cvt_pk_u8_f32((x[i] - z) * inv, i & 3,
                                                   d[i >> 2]);
    return d;
}
// the low halves of 4 bytes as 2 bytes
__device__ __forceinline__ uint32_t nibbles(uint32_t d) {
    d = (d | d >> 4) & 0x00FF00FFu;
    return (d | d >> 8) & 0xFFFFu;
}

// the four nibbles of the low 2 bytes as 4 bytes
__device__ __forceinline__ uint32_t spread(uint32_t w) {
    w = (w & 0xFFu) | (w & 0xFF00u) << 8;
    return (w | w << 4) & 0x0F0F0F0Fu;
}

// Values read back go past the caches (non-temporal stores): they push out
// nothing that is read sooner (16384 tokens of 8 heads of 128 in 17.1
// us, 24.3 without; 100000 in 108 and 118).
template <class V>
__device__ __forceinline__ void stream(V* p, V v) {
    __builtin_nontemporal_store(v, p);
}

// Bound by memory, and next by the vector ALUs (about 120 instructions for 8
// channels a lane: 16 bytes of float16): 100000 tokens of 8 heads of 128, 570
// MB, in 116 us = 4.9 TB/s.  Codes are stored the ordinary way: past the
// caches a write by itself takes 0 to 5 us less (60000 tokens of 8 heads of 64
// 36.9 for 41.3 us), but the read or the attention that comes next finds them in
// the caches (write and read of those together 66.6 us, 75.5 past the caches; of
// 16384 tokens of 4-bit codes, 128 channels 32.4 and 37.4).  NaN and infinities
// are looked for in a sum, and the values mended in the waves that have any; that
// and the short reciprocal took those 16384 tokens from 20.4 to 17.9 us.
template <int T, int LPR, int STEPS>
__global__ __launch_bounds__(kBlock) void write_kernel(
    Pages c, const void* __restrict__ k, const void* __restrict__ v,
    int64_t k_stride, int64_t v_stride, const int32_t* __restrict__ slots,
    RowsGrid g) {
    constexpr int kRows = 64 / LPR;
    int side, head;
    int64_t first;
    if (!wave_rows(g, kRows * STEPS, side, head, first)) return;
    const int lane = threadIdx.x & 63;
    const int part = lane % LPR, channel = part * 8;
    const bool mine = channel < c.dim;
    const void* src = side ? v : k;
    const int64_t stride = side ? v_stride : k_stride;
    const int bits = c.bits[side];
    const float per = bits == 8 ? 1.0f / 255.0f : 1.0f / 15.0f;
    uint32_t slot[STEPS];
    Eight<T> in[STEPS];
    const int64_t t0 = first + lane / LPR;
    int64_t at = t0 * stride + (int64_t)head * c.dim + channel;
#pragma unroll
    for (int s = 0; s < STEPS; ++s, at += kRows * stride) {
        const int64_t t = t0 + s * kRows;
        slot[s] = t < g.tokens ? (uint32_t)slots[t] : ~0u;
        if (t < g.tokens && mine) in[s].load(src, at);
        else in[s].clear();
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        float x[8], lo, hi, sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = in[s].get(i);
            sum += x[i];
        }
        extremes(x, lo, hi);
        // a NaN or an infinity among the values shows in their sum (finite
        // values' may show too: they come out as they were)
        const bool odd = !(fabsf(sum) <= kBig) ||
                         (T != kF16 && !(fmaxf(hi, -lo) <= kBig));
        if (__any(odd)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = finite(x[i]);
            extremes(x, lo, hi);
        }
        if (!mine) lo = kBig, hi = -kBig;
        lo = reduce_row<LPR>(lo, smaller);
        hi = reduce_row<LPR>(hi, larger);
        // z down to bfloat16 (towards zero by dropping the low half, one
        // step on where that went up), s up
        const uint32_t lb = f32_bits(lo), lcut = lb & 0xFFFF0000u;
        const uint32_t zb = lcut + (lcut != lb && (lb >> 31) ? 0x10000u : 0u);
        const float z = bits_f32(zb);
        const uint32_t rb = f32_bits((hi - z) * per), rcut = rb & 0xFFFF0000u;
        // (not negative: bits compare as the values do)
        const uint32_t sb = max(rcut + (rcut != rb ? 0x10000u : 0u),
                                f32_bits(0x1p-60f));
        const float inv = reciprocal(bits_f32(sb));
        if (slot[s] < c.slots && mine) {
            const uint32_t page = c.by_page.div(slot[s]);
            const int64_t row =
                row_of(c, page, head, slot[s] - page * c.by_page.d);
            const u32x2 d = codes8(x, z, inv);
            uint8_t* codes = c.codes[side];
            if (bits == 8)
                *reinterpret_cast<u32x2*>(codes + row * c.dim + channel) = d;
            else
                *reinterpret_cast<uint32_t*>(codes + row * (c.dim >> 1) +
                                             (channel >> 1)) =
                    nibbles(d[0]) | nibbles(d[1]) << 16;
            if (part == 0) c.steps[side][row] = sb >> 16 | zb;
        }
    }
}

// Bound by memory: 100000 tokens of 8 heads of 128, 570 MB, in 108 us = 5.3 TB/s,
// what a copy reaches.  (Nothing looks at a code before all of a wave's loads are
// sent: 4-bit ones spread where they are loaded took 121 us.)
//
// A lane's codes are two times 4 channels: next to each other where the values
// are written as one 16-byte store of 16 bits each, LPR lanes apart where they
// are float32, so that a store of 4 of them leaves no gap between the lanes.
template <int T, int LPR, int STEPS>
__global__ __launch_bounds__(kBlock) void read_kernel(
    Pages c, const int32_t* __restrict__ slots, void* __restrict__ k,
    void* __restrict__ v, RowsGrid g) {
    constexpr int kRows = 64 / LPR;
    constexpr int kApart = T == kF32 ? 4 * LPR : 4;
    int side, head;
    int64_t first;
    if (!wave_rows(g, kRows * STEPS, side, head, first)) return;
    const int lane = threadIdx.x & 63;
    const int channel = lane % LPR * (T == kF32 ? 4 : 8);
    const int bits = c.bits[side];
    const uint8_t* codes = c.codes[side];
    uint32_t slot[STEPS], d[STEPS][2], sz[STEPS];
    const int64_t t0 = first + lane / LPR;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int64_t t = t0 + s * kRows;
        slot[s] = t < g.tokens ? (uint32_t)slots[t] : ~0u;
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        d[s][0] = d[s][1] = sz[s] = 0;     // a slot outside the cache: 0 + 0 c
        if (slot[s] < c.slots && channel < c.dim) {
            const uint32_t page = c.by_page.div(slot[s]);
            const int64_t row = row_of(c, page, head,
                                       slot[s] - page * c.by_page.d);
            sz[s] = c.steps[side][row];
            const uint8_t* p = codes + row * (c.dim * bits >> 3) +
                               (channel * bits >> 3);
            if constexpr (T == kF32) {
                const bool both = channel + kApart < c.dim;
                if (bits == 8) {
                    d[s][0] = *reinterpret_cast<const uint32_t*>(p);
                    if (both)
                        d[s][1] = *reinterpret_cast<const uint32_t*>(p + kApart);
                } else {
                    d[s][0] = *reinterpret_cast<const uint16_t*>(p);
                    if (both)
                        d[s][1] =
                            *reinterpret_cast<const uint16_t*>(p + kApart / 2);
                }
            } else if (bits == 8) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p);
                d[s][0] = w[0], d[s][1] = w[1];
            } else {
                d[s][0] = *reinterpret_cast<const uint32_t*>(p);
            }
        }
    }
    void* dst = side ? v : k;
    int64_t at = (t0 * c.kv_heads + head) * c.dim + channel;
#pragma unroll
    for (int s = 0; s < STEPS; ++s, at += (int64_t)kRows * c.kv_heads * c.dim) {
        if (t0 + s * kRows >= g.tokens || channel >= c.dim) continue;
        const float step = step_of(sz[s]), z = offset_of(sz[s]);
        if (bits == 4) {    // (not sooner: it waits for the codes)
            if constexpr (T != kF32) d[s][1] = d[s][0] >> 16;
            d[s][0] = spread(d[s][0]);
            d[s][1] = spread(d[s][1]);
        }
        float x[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float code = (float)(d[s][i >> 2] >> 8 * (i & 3) & 255u);
            x[i] = z + code * step;      // the product is exact
        }
        if constexpr (T == kF32) {
            float* p = static_cast<float*>(dst) + at;
            stream(reinterpret_cast<f32x4*>(p),
                   f32x4{x[0], x[1], x[2], x[3]});
            if (channel + kApart < c.dim)
                stream(reinterpret_cast<f32x4*>(p + kApart),
                       f32x4{x[4], x[5], x[6], x[7]});
        } else {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
            stream(reinterpret_cast<u32x4*>(static_cast<uint16_t*>(dst) + at),
                   w);
        }
    }
}

// fn<T, LPR, STEPS>(args) for the run-time type, row width and stretch.
template <template <int, int, int> class F, int T, int LPR, class... A>
hipError_t pick_steps(int steps, A... a) {
    return steps == 2 ? F<T, LPR, 2>::go(a...) : F<T, LPR, 1>::go(a...);
}
template <template <int, int, int> class F, int T, class... A>
hipError_t pick_lpr(int lpr, int steps, A... a) {
    switch (lpr) {
        case 2: return pick_steps<F, T, 2>(steps, a...);
        case 4: return pick_steps<F, T, 4>(steps, a...);
        case 8: return pick_steps<F, T, 8>(steps, a...);
        case 16: return pick_steps<F, T, 16>(steps, a...);
        default: return pick_steps<F, T, 32>(steps, a...);
    }
}
template <template <int, int, int> class F, class... A>
hipError_t pick(int dtype, int lpr, int steps, A... a) {
    switch (dtype) {
        case kF32: return pick_lpr<F, kF32>(lpr, steps, a...);
        case kF16: return pick_lpr<F, kF16>(lpr, steps, a...);
        default: return pick_lpr<F, kBF16>(lpr, steps, a...);
    }
}

template <int T, int LPR, int STEPS>
struct Write {
    static hipError_t go(const Pages& c, const void* k, const void* v,
                         int64_t ks, int64_t vs, const int32_t* slots,
                         RowsGrid g, hipStream_t st) {
        return launch(write_kernel<T, LPR, STEPS>, (g.waves + 3) / 4, kBlock,
                      st, c, k, v, ks, vs, slots, g);
    }
};
template <int T, int LPR, int STEPS>
struct Read {
    static hipError_t go(const Pages& c, const int32_t* slots, void* k,
                         void* v, RowsGrid g, hipStream_t st) {
        return launch(read_kernel<T, LPR, STEPS>, (g.waves + 3) / 4, kBlock,
                      st, c, slots, k, v, g);
    }
};

int lanes_of_row(const Pages& c) {
    int lpr = 2;
    while (lpr * 8 < c.dim) lpr *= 2;
    return lpr;
}

// Lanes of a row, groups of a wave and grid of a call: two groups once the waves
// of single ones are more than `full` on a SIMD.
RowsGrid rows_grid(const Pages& c, int64_t tokens, int full, int* lpr,
                   int* steps) {
    *lpr = lanes_of_row(c);
    const int rows = 64 / *lpr;
    const int64_t pairs = 2 * (int64_t)c.kv_heads;
    *steps = (tokens + rows - 1) / rows * pairs >
                     (int64_t)device_cus() * 4 * full ? 2 : 1;
    RowsGrid g;
    g.tokens = tokens;
    g.groups = (uint32_t)((tokens + rows * *steps - 1) / (rows * *steps));
    g.waves = (uint32_t)(g.groups * pairs);
    g.by_pairs.init((uint32_t)pairs);
    return g;
}

}  // namespace

int device_cus() {
    constexpr int kDevices = 16;
    static int cus[kDevices];          // 0: not asked yet
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= kDevices)
        return 256;
    int n = __atomic_load_n(&cus[dev], __ATOMIC_RELAXED);
    if (n == 0) {
        if (hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount,
                                  dev) != hipSuccess || n < 1)
            n = 256;
        __atomic_store_n(&cus[dev], n, __ATOMIC_RELAXED);
    }
    return n;
}

bool rows_fit(const Pages& c, int64_t tokens) {
    // (so many come two groups to a wave)
    const int64_t per = 2 * (64 / lanes_of_row(c));
    return (tokens + per - 1) / per * 2 * c.kv_heads <=
           kBlock / 64 * kMostBlocks;
}

hipError_t launch_write(const Pages& c, const void* k, const void* v,
                        int64_t k_stride, int64_t v_stride, int dtype,
                        const int32_t* slots, int64_t tokens,
                        hipStream_t st) {
    int lpr, steps;
    // (8 heads of 128 to 8 bits, 8192 tokens, 32 waves a SIMD: 11.4 us single,
    // 12.1 in twos; 16384: 24.3 and 23.2; to 4 bits 19.6 and 17.8)
    const RowsGrid g = rows_grid(c, tokens, 32, &lpr, &steps);
    return pick<Write>(dtype, lpr, steps, c, k, v, k_stride, v_stride, slots,
                       g, st);
}

hipError_t launch_read(const Pages& c, const int32_t* slots, int64_t tokens,
                       void* k, void* v, int dtype, hipStream_t st) {
    int lpr, steps;
    // (1024 tokens of 8 heads of 128, 4 waves a SIMD: 3.4 us single, 3.5 in
    // twos; 2048: 4.1 and 3.9; 8192: 10.3 and 9.9; 100000: 139 and 108)
    const RowsGrid g = rows_grid(c, tokens, 7, &lpr, &steps);
    return pick<Read>(dtype, lpr, steps, c, slots, k, v, g, st);
}

}  // namespace bscache

// ---- entry points ----------------------------------------------------------

namespace {

thread_local char g_err[512];

bscache_status fail(bscache_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

bscache_status ok() {
    g_err[0] = '\0';
    return BSCACHE_OK;
}

bscache_status from_hip(hipError_t e, const char* what) {
    if (e == hipSuccess) return ok();
    return fail(BSCACHE_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
}

bscache_status check_ptr(const void* p, const char* name) {
    if (!p) return fail(BSCACHE_ERR_INVALID_ARG, "%s is NULL", name);
    if ((uintptr_t)p & 15u)
        return fail(BSCACHE_ERR_INVALID_ARG, "%s is not 16-byte aligned",
                    name);
    return BSCACHE_OK;
}

// A buffer of a call; outputs must not share a byte with any other buffer.
struct Range {
    const void* p;
    uint64_t bytes;
    const char* name;
};

bscache_status check_disjoint(const Range* out, int outs, const Range* in,
                              int ins) {
    for (int i = 0; i < outs; ++i)
        for (int j = i + 1; j < outs + ins; ++j) {
            const Range& a = out[i];
            const Range& b = j < outs ? out[j] : in[j - outs];
            if (a.bytes && b.bytes && (uintptr_t)a.p < (uintptr_t)b.p + b.bytes &&
                (uintptr_t)b.p < (uintptr_t)a.p + a.bytes)
                return fail(BSCACHE_ERR_INVALID_ARG, "%s overlaps %s", a.name,
                            b.name);
        }
    return BSCACHE_OK;
}

// Sizes and pointers of a cache; fills the kernels' view and the four buffers.
bscache_status check_cache(const bscache_pages* p, bscache::Pages* c,
                           Range* range, bool pointers) {
    if (!p) return fail(BSCACHE_ERR_INVALID_ARG, "cache is NULL");
    if (p->pages < 1 || p->kv_heads < 1 || p->page_tokens < 1 || p->dim < 1)
        return fail(BSCACHE_ERR_INVALID_ARG, "sizes must be >= 1");
    if (p->dim % 16 != 0 || p->dim > 256)
        return fail(BSCACHE_ERR_UNSUPPORTED,
                    "dim = %d is not a multiple of 16 up to 256", p->dim);
    if (p->page_tokens % 16 != 0)
        return fail(BSCACHE_ERR_UNSUPPORTED,
                    "page_tokens = %d is not a multiple of 16",
                    p->page_tokens);
    if ((p->kbits != 8 && p->kbits != 4) || (p->vbits != 8 && p->vbits != 4))
        return fail(BSCACHE_ERR_UNSUPPORTED, "kbits = %d, vbits = %d: 8 or 4",
                    p->kbits, p->vbits);
    if (p->pages > INT32_MAX / p->page_tokens)
        return fail(BSCACHE_ERR_UNSUPPORTED, "more than 2^31 - 1 slots");
    if (p->kv_heads > (1 << 20))
        return fail(BSCACHE_ERR_UNSUPPORTED, "more than 2^20 kv_heads");
    const uint64_t rows =
        (uint64_t)p->pages * p->kv_heads * (uint64_t)p->page_tokens;
    if (pointers) {
        bscache_status st;
        if ((st = check_ptr(p->k_codes, "k_codes")) != BSCACHE_OK) return st;
        if ((st = check_ptr(p->k_steps, "k_steps")) != BSCACHE_OK) return st;
        if ((st = check_ptr(p->v_codes, "v_codes")) != BSCACHE_OK) return st;
        if ((st = check_ptr(p->v_steps, "v_steps")) != BSCACHE_OK) return st;
        range[0] = {p->k_codes, rows * p->dim * p->kbits / 8, "k_codes"};
        range[1] = {p->k_steps, rows * 4, "k_steps"};
        range[2] = {p->v_codes, rows * p->dim * p->vbits / 8, "v_codes"};
        range[3] = {p->v_steps, rows * 4, "v_steps"};
    }
    c->codes[0] = p->k_codes;
    c->codes[1] = p->v_codes;
    c->steps[0] = reinterpret_cast<uint32_t*>(p->k_steps);
    c->steps[1] = reinterpret_cast<uint32_t*>(p->v_steps);
    c->pages = (uint32_t)p->pages;
    c->kv_heads = p->kv_heads;
    c->page_tokens = p->page_tokens;
    c->dim = p->dim;
    c->bits[0] = p->kbits;
    c->bits[1] = p->vbits;
    c->slots = (uint32_t)(p->pages * p->page_tokens);
    c->by_page.init((uint32_t)p->page_tokens);
    return BSCACHE_OK;
}

bscache_status check_dtype(int dtype) {
    if (dtype != BSCACHE_F32 && dtype != BSCACHE_F16 && dtype != BSCACHE_BF16)
        return fail(BSCACHE_ERR_INVALID_ARG, "unknown dtype %d", dtype);
    return BSCACHE_OK;
}

int64_t size_of(int dtype) { return dtype == BSCACHE_F32 ? 4 : 2; }

bscache_status check_stride(int64_t stride, int64_t least, int dtype,
                            const char* name) {
    if (stride < least)
        return fail(BSCACHE_ERR_INVALID_ARG, "%s = %lld is below a row's %lld",
                    name, (long long)stride, (long long)least);
    if (stride % (16 / size_of(dtype)) != 0)
        return fail(BSCACHE_ERR_INVALID_ARG,
                    "%s = %lld is not of whole 16 bytes", name,
                    (long long)stride);
    if (stride > ((int64_t)1 << 40))
        return fail(BSCACHE_ERR_UNSUPPORTED, "%s beyond 2^40", name);
    return BSCACHE_OK;
}

// Bytes from the first element of strided rows to the last.
uint64_t strided_bytes(int64_t rows, int64_t stride, int64_t row, int dtype) {
    return rows < 1 ? 0 : ((uint64_t)(rows - 1) * stride + row) * size_of(dtype);
}

bscache_status check_tokens(int64_t tokens, const bscache::Pages& c) {
    if (tokens < 0) return fail(BSCACHE_ERR_INVALID_ARG, "tokens < 0");
    if (tokens > INT32_MAX / (2 * (int64_t)c.kv_heads) ||
        !bscache::rows_fit(c, tokens))
        return fail(BSCACHE_ERR_UNSUPPORTED,
                    "%lld tokens have more rows than a launch has lanes for",
                    (long long)tokens);
    return BSCACHE_OK;
}

}  // namespace

extern "C" {

int bscache_abi_version(void) { return 100; }

const char* bscache_last_error(void) { return g_err; }

bscache_status bscache_write(const bscache_pages* cache, const void* k,
                             const void* v, int64_t k_stride,
                             int64_t v_stride, bscache_dtype dtype,
                             const int32_t* slots, int64_t tokens,
                             bscache_stream_t stream) {
    bscache_status st;
    bscache::Pages c;
    Range out[4];
    if ((st = check_cache(cache, &c, out, true)) != BSCACHE_OK) return st;
    if ((st = check_dtype((int)dtype)) != BSCACHE_OK) return st;
    if ((st = check_ptr(k, "k")) != BSCACHE_OK) return st;
    if ((st = check_ptr(v, "v")) != BSCACHE_OK) return st;
    if ((st = check_ptr(slots, "slots")) != BSCACHE_OK) return st;
    if ((st = check_tokens(tokens, c)) != BSCACHE_OK) return st;
    const int64_t row = (int64_t)c.kv_heads * c.dim;
    if ((st = check_stride(k_stride, row, dtype, "k_stride")) != BSCACHE_OK)
        return st;
    if ((st = check_stride(v_stride, row, dtype, "v_stride")) != BSCACHE_OK)
        return st;
    if (tokens == 0) return ok();
    const Range in[3] = {
        {k, strided_bytes(tokens, k_stride, row, dtype), "k"},
        {v, strided_bytes(tokens, v_stride, row, dtype), "v"},
        {slots, (uint64_t)tokens * 4, "slots"}};
    if ((st = check_disjoint(out, 4, in, 3)) != BSCACHE_OK) return st;
    return from_hip(bscache::launch_write(c, k, v, k_stride, v_stride,
                                          (int)dtype, slots, tokens,
                                          (hipStream_t)stream),
                    "bscache_write launch");
}

bscache_status bscache_read(const bscache_pages* cache, const int32_t* slots,
                            int64_t tokens, void* k, void* v,
                            bscache_dtype dtype, bscache_stream_t stream) {
    bscache_status st;
    bscache::Pages c;
    Range in[5];
    if ((st = check_cache(cache, &c, in, true)) != BSCACHE_OK) return st;
    if ((st = check_dtype((int)dtype)) != BSCACHE_OK) return st;
    if ((st = check_ptr(slots, "slots")) != BSCACHE_OK) return st;
    if ((st = check_ptr(k, "k")) != BSCACHE_OK) return st;
    if ((st = check_ptr(v, "v")) != BSCACHE_OK) return st;
    if ((st = check_tokens(tokens, c)) != BSCACHE_OK) return st;
    if (tokens == 0) return ok();
    in[4] = {slots, (uint64_t)tokens * 4, "slots"};
    const int64_t row = (int64_t)c.kv_heads * c.dim;
    const Range out[2] = {{k, strided_bytes(tokens, row, row, dtype), "k"},
                          {v, strided_bytes(tokens, row, row, dtype), "v"}};
    if ((st = check_disjoint(out, 2, in, 5)) != BSCACHE_OK) return st;
    return from_hip(bscache::launch_read(c, slots, tokens, k, v, (int)dtype,
                                         (hipStream_t)stream),
                    "bscache_read launch");
}

// Checks of an attention call's sizes; fills the kernels' view and the launch.
static bscache_status check_attend(const bscache_pages* cache,
                                   const bscache_attend_params* p,
                                   bscache::Attend* a, Range* range,
                                   bool pointers, int64_t* workspace) {
    bscache_status st;
    if ((st = check_cache(cache, &a->c, range, pointers)) != BSCACHE_OK)
        return st;
    if (!p) return fail(BSCACHE_ERR_INVALID_ARG, "params is NULL");
    if ((st = check_dtype(p->dtype)) != BSCACHE_OK) return st;
    if (p->batch < 0) return fail(BSCACHE_ERR_INVALID_ARG, "batch < 0");
    if (p->heads < 1 || p->max_pages < 1 || p->max_len < 1)
        return fail(BSCACHE_ERR_INVALID_ARG, "sizes must be >= 1");
    if (p->heads % a->c.kv_heads != 0)
        return fail(BSCACHE_ERR_INVALID_ARG,
                    "heads = %d is not a multiple of kv_heads = %d", p->heads,
                    a->c.kv_heads);
    if ((int64_t)p->max_len > (int64_t)p->max_pages * a->c.page_tokens)
        return fail(BSCACHE_ERR_INVALID_ARG,
                    "max_len = %d is beyond the %d pages of the table",
                    p->max_len, p->max_pages);
    if (p->window < 0) return fail(BSCACHE_ERR_INVALID_ARG, "window < 0");
    if (!isfinite(p->scale))
        return fail(BSCACHE_ERR_INVALID_ARG, "scale is not finite");
    if ((st = check_stride(p->q_stride, (int64_t)p->heads * a->c.dim, p->dtype,
                           "q_stride")) != BSCACHE_OK)
        return st;
    a->q_stride = p->q_stride;
    a->batch = p->batch;
    a->heads = p->heads;
    a->group = p->heads / a->c.kv_heads;
    a->head_tiles = (a->group + 15) / 16;
    a->max_pages = p->max_pages;
    a->max_len = p->max_len;
    a->window = p->window;
    a->dtype = p->dtype;
    a->scale = p->scale;
    // units of the longest sequence: its first visible token is taken down
    // to a multiple of 16
    int64_t span = p->max_len;
    if (p->window > 0 && (int64_t)p->window + 15 < span)
        span = (int64_t)p->window + 15;
    const int64_t units = (span + bscache::kUnit - 1) / bscache::kUnit;
    const int64_t pairs = (int64_t)a->c.kv_heads * a->head_tiles;
    if (p->batch * pairs > bscache::kMostBlocks)
        return fail(BSCACHE_ERR_UNSUPPORTED,
                    "%lld pairs of a sequence and up to 16 query heads: 2^24 or "
                    "more", (long long)(p->batch * pairs));
    if (p->batch * pairs > INT32_MAX / (2 * (units + 8)) ||
        (int64_t)p->batch * p->heads > INT32_MAX)
        return fail(BSCACHE_ERR_UNSUPPORTED,
                    "more than 2^30 units of 128 tokens, or 2^31 - 1 rows");
    bscache::plan_attend(*a, span);
    *workspace = a->workspace;
    return BSCACHE_OK;
}

bscache_status bscache_attend_workspace(const bscache_pages* cache,
                                        const bscache_attend_params* p,
                                        int64_t* bytes) {
    if (!bytes) return fail(BSCACHE_ERR_INVALID_ARG, "bytes is NULL");
    bscache::Attend a;
    const bscache_status st = check_attend(cache, p, &a, nullptr, false, bytes);
    return st == BSCACHE_OK ? ok() : st;
}

bscache_status bscache_attend_describe(const bscache_pages* cache,
                                       const bscache_attend_params* p,
                                       char* buf, int32_t len) {
    if (!buf || len < 1) return fail(BSCACHE_ERR_INVALID_ARG, "buf/len");
    buf[0] = '\0';
    bscache::Attend a;
    int64_t bytes;
    const bscache_status st =
        check_attend(cache, p, &a, nullptr, false, &bytes);
    if (st != BSCACHE_OK) return st;
    const int dp = bscache::padded_dim(a.c.dim);
    snprintf(buf, (size_t)len,
             "attend_kernel<%d, %d, %d, %s> %s grid=%d waves=%d workspace=%lld",
             dp, a.c.bits[0], a.c.bits[1],
             a.dtype == bscache::kF32   ? "f32"
             : a.dtype == bscache::kF16 ? "f16"
                                        : "bf16",
             a.wide ? "wide" : a.whole ? "whole" : "shared", a.blocks,
             bscache::group_waves(dp, a.dtype, a.wide), (long long)bytes);
    return ok();
}

bscache_status bscache_attend(const bscache_pages* cache,
                              const bscache_attend_params* p, const void* q,
                              const int32_t* table, const int32_t* lengths,
                              void* out, float* lse, void* workspace,
                              int64_t workspace_bytes,
                              bscache_stream_t stream) {
    bscache_status st;
    bscache::Attend a;
    Range in[7];
    int64_t need;
    if ((st = check_attend(cache, p, &a, in, true, &need)) != BSCACHE_OK)
        return st;
    if ((st = check_ptr(q, "q")) != BSCACHE_OK) return st;
    if ((st = check_ptr(table, "table")) != BSCACHE_OK) return st;
    if ((st = check_ptr(lengths, "lengths")) != BSCACHE_OK) return st;
    if ((st = check_ptr(out, "out")) != BSCACHE_OK) return st;
    if (lse && (st = check_ptr(lse, "lse")) != BSCACHE_OK) return st;
    if (need > 0) {
        if ((st = check_ptr(workspace, "workspace")) != BSCACHE_OK) return st;
        if (workspace_bytes < need)
            return fail(BSCACHE_ERR_INVALID_ARG,
                        "workspace of %lld bytes, %lld needed",
                        (long long)workspace_bytes, (long long)need);
    }
    if (p->batch == 0) return ok();
    const int64_t row = (int64_t)p->heads * a.c.dim;
    in[4] = {q, strided_bytes(p->batch, p->q_stride, row, p->dtype), "q"};
    in[5] = {table, (uint64_t)p->batch * p->max_pages * 4, "table"};
    in[6] = {lengths, (uint64_t)p->batch * 4, "lengths"};
    const Range outs[3] = {
        {out, strided_bytes(p->batch, row, row, p->dtype), "out"},
        {lse, lse ? (uint64_t)p->batch * p->heads * 4 : 0, "lse"},
        {workspace, (uint64_t)need, "workspace"}};
    if ((st = check_disjoint(outs, 3, in, 7)) != BSCACHE_OK) return st;
    a.q = q;
    a.table = table;
    a.lengths = lengths;
    a.out = out;
    a.lse = lse;
    a.parts = static_cast<float*>(workspace);
    return from_hip(bscache::launch_attend(a, (hipStream_t)stream),
                    "bscache_attend launch");
}

}  // extern "C"

// Attention of one new token over the pages of a quantized cache.
//
// A workgroup takes units of 128 tokens of one (sequence, key-value head, tile
// of up to 16 query heads; more heads are more tiles, each of which reads the rows
// by itself); its four waves take 32 tokens of a unit each and never wait for one
// another until the pair ends.  (The wide form is as many waves as a CU holds, and
// units of 32 tokens for each.)  Per wave and unit:
//
//   logits  S[token][head] = K q as v_mfma_f32_16x16x32_f16 with the codes as
//           the A operand (row = token, k = channel) and the queries as B
//           (column = head), 16 tokens at a time.  Lane l gets the logits of
//           head l % 16 for the tokens 4 (l / 16) .. + 3 of each 16.
//   softmax the references and sums of a head live in its 4 lanes.
//   values  O[channel][head] += V^T w, the same instruction: A = codes (row =
//           channel, k = token), B = weights (column = head, k = token).  The
//           order of k is free as long as A and B agree, so the weights stay
//           in the lanes that computed them: k 0..7 of lane group g are the
//           tokens 4 g .. + 3 of both halves, and lane l loads those tokens'
//           codes.  No weight ever moves between lanes.
//
// Codes become float16 without conversions.  For 16-bit calls a code's own bits
// are the operand: as a float16 they are the subnormal c 2^-24, which the
// matrix unit multiplies exactly (one byte permutation for two codes).  The unit
// aligns products by the operands' exponents, and the leading zeros of a
// subnormal are bits that it loses of the sum; so 4-bit codes are taken as 16 c
// and 8-bit keys as 4 c, a shift more for two of them (4-bit keys as c: lse off
// by 2 to 4 10^-6, 8-bit ones as c: up to 9 10^-7, now 5 10^-7 and less; 8-bit
// calls of one unit take 1 % longer for it, long ones as long).  8-bit values of
// 16-bit calls stay c: the sums lose up to 2^-22 of their terms, against the
// 2^-12 and 2^-9 that the outputs are rounded to.  float32 calls centre the codes: 0x6400 | c is 1024 + c, and one packed subtraction of 1024 +
// centre (128; 8 of the 4-bit ones) gives c' = c - centre exactly, so that sums
// do not grow by the offset and cancel again.  With z' = z + centre s (centre 0
// where the codes are not centred) a value is s c' + z', and
//   logit = scale (s (q . c') + z' sum q)
//   out   = (sum_t w_t c'_t + sum_t p_t z'_t) / sum_t p_t,   w = p s.
//
// Roundings: q is scaled by a power of two to below 2^14 (2^13 over 4-bit keys)
// and rounded to float16: bfloat16 and float16 values keep all their bits, but
// for what lies below 2^-30 of the row's largest; float32 queries take a second
// float16 for the rest (22 bits together), a second MFMA into the same
// accumulator.  w is two float16 as well, 22 bits.  (One, for bfloat16 calls, was
// 2^-12 of w c, whose terms are 3 times the spread of the values where codes are
// not centred, and moved outputs by a step; the second takes 1 % more: 128
// sequences of 12-16 Ki tokens 516 and 521 us.)
// Weights and the softmax's sum have references of their own.  p = 2^(logit - m),
// m the running maximum up to a whole number (a wave's only token has p = 1, and
// its value comes out as it is): the exponents of what counts are next to 0, where
// their own rounding is least, and what float32 drops is 2^-126 of the largest
// and less.  (24 below the maximum it was 2^-150, but float32 outputs half as far
// off again.)  w = 2^k p s, with k such that the largest p max(s, 2^-10 |z|) so
// far makes 2^6 to 2^7: a row counts by what is attended to of it, and one that
// is not, however wide, takes no bits from the others.
// (2^-10 |z|: z far beyond s is a row of nearly equal values, whose sums 2^k p z
// would leave float32.  It is looked at only where a sum gets large.)  Both lag
// by up to 2^8, so w stays below 2^15; it keeps its 22 bits down to 2^-9 of the
// largest, and is rounded to 2^-31 of that below.  A partial result is the mean of
// its own tokens, with m and the sum of p.  Everything else is float32.
//
// Sharing: the units of all (sequence, head tile) pairs are numbered in one row
// of places, and workgroup i of n takes the places [i U / n, (i + 1) U / n):
// every workgroup has the same work whatever the lengths.  U depends on the
// lengths, which only the device knows; each workgroup computes it from them.
// A workgroup whose range covers a pair's units whole writes its output;
// otherwise it leaves a partial result -- at most two, at the ends of its
// range -- which join_kernel adds in the order of the workgroups.  (Joining in
// the workgroup that comes last, by a counter, was tried: the results have to
// go past the L2s of the XCDs, and a call of few pairs and many partial
// results leaves them to one workgroup; 1 us shorter with up to 8 of them a
// pair, 9 to 16 us longer with 64 and more.)  Calls of short sequences
// (Attend::whole) give every pair to one workgroup instead.  Lengths that change
// during a call make its results wrong, but the number of the sequence, of the
// loops' rounds and of the partial results stays within the call's.
#pragma once

#include "cache_internal.h"

namespace bscache {

constexpr float kNone = -3.0e38f;       // reference of no logits
// k of the first tokens: the largest p is above 1/2, a step at least 2^-60.
constexpr int kMost = 68;
constexpr float kLn2 = 0.69314718055994530942f;
constexpr float kLog2e = 1.44269504088896340736f;

// ---- the row of units ------------------------------------------------------

// Visible tokens of a sequence: [first, length), first taken down to a
// multiple of 16 for its tiles.
struct Span {
    int32_t length, first;
    __device__ __forceinline__ int32_t start() const { return first & ~15; }
    // a sequence without tokens has one unit: somebody writes its zeros
    __device__ __forceinline__ int32_t units(int32_t tokens = kUnit) const {
        return (length - start() - 1) / tokens + 1;
    }
};
__device__ __forceinline__ int32_t length_of(const Attend& a, int32_t b) {
    return b < a.batch ? a.lengths[b] : 0;
}
__device__ __forceinline__ Span span_of(const Attend& a, int32_t length) {
    Span s;
    s.length = length < 0 ? 0 : length < a.max_len ? length : a.max_len;
    s.first = a.window > 0 && s.length > a.window ? s.length - a.window : 0;
    return s;
}

// Inclusive sum over the lanes of a wave up to this one: within rows of 16
// lanes, then the rows' sums passed on (DPP moves; lanes without a source add
// 0).
template <int CTRL, int ROWS>
__device__ __forceinline__ int32_t scan_step(int32_t v) {
    return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
__device__ __forceinline__ int32_t wave_scan(int32_t v) {
    v = scan_step<0x111, 0xF>(v);       // row_shr 1, 2, 4, 8
    v = scan_step<0x112, 0xF>(v);
    v = scan_step<0x114, 0xF>(v);
    v = scan_step<0x118, 0xF>(v);
    v = scan_step<0x142, 0xA>(v);       // row_bcast 15 into rows 1 and 3
    return scan_step<0x143, 0xC>(v);    // row_bcast 31 into rows 2 and 3
}

// Places of a pair in the row: its units, then an empty one for what it costs to
// begin and end a pair (5 us, against 1.2 us a unit where a workgroup has one
// or two pairs, and 2.6 us where it has many and the memory is busy; at least 3
// places a pair: 1000 sequences of 1-4096 tokens 263 us for 253).
__device__ __forceinline__ int32_t pair_places(int32_t units) {
    return units + 1;
}
// Those of sequence b, for one head tile.
__device__ __forceinline__ int32_t places_of(const Attend& a, int32_t b,
                                             int32_t length) {
    return b < a.batch ? pair_places(span_of(a, length).units()) : 0;
}

// All sequences' places, for one head tile, over the lanes of a wave: lane l has
// the `per` sequences from l per on, so that a batch of any size takes two
// rounds of loads, this one and that over one lane's sequences.
struct Row {
    int32_t per;              // sequences of a lane
    int32_t length;           // the lane's first sequence's
    int32_t mine, sum;        // the lane's places, and with the lanes' before
    int32_t total;
};
__device__ __forceinline__ Row all_places(const Attend& a, int lane) {
    constexpr int kDeep = 8;  // loads in flight
    Row r;
    r.per = (a.batch + 63) >> 6;
    r.length = length_of(a, lane * r.per);
    r.mine = places_of(a, lane * r.per, r.length);
    for (int32_t k = 1; k < r.per; k += kDeep) {
        int32_t length[kDeep];
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            length[u] = length_of(a, lane * r.per + min(k + u, r.per - 1));
#pragma unroll
        for (int u = 0; u < kDeep; ++u)
            if (k + u < r.per)
                r.mine += places_of(a, lane * r.per + k + u, length[u]);
    }
    r.sum = wave_scan(r.mine);
    r.total = __builtin_amdgcn_readlane(r.sum, 63);
    return r;
}

// A word of a table that the kernel only reads, at a place that is the same
// for the whole wave: a scalar load, whose wait does not wait for the codes
// in flight.
__device__ __forceinline__ int32_t uniform_load(const int32_t* p, int64_t at) {
    typedef const __attribute__((address_space(4))) int32_t* Constant;
    return ((Constant)(uintptr_t)p)[at];
}

// The workgroups that share u places: every one of them has at least one.
__device__ __forceinline__ int32_t sharing(const Attend& a, int32_t u) {
    return u < a.blocks ? u : a.blocks;
}
__device__ __forceinline__ int32_t range_start(int32_t i, int32_t u, int32_t n) {
    return (int32_t)((int64_t)u * i / n);
}
// Partial results: slot 2 i of workgroup i for the pair that began before its
// range, 2 i + 1 for the pair that goes on behind it.  A slot holds [16][dim]
// means and [16][2] reference and sum of p.
// Behind the slots, for every pair: the workgroups of its first and last units.
__host__ __device__ __forceinline__ int64_t part_bytes(int32_t dim) {
    return 64 * (dim + 2);
}
__device__ __forceinline__ int32_t* ends_of(const Attend& a) {
    return reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(a.parts) +
                                      2 * a.blocks * part_bytes(a.c.dim));
}
__device__ __forceinline__ float* part_of(const Attend& a, int32_t slot) {
    return a.parts + (int64_t)slot * 16 * (a.c.dim + 2);
}

// ---- codes to float16 ------------------------------------------------------

__device__ __forceinline__ uint32_t minus(uint32_t pair, _Float16 bias) {
    const half2v b = {bias, bias};
    return __builtin_bit_cast(uint32_t,
                              __builtin_bit_cast(half2v, pair) - b);
}

// Two codes, bytes A and B of the pair (hi, lo) of words, lo's are 0..3.
template <int A, int B, bool CENTRED>
__device__ __forceinline__ uint32_t byte_pair(uint32_t hi, uint32_t lo) {
    const uint32_t c =
        __builtin_amdgcn_perm(hi, lo, 0x0C000C00u | B << 16 | A);
    if constexpr (!CENTRED) return c;
    return minus(c | 0x64006400u, (_Float16)1152.0f);
}
// 4-bit codes as bytes 16 c: those in the low halves of 4 bytes (codes 0, 2, 4,
// 6 of a word) and in the high ones (1, 3, 5, 7).
__device__ __forceinline__ uint32_t low_nibbles(uint32_t x) {
    return x << 4 & 0xF0F0F0F0u;
}
__device__ __forceinline__ uint32_t high_nibbles(uint32_t x) {
    return x & 0xF0F0F0F0u;
}

// Channel-major operand of the keys: 8 codes of one token.  8 bits: 4 in x, 4
// in y, in order (as 4 c where they are not centred); 4 bits: all in x, in the order 0 2 4 6 1 3 5 7.
template <int BITS, bool CENTRED>
__device__ __forceinline__ half8v key_operand(uint32_t x, uint32_t y) {
    if constexpr (BITS == 4) {
        y = high_nibbles(x);
        x = low_nibbles(x);
    }
    u32x4 f = {byte_pair<0, 1, CENTRED>(x, x),
               byte_pair<2, 3, CENTRED>(x, x),
               byte_pair<0, 1, CENTRED>(y, y),
               byte_pair<2, 3, CENTRED>(y, y)};
    if constexpr (BITS == 8 && !CENTRED) f <<= 2;
    return __builtin_bit_cast(half8v, f);
}
// Channel of element e (0..7) of that operand.
template <int BITS>
__device__ __forceinline__ constexpr int key_channel(int e) {
    return BITS == 8 ? e : 2 * (e & 3) + (e >> 2);
}

// Token-major operands of the values: from 4 codes, as bytes, of each of 8
// tokens one operand for each of the 4 channels.
template <bool CENTRED>
__device__ __forceinline__ void value_operands(const uint32_t (&x)[8],
                                               half8v (&f)[4]) {
    u32x4 r[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const uint32_t a = x[2 * p], b = x[2 * p + 1];
        r[0][p] = byte_pair<0, 4, CENTRED>(b, a);
        r[1][p] = byte_pair<1, 5, CENTRED>(b, a);
        r[2][p] = byte_pair<2, 6, CENTRED>(b, a);
        r[3][p] = byte_pair<3, 7, CENTRED>(b, a);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = __builtin_bit_cast(half8v, r[i]);
}

__device__ __forceinline__ f32x4 mfma(half8v a, half8v b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// Over the 4 lanes of a head.
template <class F>
__device__ __forceinline__ float over_groups(float v, F f) {
    v = f(v, __shfl_xor(v, 16));
    return f(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float add(float a, float b) { return a + b; }
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }

__device__ __forceinline__ void store_out(void* out, int64_t at, int dtype,
                                          f32x4 v) {
    if (dtype == kF32) {
        *reinterpret_cast<f32x4*>(static_cast<float*>(out) + at) = v;
    } else {
        const u32x2 w = dtype == kF16
            ? u32x2{pack2<kF16>(v[0], v[1]), pack2<kF16>(v[2], v[3])}
            : u32x2{pack2<kBF16>(v[0], v[1]), pack2<kBF16>(v[2], v[3])};
        *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + at) = w;
    }
}

// Quotient of 4 sums and the sum of weights: 0 where there are none.
__device__ __forceinline__ f32x4 mean(f32x4 r, float l) {
#pragma unroll
    for (int e = 0; e < 4; ++e) r[e] = l == 0.0f ? 0.0f : r[e] / l;
    return r;
}

// Writes 4 channels of a row of the output, and its lse: of p with reference m
// and sum l.
__device__ __forceinline__ void finish(const Attend& a, int dtype, int64_t row,
                                       int d, float m, float l, f32x4 r) {
    store_out(a.out, row * a.c.dim + d, dtype, r);
    if (d == 0 && a.lse) {
        // l = 2^e f: m + e is exact, and small where m and e cancel
        const int e = __builtin_amdgcn_frexp_expf(l);
        const float f = __builtin_amdgcn_frexp_mantf(l);
        a.lse[row] =
            l == 0.0f ? -INFINITY
                      : ((m + (float)e) + __builtin_amdgcn_logf(f)) * kLn2;
    }
}

// ---- the kernel ------------------------------------------------------------

// The codes of a wave's 32 tokens as they are loaded.  Keys: lane l has, of
// token l % 16 of each half, the 16-code chunks l / 16 + 4 j.  Values: of the
// 8 tokens of its lane group, the DP / 16 codes from DP / 16 (l % 16) on.
template <int DP, int KB, int VB>
struct Codes {
    static constexpr int kChunks = DP / 64;        // 16-code chunks a lane
    static constexpr int kKeyWords = KB / 2;       // words of a chunk: 4 or 2
    static constexpr int kOwn = DP / 16;           // value channels a lane
    static constexpr int kValueWords = kOwn * VB >= 32 ? kOwn * VB / 32 : 1;
    uint32_t k[2][kChunks][kKeyWords];
    uint32_t v[8][kValueWords];
};

// The rows of half a tile as a buffer: the base stays in scalar registers, a
// lane's offset in one vector register, and nothing behind the rows can be
// read.
typedef __amdgpu_buffer_rsrc_t Rsrc;
__device__ __forceinline__ Rsrc rows_buffer(const void* base, int64_t at,
                                            int32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(
        const_cast<uint8_t*>(static_cast<const uint8_t*>(base)) + at, (short)0,
        bytes, 0x00020000);   // 32-bit data format
}
// N words from a 4 N-byte aligned offset.  Rows of 8-bit values are read with
// the non-temporal policy: one instruction takes whole lines of them, and they
// leave the caches to the rest (100 sequences of 500-3000 tokens 85 -> 79 us).
// Keys and 4-bit values come by two instructions a line, and the second one
// would often find it gone (128 x 12-16 Ki tokens, 4-bit values 521 -> 551 us).
constexpr int kOnce = 2;
template <int POLICY, int N>
__device__ __forceinline__ void load_words(Rsrc rows, uint32_t at,
                                           uint32_t (&w)[N]) {
    if constexpr (N == 1) {
        w[0] = __builtin_amdgcn_raw_buffer_load_b32(rows, at, 0, POLICY);
    } else if constexpr (N == 2) {
        const u32x2 t = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_raw_buffer_load_b64(rows, at, 0, POLICY));
        w[0] = t[0], w[1] = t[1];
    } else {
        static_assert(N == 4);
        const u32x4 t = __builtin_bit_cast(
            u32x4, __builtin_amdgcn_raw_buffer_load_b128(rows, at, 0, POLICY));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = t[i];
    }
}

// x, as a value that the compiler computes with from here on only: what is
// derived from it is not computed ahead of the loops, where it would take
// registers from them (11 to 54 spilled, in the loops too).
__device__ __forceinline__ int here(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// x with all its bits as they are here.  A product that is rounded to float16 may
// be computed a second time for that, with one rounding instead of two
// (v_fma_mixlo_f16, whatever -ffp-contract says): next to a tie the two differ
// by a step of float16, and a rest taken from the other one misses it.
__device__ __forceinline__ float rounded(float x) {
    asm("" : "+v"(x));
    return x;
}

// Where the two halves of a wave's tile lie: the row of each half's first
// token, and the end of its visible tokens (0 where its page is none of the
// cache).  Half a tile never leaves a page (pages are multiples of 16 tokens).
struct Tile {
    uint32_t token;         // first token (a unit may end beyond 2^31)
    int64_t row[2];
    uint32_t end[2];
};

template <int DP, int KB, int VB, int T, bool WIDE>
__global__ __launch_bounds__(64 * group_waves(DP, T, WIDE),
                             attend_waves(DP, T))
void attend_kernel(const Attend a) {
    using C = Codes<DP, KB, VB>;
    constexpr int kWaves = group_waves(DP, T, WIDE), kThreads = 64 * kWaves;
    constexpr int kStep = 32 * kWaves;          // tokens of a workgroup's step
    const bool one = WIDE || a.whole;           // every pair one workgroup's
    constexpr int kSteps = DP / 32;             // MFMAs of the logits
    constexpr int kOwn = C::kOwn;
    constexpr bool kTwoQ = T == kF32, kCentred = T == kF32;
    constexpr float kCentreK = !kCentred ? 0.0f : KB == 8 ? 128.0f : 8.0f;
    constexpr float kCentreV = !kCentred ? 0.0f : VB == 8 ? 128.0f : 8.0f;
    // codes over what they are as float16; of keys, and with what the products'
    // sums are brought down by, 2^kUnitK
    constexpr float kCode = kCentred ? 1.0f : 0x1p24f;
    constexpr int kDown = kCentred ? 26 : 0;
    constexpr int kUnitK =
        (kCentred ? kDown : 24) - (KB == 4 ? 4 : kCentred ? 0 : 2);
    // Queries are brought to below 2^(kQ + 1).  With that and kDown the sum of
    // 256 products with keys of up to 2^126 (1 + 2^-6) stays within float32:
    // 2^-kUnitK 2^8 2^(kQ + 1) 2^126 is 2^126 and 2^127 for 8- and 4-bit keys of
    // 16-bit calls, 2^122 and 2^126 for float32.
    constexpr int kQ = KB == 4 && !kCentred ? 12 : 13;
    constexpr float kCodeV = VB == 8 ? kCode : kCode / 16;
    __shared__ float sm_o[kWaves][16][DP + 4];
    __shared__ float sm_m[kWaves][16], sm_l[kWaves][16];
    __shared__ int sm_k[kWaves][16];

    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int dim = a.c.dim;
    const int32_t pairs = a.c.kv_heads * a.head_tiles;

    // this workgroup's places and the pair of the first
    const int32_t self = blockIdx.x;
    int32_t place = 0, place_end = 0, pair_start = 0, seq = 0, pair = 0;
    // lengths of 64 sequences, from `lengths_of` on
    int32_t lengths = 0, lengths_of = 0;
    if (one) {
        seq = self / pairs;
        pair = self - seq * pairs;
        lengths = uniform_load(a.lengths, seq);
        lengths_of = seq;
    } else {
        const Row r = all_places(a, lane);
        const int32_t total = r.total * pairs;
        const int32_t sharers = sharing(a, total);
        if (self >= sharers) return;
        place = range_start(self, total, sharers);
        place_end = range_start(self + 1, total, sharers);
        // the lane whose sequences hold the first place, then the sequence
        int at = __builtin_ctzll(__ballot(r.sum * pairs > place));
        int32_t before = __builtin_amdgcn_readlane(r.sum - r.mine, at);
        int32_t own = r.mine, sum = r.sum;
        lengths = r.length;
        if (r.per > 1) {
            lengths_of = at * r.per;
            for (;;) {
                lengths = length_of(a, lengths_of + lane);
                own = places_of(a, lengths_of + lane, lengths);
                sum = before + wave_scan(own);
                const uint64_t past = __ballot(sum * pairs > place);
                if (past) {
                    at = __builtin_ctzll(past);
                    break;
                }
                before = __builtin_amdgcn_readlane(sum, 63);
                lengths_of += 64;
                if (lengths_of >= a.batch) return;   // (see above)
            }
        }
        const int32_t its = __builtin_amdgcn_readlane(own, at);
        seq = lengths_of + at;
        before = __builtin_amdgcn_readlane(sum, at) - its;
        pair = (place - before * pairs) / its;
        pair_start = before * pairs + pair * its;
    }

    for (bool again = false;;) {
        if (seq - lengths_of >= 64) {
            lengths_of = seq;
            lengths = length_of(a, seq + lane);
        }
        const Span span = span_of(
            a, __builtin_amdgcn_readlane(lengths, seq - lengths_of));
        const int32_t units = span.units(kStep);
        // units [c0, c1) of this pair
        int32_t c0 = 0, c1 = units;
        if (!one) {
            c0 = min(place - pair_start, units);
            c1 = min(place_end - pair_start, units);
            if (c0 < c1 && wave == 0 && lane == 0) {
                // for the join: the first and the last workgroup of the pair
                int32_t* ends = ends_of(a) + 2 * ((int64_t)seq * pairs + pair);
                const int me = here(self);
                if (c0 == 0) ends[0] = me;
                if (c1 == units) ends[1] = me;
            }
            pair_start += pair_places(units);
            place = pair_start;
        }
        const int32_t kvh = pair / a.head_tiles;
        const int32_t tile16 = pair - kvh * a.head_tiles;
        const int32_t now_seq = seq;
        if (++pair == pairs) {
            pair = 0;
            ++seq;
        }
        const bool last = one || place >= place_end || seq >= a.batch;
        if (c0 >= c1) {              // nothing but empty places
            if (last) break;
            continue;
        }
        if (again) __syncthreads();  // the results of the pair before are read
        again = true;
        const int32_t h0 = kvh * a.group + tile16 * 16;
        const int32_t heads =
            a.group - tile16 * 16 < 16 ? a.group - tile16 * 16 : 16;

        const int my_lane = here(lane);
        const int head = my_lane & 15, group = my_lane >> 4;
        // lane offsets, in bytes, of the codes within 16 rows; lanes behind the
        // last channel read their row's first codes (their products are dropped)
        const int k_row = dim * KB / 8, v_row = dim * VB / 8;
        uint32_t k_at[C::kChunks];
#pragma unroll
        for (int j = 0; j < C::kChunks; ++j) {
            const int chunk = group + 4 * j;
            k_at[j] = head * k_row + (chunk * 16 < dim ? chunk * 2 * KB : 0);
        }
        const uint32_t v_at =
            4 * group * v_row + (head * kOwn < dim ? head * kOwn * VB / 8 : 0);

        // ---- tiles and their loads
        C codes;
        uint32_t ks[2][4], vs[2][4];
        const int64_t table = (int64_t)now_seq * a.max_pages;
        auto find = [&](int32_t c) {
            Tile t;
            t.token = (uint32_t)span.start() + (uint32_t)c * kStep + wave * 32;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t at = t.token + 16 * s;
                const bool in = at < (uint32_t)span.length && c < c1;
                const uint32_t p = in ? a.c.by_page.div(at) : 0;
                const uint32_t page = uniform_load(a.table, table + p);
                const bool there = in && page < a.c.pages;
                t.end[s] = there ? span.length : 0;
                t.row[s] = row_of(a.c, there ? page : 0, kvh,
                                  there ? at - p * a.c.by_page.d : 0);
            }
            return t;
        };
        auto load_keys = [&](const Tile& t) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Rsrc rows =
                    rows_buffer(a.c.codes[0], t.row[s] * k_row, 16 * k_row);
#pragma unroll
                for (int j = 0; j < C::kChunks; ++j)
                    load_words<0>(rows, k_at[j], codes.k[s][j]);
            }
        };
        auto load_steps = [&](const Tile& t) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                load_words<0>(rows_buffer(a.c.steps[0], t.row[s] * 4, 64),
                           16 * group, ks[s]);
                load_words<0>(rows_buffer(a.c.steps[1], t.row[s] * 4, 64),
                           16 * group, vs[s]);
            }
        };
        auto load_values = [&](const Tile& t) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const Rsrc rows =
                    rows_buffer(a.c.codes[1], t.row[s] * v_row, 16 * v_row);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t at = v_at + i * v_row;
                    if constexpr (kOwn * VB < 32)
                        codes.v[4 * s + i][0] =
                            __builtin_amdgcn_raw_buffer_load_b16(rows, at, 0,
                                                                 0);
                    else
                        load_words<VB == 8 ? kOnce : 0>(rows, at,
                                                        codes.v[4 * s + i]);
                }
            }
        };

        // the queries of this lane's head, loaded ahead of the codes and kept
        // as they are stored until they become operands
        Eight<T> qx[kSteps];
        const bool mine = head < heads;
        {
            const int64_t base =
                now_seq * a.q_stride + (int64_t)(h0 + (mine ? head : 0)) * dim;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const int chunk = group + 4 * (i >> 1);
                qx[i].load(a.q, base + (chunk * 16 < dim
                                            ? chunk * 16 + 8 * (i & 1) : 0));
            }
        }
        Tile now = find(c0);
        load_keys(now);
        load_steps(now);
        load_values(now);
        Tile next = find(c0 + 1);

        // ---- the queries as B operands
        half8v q_hi[kSteps], q_lo[kTwoQ ? kSteps : 1];
        // a logit in units of log2 is (s (q' . c') + z' q_sum) q_scale
        float q_scale, q_sum;
        {
            float top = 0.0f, sum = 0.0f;
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                if (!mine || (group + 4 * (i >> 1)) * 16 >= dim) qx[i].clear();
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    top = fmaxf(top, fabsf(qx[i].get(e)));
            }
            top = over_groups(top, larger);
            // 2^-e brings the largest into [2^kQ, 2^(kQ + 1)); rows below 2^-114
            // may stay below
            const int e = max((int)(f32_bits(top) >> 23), kQ) - 127 - kQ;
            // (the sign of the scale goes into q: q_scale is not negative)
            const float down = copysignf(ldexpf(1.0f, -e), a.scale);
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    // (a power of two: exact)
                    const float y = qx[i].get(key_channel<KB>(j)) * down;
                    const _Float16 hi = (_Float16)y;
                    q_hi[i][j] = hi;
                    if constexpr (kTwoQ) q_lo[i][j] = (_Float16)(y - (float)hi);
                }
            // (of what is scaled: a finite row's own sum may be beyond float32)
#pragma unroll
            for (int i = 0; i < kSteps; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) sum += qx[i].get(e) * down;
            sum = over_groups(sum, add);
            // an infinity makes the whole head NaN, as a NaN does by itself
            if (!(top < INFINITY)) sum = NAN;
            // (above 0, so that a masked -inf stays one, and so little that
            // nothing finite gets above 2^-20 by it)
            q_scale =
                fmaxf(ldexpf(fabsf(a.scale), e + kUnitK) * kLog2e, 0x1p-149f);
            q_sum = ldexpf(sum, -kUnitK);
        }

        f32x4 o[kOwn];
#pragma unroll
        for (int j = 0; j < kOwn; ++j) o[j] = f32x4{0, 0, 0, 0};
        float m = kNone;            // reference of p
        int k = kMost;              // of the weights: w = 2^k p s
        float sum_p = 0.0f;
        float sum_z = 0.0f;         // of 2^k p z

        for (int32_t c = c0; c < c1; ++c) {
            // ---- logits
            f32x4 acc[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    const uint32_t(&w)[C::kKeyWords] = codes.k[s][i >> 1];
                    half8v f;
                    if constexpr (KB == 8)
                        f = key_operand<8, kCentred>(w[2 * (i & 1)],
                                                     w[2 * (i & 1) + 1]);
                    else
                        f = key_operand<4, kCentred>(w[i & 1], 0);
                    acc[s] = mfma(f, q_hi[i], acc[s]);
                    if constexpr (kTwoQ) acc[s] = mfma(f, q_lo[i], acc[s]);
                }
            const bool more = c + 1 < c1;
            if (more) load_keys(next);

            // ---- softmax
            const uint32_t first = span.first;
            const bool whole = now.token >= first &&
                               now.token + 16 <= now.end[0] &&
                               now.token + 32 <= now.end[1];
            float x[2][4];
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float step = step_of(ks[s][i]);
                    float z = offset_of(ks[s][i]);
                    if constexpr (kCentred)
                        z = __builtin_fmaf(step, kCentreK, z);
                    const float qc =
                        kDown ? acc[s][i] * ldexpf(1.0f, -kDown) : acc[s][i];
                    x[s][i] = __builtin_fmaf(step, qc, z * q_sum);
                }
            bool lone = false;       // one token is all that this wave has
            if (!whole) {
                // tokens that are not seen: no weight, no value, whatever
                // their rows (nobody may have written them) and the query hold
                int seen_here = 0;
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const uint32_t begin = now.token + 16 * s;
                    seen_here += max((int)(min(now.end[s], begin + 16) -
                                           max(first, begin)), 0);
                }
                lone = seen_here == 1 && c0 + 1 == c1;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t t = now.token + 16 * s + 4 * group + i;
                        const bool seen = (t >= first) & (t < now.end[s]);
                        vs[s][i] = seen ? vs[s][i] : 0;
                        x[s][i] = seen ? x[s][i] : -INFINITY;
                    }
            }
            float big = -INFINITY;
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int i = 0; i < 4; ++i) big = fmaxf(big, x[s][i]);
            big *= q_scale;
            if (__any(big > m + 8.0f)) {
                // (of the heads that need it: the others stay as they would
                // without this one beside them)
                const float all = over_groups(big, larger);
                const float m_new = lone           ? fmaxf(m, all)
                                    : all > m + 8.0f ? ceilf(all)
                                                     : m;
                // (from kNone: more than any exponent)
                const int up = (int)fminf(m_new - m, 2000.0f);
                // what p falls by the weights keep, as far as k goes
                const int k_new = min(k + up, kMost);
                const float f = ldexpf(1.0f, k_new - k - up);
                sum_p *= ldexpf(1.0f, -up);
                sum_z *= f;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) o[j] *= f;
                m = m_new;
                k = k_new;
            }
            float p[8], w[8], z_next;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                p[i] = __builtin_amdgcn_exp2f(
                    __builtin_fmaf(x[i >> 2][i & 3], q_scale, -m));
            // where binary32's steps are not far below 1, the logits as they are
            // rounded, as the maximum is; so is the only one (p = 1: its value
            // comes out as a read gives it)
            const bool far = lone || !(fabsf(m) < 0x1p20f);
            if (__any(far)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float y = __builtin_amdgcn_exp2f(
                        x[i >> 2][i & 3] * q_scale - m);
                    p[i] = far ? y : p[i];
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) sum_p += p[i];
            auto offset = [&](int i) {
                const float z = offset_of(vs[i >> 2][i & 3]);
                return kCentred ? __builtin_fmaf(step_of(vs[i >> 2][i & 3]),
                                                 kCentreV, z)
                                : z;
            };
            auto weigh = [&] {
                z_next = sum_z;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float t = ldexpf(p[i], k);
                    w[i] = rounded(t * step_of(vs[i >> 2][i & 3]));
                    z_next = __builtin_fmaf(t, offset(i), z_next);
                }
            };
            weigh();
            float w_big = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) w_big = fmaxf(w_big, w[i]);
            const bool large = w_big > 0x1p15f || !(fabsf(z_next) <= 0x1p100f);
            if (__any(large)) {
                const bool its = over_groups(large ? 1.0f : 0.0f, larger) > 0.0f;
                float most = 0.0f;          // of 2^-64 p max(s, 2^-10 |z|)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    most = fmaxf(most,
                                 ldexpf(p[i], -64) *
                                     fmaxf(step_of(vs[i >> 2][i & 3]),
                                           fabsf(offset(i)) * 0x1p-10f));
                // these, and the sum, are below 2^e
                const int e = (int)(f32_bits(over_groups(most, larger)) >> 23) -
                              126 + 64;
                const int e_z =
                    (int)(f32_bits(over_groups(fabsf(sum_z), larger)) >> 23) -
                    126;
                const int k_new = its ? min(k, min(7 - e, k + 40 - e_z)) : k;
                const float f = ldexpf(1.0f, k_new - k);
                sum_z *= f;
#pragma unroll
                for (int j = 0; j < kOwn; ++j) o[j] *= f;
                k = k_new;
                weigh();
            }
            sum_z = z_next;
            half8v w_hi, w_lo;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const _Float16 hi = (_Float16)w[i];
                w_hi[i] = hi;
                w_lo[i] = (_Float16)(w[i] - (float)hi);
            }
            if (more) load_steps(next);

            // ---- values
            auto add_values = [&](const uint32_t (&y)[8], int first, int by) {
                half8v f[4];
                value_operands<kCentred>(y, f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f32x4& sum = o[first + e * by];
                    sum = mfma(f[e], w_hi, sum);
                    sum = mfma(f[e], w_lo, sum);
                }
            };
            if constexpr (VB == 8) {
#pragma unroll
                for (int j = 0; j < kOwn; j += 4) {
                    uint32_t y[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) y[i] = codes.v[i][j >> 2];
                    add_values(y, j, 1);
                }
            } else {
#pragma unroll
                for (int j = 0; j < kOwn; j += 8) {
                    uint32_t y[8], z[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        y[i] = low_nibbles(codes.v[i][j >> 3]);
                        z[i] = high_nibbles(codes.v[i][j >> 3]);
                    }
                    if constexpr (kOwn >= 8) {
                        add_values(y, j, 2);         // channels 0, 2, 4, 6
                        add_values(z, j + 1, 2);     // 1, 3, 5, 7
                    } else {
                        // 4 codes: bytes 0 and 1 of each
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            y[i] = __builtin_amdgcn_perm(z[i], y[i],
                                                         0x05010400u);
                        add_values(y, j, 1);
                    }
                }
            }
            if (more) {
                load_values(next);
                now = next;
                next = find(c + 2);
            }
        }

        // ---- the waves' results
        sum_p = over_groups(sum_p, add);
        sum_z = over_groups(sum_z, add);
        const int end_lane = here(lane);
        const int col = end_lane & 15, quarter = end_lane >> 4;
        if (quarter == 0) {
            sm_m[wave][col] = m;
            sm_l[wave][col] = sum_p;
            sm_k[wave][col] = k;
        }
        // o[j][i] is channel kOwn (4 (lane / 16) + i) + j of head lane % 16
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < kOwn; j += 4) {
                f32x4 r;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    r[e] = __builtin_fmaf(
                        o[j + e][i], kCodeV, sum_z);
                *reinterpret_cast<f32x4*>(
                    &sm_o[wave][col][kOwn * (4 * quarter + i) + j]) = r;
            }
        __syncthreads();
        const bool is_whole = c0 == 0 && c1 == units;
        const int64_t row0 = (int64_t)now_seq * a.heads + h0;
        float* part = is_whole ? nullptr
                               : part_of(a, 2 * self + (c0 > 0 ? 0 : 1));
        const int quads = dim >> 2;
        for (int n = 64 * wave + end_lane; n < heads * quads; n += kThreads) {
            const int h = n / quads, d = 4 * (n - h * quads);
            float top = sm_m[0][h];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) top = fmaxf(top, sm_m[w][h]);
            // a wave's sums are its means times 2^(k + its p's): the largest
            // of the factors that bring them to p of `top`, then the sums
            int down = -4000;
#pragma unroll
            for (int w = 0; w < kWaves; ++w)
                down = max(down, (int)fmaxf(sm_m[w][h] - top, -2000.0f) -
                                     sm_k[w][h]);
            f32x4 r = {0, 0, 0, 0};
            float l = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float by = __builtin_amdgcn_exp2f(sm_m[w][h] - top);
                const float f = ldexpf(by, -sm_k[w][h] - down);
                l = __builtin_fmaf(by, sm_l[w][h], l);
                const f32x4 y =
                    *reinterpret_cast<const f32x4*>(&sm_o[w][h][d]);
#pragma unroll
                for (int e = 0; e < 4; ++e) r[e] = __builtin_fmaf(f, y[e], r[e]);
            }
            r = mean(r, l);
#pragma unroll
            for (int e = 0; e < 4; ++e) r[e] = ldexpf(r[e], down);
            if (is_whole) {
                finish(a, T, row0 + h, d, top, l, r);
            } else {
                *reinterpret_cast<f32x4*>(part + h * dim + d) = r;
                if (d == 0)
                    *reinterpret_cast<float2*>(part + 16 * dim + 2 * h) =
                        make_float2(top, l);
            }
        }
        if (last) break;
    }
}

// Launches the kernel for DP padded channels (one translation unit each).
template <int DP>
hipError_t launch_attend_dp(const Attend& a, hipStream_t st);

}  // namespace bscache

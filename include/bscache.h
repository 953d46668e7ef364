/*
 * bscache.h -- C ABI of libbscache.so: a paged key-value cache of B-bit codes
 * and the attention that reads it, for AMD MI355X (gfx950).
 *
 * The quantization operator applied to what a program that answers with a
 * language model keeps: the keys and values of every token seen so far.  A
 * row -- one token's `dim` channels of one key-value head -- is kept as dim
 * unipolar codes of B bits (B = 8 or 4, for keys and for values separately)
 * and a step s and offset z in bfloat16; it stands for z + s c.
 *
 *   bscache_write   float rows of new tokens -> codes, steps and offsets
 *   bscache_read    the values that rows stand for
 *   bscache_attend  attention of one new token of each sequence over its rows
 *
 * Row of a float vector x (fl32: rounded to binary32, half to even):
 *   x' = 0 where x is NaN, otherwise x clamped to +-2^126
 *   z  = the largest bfloat16 <= min x'
 *   s  = max(2^-60, the smallest bfloat16 >=
 *                   fl32(fl32(max x' - z) * fl32(1 / (2^B - 1))))
 *   c  = min(2^B - 1, round_half_to_even(fl32(fl32(x' - z) * fl32(1 / s))))
 *   value = fl32(z + s c)
 * so a value is off by at most s / 2 (and a few units of binary32).
 *
 * Conventions (as bitserial.h):
 *  - Data pointers are DEVICE pointers owned by the caller; the library never
 *    allocates, frees or keeps them, and keeps no state between calls.  Every
 *    base pointer must be 16-byte aligned.
 *  - Calls are asynchronous on `stream` (a hipStream_t of the current device;
 *    NULL = null stream) and may be captured into a graph: they enqueue
 *    kernels only.
 *  - Arguments are validated on the host before anything is enqueued; an
 *    invalid call returns its status and enqueues nothing.
 *    bscache_last_error() then describes the problem.
 *  - An empty problem (tokens == 0 or batch == 0) is valid and enqueues
 *    nothing.
 *  - An output must not share a byte with an input or another output.
 *  - Slots, page tables and lengths are data on the device: what they say is
 *    checked by the kernels, which never read or write outside the cache
 *    whatever they hold (see each call).
 *  - Results do not depend on timing: no kernel uses atomics, so repeated
 *    calls are bit-identical.
 *  - Thread safety: calls from several host threads are safe; the error
 *    string is per thread.
 *  - Calls in flight on several streams are independent unless one writes
 *    what another reads or writes: a workspace belongs to one call at a time
 *    (two captured graphs that may run at once need one each).
 */
#ifndef BSCACHE_H
#define BSCACHE_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* The values are bs_status's. */
typedef enum {
    BSCACHE_OK = 0,
    BSCACHE_ERR_INVALID_ARG = 1, /* NULL/misaligned pointer, bad size */
    BSCACHE_ERR_UNSUPPORTED = 2, /* a size this library does not cover */
    BSCACHE_ERR_HIP = 4          /* the HIP runtime refused the launch */
} bscache_status;

/* Type of keys, values, queries and outputs. */
typedef enum { BSCACHE_F32 = 0, BSCACHE_F16 = 1, BSCACHE_BF16 = 2 }
    bscache_dtype;

typedef void *bscache_stream_t;   /* a hipStream_t */

/* A cache: pages of page_tokens tokens each.
 *   codes: [pages][kv_heads][page_tokens][dim B / 8] uint8; of 4-bit codes,
 *          code 2 i is the low half of byte i and code 2 i + 1 the high one;
 *   steps: [pages][kv_heads][page_tokens][2] bfloat16: s, z.
 * A token's slot is page * page_tokens + its place in the page.
 * Sizes: dim a multiple of 16 up to 256, page_tokens a multiple of 16, bits
 * 8 or 4, at most 2^31 - 1 slots. */
typedef struct {
    int64_t pages;
    int32_t kv_heads, page_tokens, dim, kbits, vbits;
    uint8_t *k_codes;
    uint16_t *k_steps;
    uint8_t *v_codes;
    uint16_t *v_steps;
} bscache_pages;

/* Writes the rows of `tokens` new tokens.
 *   k, v: [tokens][kv_heads][dim] of type dtype; a token's kv_heads * dim
 *         values lie together, tokens k_stride and v_stride elements apart
 *         (slices of one projection's output; strides of whole 16 bytes);
 *   slots: [tokens] int32.  A token whose slot is outside the cache (-1: a
 *         padded place of a batch) is left out.
 * Rows of other slots keep their bytes.  Two tokens of one call must not name
 * the same slot: that slot's rows would hold a mixture of both.
 * Errors: INVALID_ARG for NULL/misaligned pointers, sizes < 1 (tokens < 0),
 * strides < kv_heads * dim or not of whole 16 bytes, an unknown dtype, buffers
 * that overlap; UNSUPPORTED for sizes beyond those of bscache_pages and for
 * calls of more than 2^31 - 1 rows (keys' and values'), or of 2^33 / L and more
 * with L = dim / 8 up to a power of two (a launch has 2^32 lanes). */
bscache_status bscache_write(const bscache_pages *cache, const void *k,
                             const void *v, int64_t k_stride,
                             int64_t v_stride, bscache_dtype dtype,
                             const int32_t *slots, int64_t tokens,
                             bscache_stream_t stream);

/* Reads the rows of `tokens` slots back, as the values they stand for rounded
 * to dtype (half to even).
 *   slots: [tokens] int32, any order, any slot more than once; a slot outside
 *         the cache gives zeros;
 *   k, v: [tokens][kv_heads][dim] of type dtype, fully overwritten.
 * Errors: as bscache_write. */
bscache_status bscache_read(const bscache_pages *cache, const int32_t *slots,
                            int64_t tokens, void *k, void *v,
                            bscache_dtype dtype, bscache_stream_t stream);

/* Attention of one new token of each of `batch` sequences:
 *   l[b][h][t] = scale * sum_d q[b][h][d] key[t][d]
 *   out[b][h]  = sum_t softmax_t(l[b][h])_t value[t]
 *   lse[b][h]  = log sum_t exp(l[b][h][t])
 * over the visible tokens t of sequence b: the last `window` (0: all) of its
 * lengths[b] tokens, keys and values those of key-value head
 * h / (heads / kv_heads).  The new token's own row is written before
 * (bscache_write) where it is to be seen.
 *   q:       [batch][heads][dim] of type dtype, sequences q_stride elements
 *            apart (whole 16 bytes);
 *   table:   [batch][max_pages] int32: token t of sequence b lies in page
 *            table[b][t / page_tokens]; entries behind its last page are not
 *            used.  Tokens of an entry outside the cache are not visible;
 *   lengths: [batch] int32; one above max_len counts as max_len, one below 0
 *            as 0; they must not change while the call runs;
 *   out:     [batch][heads][dim] of type dtype;
 *   lse:     [batch][heads] float32, or NULL.
 * A sequence without a visible token gets out = 0 and lse = -inf, whatever its
 * query holds.  Otherwise a query that holds a NaN or an infinity gives NaN for
 * its head alone.  Logits have to stay within binary32 (times log2 e), and
 * |scale| times a query's largest element below 2^100.
 * Products are of the exact codes: q enters the matrix units scaled by a power
 * of two as float16 (bfloat16 and float16 values keep their bits but for what
 * lies below 2^-30 of the row's largest; float32 as two float16 of 22 bits
 * together), weights times s as two float16 of 22 bits together, and to 2^-31 of
 * the largest weight times max(s, 2^-10 |z|); sums and the softmax are binary32,
 * weights below 2^-126 of the largest 0.
 * The workspace holds partial results of sequences that several workgroups
 * share: bscache_attend_workspace() bytes (0 for short max_len), 16-byte
 * aligned, contents irrelevant before and after.
 * Errors: INVALID_ARG for NULL/misaligned pointers, batch < 0, other sizes
 * < 1, heads not a multiple of kv_heads, max_len beyond max_pages *
 * page_tokens, window < 0, a scale that is not finite, q_stride < heads * dim
 * or not of whole 16 bytes, a workspace that is too small, buffers that
 * overlap; UNSUPPORTED as bscache_pages and for problems of 2^24 or more pairs
 * of a sequence and up to 16 query heads of a key-value head, of more than 2^30
 * units of 128 tokens of them (8 added for each), or of more than 2^31 - 1 rows
 * of out. */
typedef struct {
    int64_t q_stride;
    int32_t batch, heads;
    int32_t max_pages;           /* places of a row of the table */
    int32_t max_len;             /* no sequence is longer: sets the launch */
    int32_t window;
    int32_t dtype;               /* bscache_dtype of q and out */
    float scale;
} bscache_attend_params;

bscache_status bscache_attend_workspace(const bscache_pages *cache,
                                        const bscache_attend_params *p,
                                        int64_t *bytes);

bscache_status bscache_attend(const bscache_pages *cache,
                              const bscache_attend_params *p, const void *q,
                              const int32_t *table, const int32_t *lengths,
                              void *out, float *lse, void *workspace,
                              int64_t workspace_bytes,
                              bscache_stream_t stream);

/* Describes, as text, the kernel and launch that bscache_attend would use (the
 * way the call is shared out, workgroups, waves of each, workspace bytes).
 * Writes at most len bytes including the terminating NUL into buf (truncating);
 * host only, nothing is enqueued, the cache's pointers are not looked at.
 * Errors: as bscache_attend's checks of sizes; INVALID_ARG for a NULL buf or
 * len < 1. */
bscache_status bscache_attend_describe(const bscache_pages *cache,
                                       const bscache_attend_params *p,
                                       char *buf, int32_t len);

/* Detail of the last non-OK status returned on the calling thread ("" if
 * none).  The string stays valid until the next call on that thread. */
const char *bscache_last_error(void);

/* ABI version of this header (major * 100 + minor). */
int bscache_abi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* BSCACHE_H */

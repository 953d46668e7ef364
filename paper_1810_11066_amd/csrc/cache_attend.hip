// Launch of the cache's attention: how many workgroups share a call, which
// kernel takes it, and the join of their partial results.
#include <algorithm>

#include "cache_attend.h"

namespace bscache {
namespace {

// Adds the partial results of a pair that several workgroups share, in their
// order.  A workgroup of this kernel takes a.few query heads of one pair.
// Threads are columns of 4 channels of a head, times rows that take every
// rows-th partial result and are added at the end; a thread has kDeep of them
// in flight, and a running maximum of its own, so that no load waits for
// another but the pair's entry.  4 to 5 us, most of it the launch and two
// loads after one another.
constexpr int kDeep = 8, kThreads = 256;

__global__ __launch_bounds__(kThreads) void join_kernel(const Attend a) {
    __shared__ f32x4 sm_r[kThreads];
    __shared__ float2 sm_ml[kThreads];
    const int dim = a.c.dim, quads = dim >> 2;
    const int32_t pairs = a.c.kv_heads * a.head_tiles;
    const int32_t few = a.few;
    const int32_t slices = (min(a.group, 16) + few - 1) / few;
    const int32_t at = blockIdx.x / slices;
    const int32_t seq = at / pairs, pair = at - seq * pairs;
    const int32_t kvh = pair / a.head_tiles;
    const int32_t tile16 = pair - kvh * a.head_tiles;
    const int32_t h0 = (blockIdx.x - at * slices) * few;
    const int32_t heads = min(few, min(a.group - tile16 * 16, 16) - h0);
    const int64_t row0 =
        (int64_t)seq * a.heads + kvh * a.group + tile16 * 16 + h0;

    const int2 ends = *reinterpret_cast<const int2*>(ends_of(a) + 2 * at);
    const int32_t i0 = max(ends.x, 0);
    const int32_t parts = min(ends.y, a.blocks - 1) - i0 + 1;
    if (parts <= 1) return;          // its workgroup wrote the output

    const int32_t columns = heads * quads;
    const int32_t rows = columns < kThreads ? kThreads / max(columns, 1) : 1;
    for (int32_t c0 = 0; c0 < columns; c0 += kThreads) {
        const int32_t mine = rows > 1 ? threadIdx.x / columns : 0;
        const int32_t column = c0 + threadIdx.x - mine * columns;
        const int32_t h = column / quads, d = 4 * (column - h * quads);
        const bool on = mine < rows && column < columns;
        float m = kNone, l = 0.0f;
        f32x4 r = {0, 0, 0, 0};
        for (int32_t p = mine; on && p < parts; p += kDeep * rows) {
            float2 ml[kDeep];
            f32x4 y[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                const int32_t n = min(p + u * rows, parts - 1);
                const float* q = part_of(a, 2 * (i0 + n) + (n == 0 ? 1 : 0));
                ml[u] = *reinterpret_cast<const float2*>(q + 16 * dim +
                                                         2 * (h0 + h));
                y[u] = *reinterpret_cast<const f32x4*>(q + (h0 + h) * dim + d);
                if (p + u * rows >= parts) ml[u].x = -INFINITY;  // not again
            }
            // (means of means: a sum of products with values at either end
            // would leave binary32)
            float top = m;
#pragma unroll
            for (int u = 0; u < kDeep; ++u) top = fmaxf(top, ml[u].x);
            const float own = l * __builtin_amdgcn_exp2f(m - top);
            m = top;
            l = own;
            float g[kDeep];
#pragma unroll
            for (int u = 0; u < kDeep; ++u) {
                g[u] = __builtin_amdgcn_exp2f(ml[u].x - top) * ml[u].y;
                l += g[u];
            }
            const float per = l == 0.0f ? 0.0f : 1.0f / l;
            r *= own * per;
#pragma unroll
            for (int u = 0; u < kDeep; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    r[e] = __builtin_fmaf(g[u] * per, y[u][e], r[e]);
        }
        if (rows > 1) {              // (then there is one pass over columns)
            sm_r[threadIdx.x] = r;
            sm_ml[threadIdx.x] = make_float2(m, l);
            __syncthreads();
            if (mine == 0) {
                for (int32_t w = 1; w < rows; ++w)
                    m = fmaxf(m, sm_ml[w * columns + column].x);
                l = 0.0f;
                for (int32_t w = 0; w < rows; ++w) {
                    const float2 ml = sm_ml[w * columns + column];
                    l = __builtin_fmaf(__builtin_amdgcn_exp2f(ml.x - m), ml.y,
                                       l);
                }
                const float per = l == 0.0f ? 0.0f : 1.0f / l;
                r = f32x4{0, 0, 0, 0};
                for (int32_t w = 0; w < rows; ++w) {
                    const float2 ml = sm_ml[w * columns + column];
                    r += __builtin_amdgcn_exp2f(ml.x - m) * ml.y * per *
                         sm_r[w * columns + column];
                }
            }
        }
        if (on && mine == 0)
            finish(a, a.dtype, row0 + h, d, m, l, r);
    }
}

}  // namespace

template <> hipError_t launch_attend_dp<64>(const Attend&, hipStream_t);
template <> hipError_t launch_attend_dp<128>(const Attend&, hipStream_t);
template <> hipError_t launch_attend_dp<256>(const Attend&, hipStream_t);

// How a call is shared out, by what the host knows: the pairs of sequences and
// head tiles, and the tokens that the longest sequence may span.
//
// A pair to one workgroup needs no plan of the lengths and no join (4 us and a
// launch), but the longest pair sets the time: 5 us and 1.2 us a unit of
// 128 tokens.  Up to 4 units that is always shorter (8 pairs of 4 units 9.7 us whole
// and 10.5 shared, of 8 units 14.5 and 10.6; 128 pairs of 4 units 11.1 and 13.5).
// Longer ones win where the pairs fill the GPU anyway: up to 8 units with a pair
// for every CU (320 pairs of 8 units 23.7 and 26.6 us), up to 16 with pairs for
// half of the workgroups that run at once (512 pairs of 16 units 57.6 and 63.7 us,
// 64 channels 35.8 and 36.0).  Lengths from a quarter of the longest to all of it
// leave that so (384 pairs of 375 to 1500 tokens 29.4 and 28.1, 2000 pairs 99 and
// 108); where few are long, what the longest takes is lost (384 pairs of lengths
// spread by their logarithm from 1: to 1000 tokens 17.5 and 17.5, to 2000 29.1 and
// 19.3).
//
// With fewer pairs than CUs a workgroup can have its CU to itself: the wide
// form, of as many waves as the CU holds (8 to 16).  A CU's own rate of reading
// bounds it, so it needs pairs on a quarter of the CUs, and sequences of more
// than 4 units that it takes in 4 steps (128 pairs of 748 tokens 12.3 us wide,
// 15.2 shared; of 1132 14.8 and 17.7; of 1516 17.2 and 18.9; 64 pairs 11.7 and
// 12.6, 14.3 and 14.6, 16.9 and 15.3).
//
// Everything else is shared: as many workgroups as run at once, each with its
// part (4 times as many, taken up as others end: 551 us for 524 at 128
// sequences of 12-16 Ki tokens).  The join takes all heads of a tile together
// where pairs are many (64 ragged sequences 32.2 us, 34.3 head by head), and
// where one round of loads does for as many partial results as a sequence may
// have (16 x 2048 tokens 21.8 and 22.7); otherwise it takes them one by one (1 x
// 8192 tokens 13.7 us, 15.7 together; of 256 channels 18.0 and 21.5).
void plan_attend(Attend& a, int64_t tokens) {
    const int64_t pairs = (int64_t)a.batch * a.c.kv_heads * a.head_tiles;
    const int dp = padded_dim(a.c.dim);
    const int waves = attend_waves(dp, a.dtype);
    const int64_t units = (tokens + kUnit - 1) / kUnit;
    const int64_t cus = device_cus(), at_once = cus * waves;
    a.wide = waves > 1 && pairs <= cus && 4 * pairs >= cus && units > 4 &&
             tokens <= 4 * 32 * group_waves(dp, a.dtype, true);
    a.whole = a.wide || units <= 4 || (units <= 8 && pairs >= cus) ||
              (units <= 16 && 2 * pairs >= at_once);
    const int64_t n = a.whole ? pairs : std::min(pairs * units, at_once);
    a.blocks = (int32_t)std::max(n, (int64_t)1);
    const int heads = std::min(a.group, 16);
    a.few = pairs >= cus || heads * (a.c.dim >> 2) * units <= kDeep * kThreads
                ? heads : 1;
    const int64_t parts = 2 * a.blocks * part_bytes(a.c.dim);
    a.workspace = a.whole || pairs == 0 ? 0 : parts + 8 * pairs;
}

hipError_t launch_attend(const Attend& a, hipStream_t st) {
    const int dp = padded_dim(a.c.dim);
    const hipError_t e = dp == 256   ? launch_attend_dp<256>(a, st)
                         : dp == 128 ? launch_attend_dp<128>(a, st)
                                     : launch_attend_dp<64>(a, st);
    if (e != hipSuccess || a.whole) return e;
    const int32_t pairs = a.batch * a.c.kv_heads * a.head_tiles;
    const int32_t slices = (std::min(a.group, 16) + a.few - 1) / a.few;
    return launch(join_kernel, pairs * slices, kThreads, st, a);
}

}  // namespace bscache

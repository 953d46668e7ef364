// Internal declarations shared by the HIP sources of libbscache.so.  The
// public interface is include/bscache.h.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "bs_internal.h"   // FastDiv

namespace bscache {

using bs::FastDiv;

// ---- the cache as the kernels see it ---------------------------------------

struct Pages {
    uint8_t* codes[2];        // keys, values
    uint32_t* steps[2];       // s in the low half, z in the high one
    uint32_t pages;
    int32_t kv_heads, page_tokens, dim;
    int32_t bits[2];
    uint32_t slots;           // pages * page_tokens
    FastDiv by_page;          // by page_tokens
};

// Row number (in units of rows) of a slot's first head, and the distance of
// its heads, are page * kv_heads * page_tokens + place and page_tokens.
__device__ __forceinline__ int64_t row_of(const Pages& c, uint32_t page,
                                          int32_t head, uint32_t place) {
    return ((int64_t)page * c.kv_heads + head) * c.page_tokens + place;
}

// ---- element types (the values of bscache_dtype) ---------------------------

constexpr int kF32 = 0, kF16 = 1, kBF16 = 2;

__device__ __forceinline__ float bits_f32(uint32_t u) {
    return __builtin_bit_cast(float, u);
}
__device__ __forceinline__ uint32_t f32_bits(float f) {
    return __builtin_bit_cast(uint32_t, f);
}
// s and z of a row's steps word
__device__ __forceinline__ float step_of(uint32_t w) { return bits_f32(w << 16); }
__device__ __forceinline__ float offset_of(uint32_t w) {
    return bits_f32(w & 0xFFFF0000u);
}

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8v __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Two float32 rounded (half to even) to float16 or bfloat16, in one word.
template <int T>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (T == kF16) {
        const half2v h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(uint32_t, h);
    } else {
        typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
        const bf2 h = {(__bf16)a, (__bf16)b};
        return __builtin_bit_cast(uint32_t, h);
    }
}

// The two values of a word of float16 or bfloat16.
template <int T>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b) {
    if constexpr (T == kF16) {
        const half2v h = __builtin_bit_cast(half2v, w);
        a = (float)h[0];
        b = (float)h[1];
    } else {
        a = bits_f32(w << 16);
        b = bits_f32(w & 0xFFFF0000u);
    }
}

// Eight consecutive elements, in registers as they are stored.
template <int T>
struct Eight {
    u32x4 w[T == kF32 ? 2 : 1];
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const u32x4* p = reinterpret_cast<const u32x4*>(
            static_cast<const uint8_t*>(base) + at * (T == kF32 ? 4 : 2));
        w[0] = p[0];
        if constexpr (T == kF32) w[1] = p[1];
    }
    __device__ __forceinline__ void clear() {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (T == kF32) w[1] = u32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ float get(int i) const {
        if constexpr (T == kF32) return bits_f32(w[i >> 2][i & 3]);
        float a, b;
        unpack2<T>(w[0][i >> 1], a, b);
        return i & 1 ? b : a;
    }
};

// ---- kernel launch ---------------------------------------------------------

template <typename P>
struct Same {
    using type = P;
};
// The arguments convert to the kernel's parameter types.
template <typename... P>
hipError_t launch(void (*fn)(P...), uint32_t blocks, uint32_t threads,
                  hipStream_t st, typename Same<P>::type... args) {
    void* argv[] = {(void*)&args...};
    return hipLaunchKernel((const void*)fn, dim3(blocks), dim3(threads), argv,
                           0, st);
}

// Workgroups of kBlock that a launch may have: the grid of all threads has 32
// bits, and so has a thread's number.
constexpr int kBlock = 256;
constexpr int64_t kMostBlocks = ((int64_t)1 << 32) / kBlock - 1;

// ---- launchers (each returns hipSuccess or the launch error) ---------------

// Compute units of the current device (cached per device).
int device_cus();

// Whether write and read launch so many tokens' rows at once.
bool rows_fit(const Pages& c, int64_t tokens);

hipError_t launch_write(const Pages& c, const void* k, const void* v,
                        int64_t k_stride, int64_t v_stride, int dtype,
                        const int32_t* slots, int64_t tokens, hipStream_t st);

hipError_t launch_read(const Pages& c, const int32_t* slots, int64_t tokens,
                       void* k, void* v, int dtype, hipStream_t st);

// One attention call, as the kernels see it.
struct Attend {
    Pages c;
    const void* q;
    const int32_t* table;
    const int32_t* lengths;
    void* out;
    float* lse;
    float* parts;             // workspace: two slots of partials a workgroup
    int64_t q_stride;
    int32_t batch, heads, group;
    int32_t head_tiles;       // tiles of up to 16 query heads of a kv head
    int32_t max_pages, max_len, window, dtype;
    float scale;
    bool whole;               // every pair is one workgroup's
    bool wide;                // of as many waves as a CU holds (whole too)
    int32_t blocks;           // workgroups
    int32_t few;              // query heads of a workgroup of the join
    int64_t workspace;        // bytes
};

// Channels that the attention kernel for a row of dim channels is made for.
constexpr int padded_dim(int dim) {
    return dim > 128 ? 256 : dim > 64 ? 128 : 64;
}

// Waves of a SIMD that the attention kernel for dp padded channels and a type
// leaves room for (its registers), and workgroups of a CU.
constexpr int attend_waves(int dp, int dtype) {
    return (dp == 64 ? 4 : dp == 128 ? 3 : 2) - (dtype == kF32 ? 1 : 0);
}

// Waves of a workgroup: 4, or all that a CU holds.
constexpr int group_waves(int dp, int dtype, bool wide) {
    return wide ? 4 * attend_waves(dp, dtype) : 4;
}

// Tokens of a unit: what the 4 waves of a workgroup take in one step.
constexpr int kUnit = 128;

// Chooses `whole`, `wide`, `blocks`, `few` and the workspace for a call whose
// longest sequence spans `tokens` tokens.
void plan_attend(Attend& a, int64_t tokens);

hipError_t launch_attend(const Attend& a, hipStream_t st);

}  // namespace bscache

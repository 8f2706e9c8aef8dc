// serve.cuh -- shared by the attention operators (prompt.cuh, token.cuh) and the
// paged cache under them (pages.cu).
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace opattr {

// What these operators find wrong on the device, kept in a word of the context
// until opattr_check asks for it: unlike the join's calls they do not wait.
enum ServeErr : unsigned {
    SERVE_INVALID = 1u,   // an offset, sequence, length or page that is out of range
    SERVE_PAGES = 2u,     // no free page left
    SERVE_TIMEOUT = 4u,   // a bounded wait gave up
};

// Device state of the context's operators, made by the first of their calls.
struct Serve {
    unsigned *err = nullptr;         // ServeErr bits, sticky; at word 16 the prompts' count of work items drawn
    uint32_t *tickets = nullptr;     // arrivals at each block's cut results; zero between launches
    unsigned prompt_room = 0;        // variants of the prompt kernel that have their shared memory
    // OPATTR_FAULT=prompt:N in the environment of a context's first call: in the first prompt
    // launch, every block's copies end before the N-th tile; N is SILENT_PARTS: one warp in four does
    // not come where parts are joined.  To exercise the waits' limit without a GPU fault.
    int silent = 0;
};
constexpr int SILENT_PARTS = -1;

constexpr int TICKETS = 4096;        // at most four blocks an SM, or their sixteen warps, count in them
constexpr int ALL_TICKETS = 3 * TICKETS;   // and in two more each, where parts are joined in groups
// Entries of a cache call: loops over them step past the last one by a block of threads at most, in 32 bits.
constexpr int32_t MOST_SEQS = INT32_MAX - 1024;
opattr_status serve_ready(Ctx &c, Serve &s);
void serve_free(Serve &s);

template <typename T>
struct Type2;
template <>
struct Type2<__nv_bfloat16> {
    static __device__ __forceinline__ float2 up(uint32_t x) {
        return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
    }
    // two values, each rounded to nearest even; `lo` in the low half
    static __device__ __forceinline__ uint32_t down(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    // 0 x + sum, for both values
    static __device__ __forceinline__ uint32_t add_zeros(uint32_t x, uint32_t sum) {
        uint32_t r;
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(sum));
        return r;
    }
};
template <>
struct Type2<__half> {
    static __device__ __forceinline__ float2 up(uint32_t x) {
        return __half22float2(*reinterpret_cast<const __half2 *>(&x));
    }
    static __device__ __forceinline__ uint32_t down(float lo, float hi) {
        uint32_t r;
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    static __device__ __forceinline__ uint32_t add_zeros(uint32_t x, uint32_t sum) {
        uint32_t r;
        asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(x), "r"(0u), "r"(sum));
        return r;
    }
};

// 2^x, to 2 ulp of the special function unit; 2^-inf is 0.
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

// The sequence of row `t`: offsets[b] <= t < offsets[b + 1], with 0 <= t < offsets[n].
__device__ __forceinline__ int seq_of_row(const int32_t *offsets, int n, int t) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (offsets[mid] <= t) lo = mid;
        else hi = mid;
    }
    return lo;
}

// A cache whose pages hold 8 bits, else NULL (then what follows the struct is not its own).
inline const opattr_cache8 *cache8(const opattr_cache *kv) {
    return kv->dtype == OPATTR_E4M3 ? reinterpret_cast<const opattr_cache8 *>(kv) : nullptr;
}

// Views with 16-byte rows: every operator moves rows by 16 bytes.
bool rows_ok(const opattr_rows &r, int64_t tokens, int heads, int dim);

}  // namespace opattr

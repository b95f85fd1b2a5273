// Shared by the two kernels of attention over the 4-bit store (fi_attend.cu, fi_attend_prompt.cu).
#pragma once

#include <cfloat>

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "fi_internal.cuh"

namespace fi {

constexpr float kMinScale = 0x1p-40f;      // smallest scale append stores
constexpr float kNoMax = -FLT_MAX;         // maximum of nothing
constexpr float kStart = 7.f, kMost = 15.f;   // log2 of the largest weight: as it is set, and as it may become
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttendParams {
    const void *q;
    void *out;
    float *lse;
    const int32_t *lens, *block_table, *row_idx, *batch_count, *cu_tokens, *granted;
    const unsigned char *k_codes, *v_codes;
    const uint32_t *k_meta, *v_meta;
    float *partial;
    uint32_t *tickets;
    int32_t *status;
    long long q_ts, q_hs, out_ts, out_hs;             // elements
    long long hs, mhs;                                // pools: strides of heads,
    uint32_t ps, ts, mps, mts;                        // of pages and of tokens (codes: 16 bytes, meta: pairs)
    long long table_ld;
    int rows, max_blocks, batch_max, max_tokens, window;
    int num_pages, page_shift, kv_heads, group;
    float scale_log2;                                 // scale * log2(e)
    long long wait_limit;                             // SM cycles
};

template <bool B>
struct Bool {
    static constexpr bool value = B;
};

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Natural logarithm of 2^top sum, a softmax sum.  Where values have small scales (or a tile a large power) top and the sum's exponent
// are large and cancel, so they are added up before the logarithm of the rest comes to them.
__device__ __forceinline__ float log_sum(float top, float sum) {
    if (sum == 0.f) return -INFINITY;
    if (!(sum >= FLT_MIN && sum < INFINITY)) return (top + log2f(sum)) * kLn2;
    const uint32_t bits = __float_as_uint(sum);
    return (top + (float)((int)(bits >> 23) - 127) + log2f(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u))) * kLn2;
}

__device__ __forceinline__ float meta_scale(uint32_t m) { return __uint_as_float(m << 16); }
__device__ __forceinline__ float meta_offset(uint32_t m) { return __uint_as_float(m & 0xffff0000u); }

__device__ __forceinline__ uint32_t smem_at(const void *p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }

// few rows per key head: any type, any head size (fi_attend.cu); many rows of bf16 queries (fi_attend_prompt.cu)
bool prompt_kernel_serves(const fi_kv *kv, const AttendParams &p, int dtype, long long queries);
fi_status_t prepare_attend_prompt(const fi_kv *kv);
fi_status_t launch_attend_prompt(const fi_kv *kv, const AttendParams &p, long long rows, cudaStream_t stream);

}  // namespace fi

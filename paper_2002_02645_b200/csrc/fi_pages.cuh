// Shared by the kernels of the page tables (fi_kv.cu, fi_pages_share.cu).
#pragma once

#include "fi_internal.cuh"

struct fi_pages {
    fi_pages_config_t cfg;
    int sm_count;
    uint32_t *ticket;   // [1] CTAs of the running call that are done; the last one puts it back to 0
    int32_t *segments;  // [kPageSegments] fi_pages_free: pages of each 256 that lost their last owner; 0 between calls
};

namespace fi {

constexpr int kPageSegments = 4096, kSegmentShift = 8;   // of 256 pages each

cudaError_t prepare_pages_share();    // one-time set-up of the kernels of fi_pages_share.cu on the current device

namespace {

constexpr int kPageThreads = 1024;
constexpr int kPageMaxBatch = 8192;
constexpr int kRefused = -2147483647 - 1;
constexpr int kPageItems = kPageMaxBatch / kPageThreads;   // requests per thread, at most

// Exclusive sum over the block of one value per thread; *total receives the sum.  64 bits: lengths come from the device
// unchecked, and their sum must not wrap.
__device__ long long block_exclusive(long long v, long long *total) {
    __shared__ long long warp_sum[kPageThreads / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    long long inc = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, inc, d);
        if (lane >= d) inc += o;
    }
    if (lane == 31) warp_sum[warp] = inc;
    __syncthreads();
    // every warp adds up the warps' sums for itself: one barrier less than handing them back
    long long w = lane < warps ? warp_sum[lane] : 0;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, w, d);
        if (lane >= d) w += o;
    }
    const long long before = warp ? __shfl_sync(0xffffffffu, w, warp - 1) : 0;
    *total = __shfl_sync(0xffffffffu, w, 31);
    __syncthreads();   // the next call writes warp_sum again
    return before + inc - v;
}

__device__ __forceinline__ int clamp_int(long long v) { return v > 2147483647ll ? 2147483647 : (int)v; }

// last i in [0, n) with first[i] <= x, for non-decreasing first[] with first[0] <= x
__device__ __forceinline__ int find_last(const int *first, int n, int x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// True in the last CTA of the grid to get here; everything the grid read before is then free to be overwritten.
__device__ bool last_cta(uint32_t *ticket) {
    if (gridDim.x == 1) {
        __syncthreads();
        return true;
    }
    __shared__ bool last;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        last = atomicAdd(ticket, 1u) == gridDim.x - 1;
        if (last) *ticket = 0;
        __threadfence();
    }
    __syncthreads();
    return last;
}

// lens_out = lens, unless they are one array: each CTA copies its share before the last one enters the new lengths.  The loads
// are issued at the start of the kernel and stored (put) when their values are there anyway.
struct LensCopy {
    int v[4];
    int first, threads, rows;

    __device__ __forceinline__ void get(const int32_t *lens, const int32_t *lens_out, int rows_) {
        threads = gridDim.x * blockDim.x;
        first = blockIdx.x * blockDim.x + threadIdx.x;
        rows = lens_out == lens ? 0 : rows_;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e * (long long)threads < rows) v[e] = lens[first + e * threads];
    }

    __device__ __forceinline__ void put(const int32_t *lens, int32_t *lens_out) const {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (first + e * (long long)threads < rows) lens_out[first + e * threads] = v[e];
        for (long long r = first + 4ll * threads; r < rows; r += threads) lens_out[r] = lens[r];
    }
};

__device__ __forceinline__ int actual_count(const int32_t *count_dev, int most) {
    if (!count_dev) return most;
    const int c = *count_dev;
    return c < 0 ? 0 : c > most ? most : c;
}

}  // namespace
}  // namespace fi

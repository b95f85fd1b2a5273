// Page tables of a layer's key/value store, and the store itself in 4 bits (the attention that reads it is in
// fi_attend.cu).
#include <cfloat>
#include <new>

#include <cuda_bf16.h>

#include "fi_pages.cuh"

namespace fi {
namespace {

// The step of the tables.  Every CTA forms both sums (tokens, then wanted pages) over all requests for itself: up to
// 8,192 lengths from L2 cost less than a second launch, and one CTA is all that a decode step needs.  The tokens are
// then dealt out, four neighbours per thread, which mostly share their request (found in the sums by binary search in
// shared memory) and their page; a token that opens a new page also writes the table entry.  Bound by the 12 bytes
// written per token for prompts, and by the chain of loads and block sums for a decode step.  Lengths and the free count
// are committed by the last CTA to finish, so they may be updated in place.
// ITEMS: most requests per thread (1 keeps the code short: a decode step also waits for its instructions).
template <int ITEMS>
__global__ void __launch_bounds__(kPageThreads) pages_extend_kernel(fi_pages_extend_t a, int page_shift, int max_blocks,
                                                                    bool wide, uint32_t *ticket) {
    extern __shared__ int smem[];
    int *const s_cu = smem;                       // first token of each request
    int *const s_first = s_cu + a.batch_max;      // place of its first page in the free stack, or kRefused
    int *const s_have = s_first + a.batch_max;
    int *const s_row = s_have + a.batch_max;
    __shared__ int s_taken;
    if (threadIdx.x == 0) s_taken = 0;
    const int items = ITEMS == 1 ? 1 : (a.batch_max + blockDim.x - 1) / blockDim.x;
    const int i0 = threadIdx.x * items;
    int have[ITEMS], fresh[ITEMS], rows[ITEMS];
    // rows and lengths are loaded for the largest batch, beside the actual one
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        rows[e] = -1;
        if (e < items && i < a.batch_max) {
            rows[e] = a.row_idx ? a.row_idx[i] : i;
            fresh[e] = a.new_lens ? a.new_lens[i] : 1;
        }
    }
    LensCopy copy;
    copy.get(a.lens, a.lens_out, a.rows);
    const int n = actual_count(a.batch_count, a.batch_max);
    const int free_count = min(max(*a.free_count, 0), a.num_pages);
    long long sum = 0;
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        const bool ok = rows[e] >= 0 && rows[e] < a.rows;
        have[e] = ok ? a.lens[rows[e]] : 0;
        if (!ok || have[e] < 0 || fresh[e] < 0 || i >= n) fresh[e] = 0;
        if (have[e] < 0) have[e] = 0;
        if (!ok) rows[e] = -1;
        if (e < items && i < n) {
            s_row[i] = rows[e];
            s_have[i] = have[e];
            sum += fresh[e];
        }
    }
    long long tokens;
    long long cu = block_exclusive(sum, &tokens);
    long long need_sum = 0;
    int need[ITEMS];
    const long long page_mask = (1ll << page_shift) - 1;
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        need[e] = -1;
        if (e < items && i < n) {
            s_cu[i] = clamp_int(cu);
            if (blockIdx.x == 0) a.cu_tokens[i] = clamp_int(cu);
            cu += fresh[e];
            const long long had = (have[e] + page_mask) >> page_shift, want = (have[e] + (long long)fresh[e] + page_mask) >> page_shift;
            if (want <= max_blocks && cu <= a.max_tokens) {
                need[e] = (int)(want - had);
                need_sum += need[e];
            }
        }
    }
    long long pages;
    long long before = block_exclusive(need_sum, &pages);
    int taken = 0;
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        if (e < items && i < n) {
            const bool given = need[e] >= 0 && (need[e] == 0 || before + need[e] <= free_count);
            // a request that needs no page may stand behind any number of refused ones: its place is not used
            s_first[i] = !given ? kRefused : need[e] == 0 ? 0 : free_count - 1 - (int)before;
            if (need[e] > 0) before += need[e];
            if (given) taken += need[e];
            if (blockIdx.x == 0) a.granted[i] = given ? fresh[e] : 0;
            fresh[e] = given ? fresh[e] : 0;
        }
    }
    if (taken > 0) atomicAdd(&s_taken, taken);
    copy.put(a.lens, a.lens_out);
    __syncthreads();
    if (blockIdx.x == 0) {
        for (int i = n + threadIdx.x; i <= a.batch_max; i += blockDim.x) {
            a.cu_tokens[i] = clamp_int(tokens);
            if (i < a.batch_max) a.granted[i] = 0;
        }
    }
    const long long step = (long long)gridDim.x * blockDim.x * 4;
    for (long long t0 = ((long long)blockIdx.x * blockDim.x + threadIdx.x) * 4; t0 < a.max_tokens; t0 += step) {
        long long slot[4] = {-1, -1, -1, -1};
        int pos[4] = {-1, -1, -1, -1};
        if (t0 < tokens) {
            // requests without tokens share their first token with the next one: the last of them owns it
            int i = find_last(s_cu, n, (int)t0);
            int end = i + 1 < n ? s_cu[i + 1] : clamp_int(tokens);
            const int first0 = s_first[i], p0 = s_have[i] + ((int)t0 - s_cu[i]), place0 = p0 & (int)page_mask;
            if (t0 + 4 <= end && first0 != kRefused && place0 + 4 <= page_mask + 1) {
                // the usual four: one request, one page
                const int block = p0 >> page_shift, had = (int)((s_have[i] + page_mask) >> page_shift);
                int32_t *const entry = a.block_table + (long long)s_row[i] * a.table_ld + block;
                const int page = block >= had ? a.free_pages[first0 - (block - had)] : *entry;
                if (block >= had && place0 == 0) *entry = page;
                const long long slot0 = ((long long)page << page_shift) + place0;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    pos[e] = p0 + e;
                    slot[e] = page >= 0 ? slot0 + e : -1;
                }
            } else {
#pragma unroll 1
                for (int e = 0; e < 4 && t0 + e < tokens; ++e) {
                    const int t = (int)t0 + e;
                    while (t >= end) {
                        ++i;
                        end = i + 1 < n ? s_cu[i + 1] : clamp_int(tokens);
                    }
                    const long long p = (long long)s_have[i] + (t - s_cu[i]);
                    long long sl = -1;
                    const int first = s_first[i];
                    if (first != kRefused) {
                        const int block = (int)(p >> page_shift), had = (int)((s_have[i] + page_mask) >> page_shift);
                        int32_t *const entry = a.block_table + (long long)s_row[i] * a.table_ld + block;
                        const int page = block >= had ? a.free_pages[first - (block - had)] : *entry;
                        if (block >= had && (p & page_mask) == 0) *entry = page;
                        if (page >= 0) sl = ((long long)page << page_shift) + (p & page_mask);
                    }
                    const int ps = clamp_int(p);
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (x == e) {
                            slot[x] = sl;
                            pos[x] = ps;
                        }
                }
            }
        }
        if (wide && t0 + 4 <= a.max_tokens) {
            reinterpret_cast<longlong2 *>(a.slot_map + t0)[0] = make_longlong2(slot[0], slot[1]);
            reinterpret_cast<longlong2 *>(a.slot_map + t0)[1] = make_longlong2(slot[2], slot[3]);
            *reinterpret_cast<int4 *>(a.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (t0 + e < a.max_tokens) {
                    a.slot_map[t0 + e] = slot[e];
                    a.positions[t0 + e] = pos[e];
                }
        }
    }
    if (!last_cta(ticket)) return;
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        if (e < items && i < n && s_row[i] >= 0 && fresh[e] > 0) a.lens_out[s_row[i]] = have[e] + fresh[e];
    }
    if (threadIdx.x == 0) *a.free_count_out = free_count - s_taken;
}

struct ReleaseParams {
    const int32_t *row_idx, *batch_count, *lens, *block_table, *free_count;
    int32_t *free_pages, *lens_out, *free_count_out;
    long long table_ld;
    int batch_max, rows, num_pages, max_blocks, page_shift;
};

// The way back: the pages of the listed rows are copied behind the free stack, in list order.
template <int ITEMS>
__global__ void __launch_bounds__(kPageThreads) pages_release_kernel(ReleaseParams a, uint32_t *ticket) {
    extern __shared__ int smem[];
    int *const s_cu = smem;
    int *const s_row = s_cu + a.batch_max;
    LensCopy copy;
    copy.get(a.lens, a.lens_out, a.rows);
    const int n = actual_count(a.batch_count, a.batch_max);
    const int free_count = min(max(*a.free_count, 0), a.num_pages);
    const int items = ITEMS == 1 ? 1 : (a.batch_max + blockDim.x - 1) / blockDim.x;
    const int i0 = threadIdx.x * items;
    int used[ITEMS];
    long long sum = 0;
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        used[e] = 0;
        if (e < items && i < n) {
            const int row = a.row_idx[i];
            const bool ok = row >= 0 && row < a.rows;
            if (ok) {
                const long long len = max(a.lens[row], 0);
                used[e] = (int)min((len + (1ll << a.page_shift) - 1) >> a.page_shift, (long long)a.max_blocks);
            }
            s_row[i] = ok ? row : -1;
            sum += used[e];
        }
    }
    long long pages;
    long long cu = block_exclusive(sum, &pages);
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
        const int i = i0 + e;
        if (e < items && i < n) {
            s_cu[i] = clamp_int(cu);
            cu += used[e];
        }
    }
    __syncthreads();
    copy.put(a.lens, a.lens_out);
    if (pages > a.num_pages - free_count) pages = a.num_pages - free_count;   // a row listed twice: nothing is written past the stack
    const long long step = (long long)gridDim.x * blockDim.x;
    for (long long p = (long long)blockIdx.x * blockDim.x + threadIdx.x; p < pages; p += step) {
        const int i = find_last(s_cu, n, (int)p);
        a.free_pages[free_count + p] = a.block_table[(long long)s_row[i] * a.table_ld + ((int)p - s_cu[i])];
    }
    if (!last_cta(ticket)) return;
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        if (s_row[i] >= 0) a.lens_out[s_row[i]] = 0;
    if (threadIdx.x == 0) *a.free_count_out = free_count + (int)pages;
}

// ------------------------------------------------------------------------------------------------------- 4-bit append

struct AppendParams {
    const void *k, *v;
    const int64_t *slot_map;
    const int32_t *tokens_dev;
    void *k_stored, *v_stored;
    long long k_ts, k_hs, v_ts, v_hs;          // elements
    unsigned char *k_codes, *v_codes;
    uint32_t *k_meta, *v_meta;
    long long ps, hs, ts, mps, mhs, mts;
    long long rows, slots;                     // tokens * heads; slots of the pool
    int heads, page_shift;
    int32_t *status;
};

template <bool BF16>
__device__ __forceinline__ void store16(void *base, long long elem, const float (&x)[16]) {
    if constexpr (BF16) {
        uint4 *p = reinterpret_cast<uint4 *>(static_cast<char *>(base) + elem * 2);
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = reinterpret_cast<const uint32_t &>(h);
        }
        p[0] = make_uint4(w[0], w[1], w[2], w[3]);
        p[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + elem);
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i] = make_float4(x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]);
    }
}

// largest bf16 value not above x (as fp32); the scale is rounded up by the same function on -x
__device__ __forceinline__ float bf16_down(float x) {
    const uint32_t bits = __float_as_uint(x), cut = bits & 0xffff0000u;
    return __uint_as_float(x < 0.f && bits != cut ? cut + 0x10000u : cut);
}

// two floats in one register pair, and the operations that take both at once
__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

constexpr float kRound = 12582912.f;           // adding 1.5 x 2^23 rounds to a whole number, ties to even, in the low bits
constexpr uint32_t kRoundBits = 0x4b400000u;

// 16 consecutive values of a vector: as they are in memory, their least and largest, and whether all are finite
template <bool BF16>
struct Values16 {
    uint4 w[BF16 ? 2 : 4];

    __device__ __forceinline__ void load(const void *base, long long elem) {
        const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + elem * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) w[i] = p[i];
    }

    __device__ __forceinline__ void widen(float (&x)[16]) const {
#pragma unroll
        for (int i = 0; i < (BF16 ? 2 : 4); ++i) {
            const uint32_t u[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (BF16) {
                    x[8 * i + 2 * e] = __uint_as_float(u[e] << 16);
                    x[8 * i + 2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
                } else {
                    x[4 * i + e] = __uint_as_float(u[e]);
                }
            }
        }
    }

    __device__ __forceinline__ void range(const float (&x)[16], float &lo, float &hi, bool &finite) const {
        if constexpr (BF16) {
            const uint32_t u[8] = {w[0].x, w[0].y, w[0].z, w[0].w, w[1].x, w[1].y, w[1].z, w[1].w};
            const auto h = [&](int i) { return reinterpret_cast<const __nv_bfloat162 &>(u[i]); };
            const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
            __nv_bfloat162 least = h(0), most = h(0), none = __hmul2(h(0), zero);
#pragma unroll
            for (int i = 1; i < 8; ++i) {
                least = __hmin2(least, h(i));
                most = __hmax2(most, h(i));
                none = __hfma2(h(i), zero, none);      // NaN as soon as a value is one or is infinite
            }
            lo = fminf(__low2float(least), __high2float(least));
            hi = fmaxf(__low2float(most), __high2float(most));
            finite = __low2float(none) + __high2float(none) == 0.f;
        } else {
            float none = 0.f;
            lo = hi = x[0];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                lo = fminf(lo, x[i]);
                hi = fmaxf(hi, x[i]);
                none = fmaf(x[i], 0.f, none);
            }
            finite = none == 0.f;
        }
    }
};

// One vector held by LANES neighbouring lanes, 16 values each (lanes past D / 16 hold none).
// A code is round(a / scale), ties to even, of the correctly rounded quotient.  With the correctly rounded reciprocal r of the
// scale, q = a r and q + r (a - q scale) is that quotient (Markstein, "Computation of elementary functions on the IBM RISC
// System/6000 processor", 1990): two operations more than the product, and no division, as long as r is a normal number.  The
// scale has 8 significant bits, so a - q scale is exact, and no quotient lies within 2^-9 of a last place of a tie.
// What bounds it: 16,384 tokens of 8 heads of 128 (bf16, k and v) took 58.8 us with a division per value, 37.4 with one only
// near a tie, and take 28.7 us, 5.3 TB/s; the extremes are found on the bf16 values, two at a time, and sums and products on pairs.
template <int D, int LANES, bool BF16>
__device__ __forceinline__ void pack_vector(const Values16<BF16> &v, bool active, bool write, unsigned char *codes, uint32_t *meta,
                                            void *stored, long long stored_at) {
    float x[16], lo = FLT_MAX, hi = -FLT_MAX;
    if (active) {
        bool finite;
        v.widen(x);
        v.range(x, lo, hi, finite);
        if (!finite) lo = -INFINITY;           // travels through the minimum below, and -inf marks the vector
    }
    const int lane = (threadIdx.x & 31) & (LANES - 1);
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, d));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, d));
    }
    if (!active) return;
    float offset = bf16_down(lo);
    float scale = fmaxf(-bf16_down(-__fdiv_rn(__fsub_rn(hi, offset), 15.f)), 0x1p-40f);
    uint32_t packed[2] = {0u, 0u};
    if (lo >= -FLT_MAX && offset >= -FLT_MAX && scale <= FLT_MAX) {
        const uint64_t off2 = pair(-offset, -offset), plus2 = pair(offset, offset), scale2 = pair(scale, scale), up2 = pair(kRound, kRound),
                       down2 = pair(-kRound, -kRound);
        const auto code2 = [&](int i, uint64_t quotient) {
            const uint64_t r = add2(quotient, up2);
            float r0, r1;
            unpair(r, r0, r1);
            packed[i >> 3] += (__float_as_uint(r0) - kRoundBits) << (4 * (i & 7));
            packed[i >> 3] += (__float_as_uint(r1) - kRoundBits) << (4 * (i & 7) + 4);
            unpair(fma2(add2(r, down2), scale2, plus2), x[i], x[i + 1]);
        };
        if (scale <= 0x1p100f) {
            const float inv = __frcp_rn(scale);
            const uint64_t inv2 = pair(inv, inv), minus2 = pair(-scale, -scale);
#pragma unroll
            for (int i = 0; i < 16; i += 2) {
                const uint64_t a = add2(pair(x[i], x[i + 1]), off2), q = mul2(a, inv2);
                code2(i, fma2(fma2(q, minus2, a), inv2, q));
            }
        } else {                               // the reciprocal is hardly a normal number
#pragma unroll
            for (int i = 0; i < 16; i += 2)
                code2(i, pair(__fdiv_rn(__fsub_rn(x[i], offset), scale), __fdiv_rn(__fsub_rn(x[i + 1], offset), scale)));
        }
    } else {
        offset = __uint_as_float(0x7fc00000u);
        scale = 1.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = offset;
    }
    if (write) {
        *reinterpret_cast<uint2 *>(codes + lane * 8) = make_uint2(packed[0], packed[1]);
        if (lane == 0) *meta = (__float_as_uint(scale) >> 16) | (__float_as_uint(offset) & 0xffff0000u);
    }
    if (stored) store16<BF16>(stored, stored_at + lane * 16, x);
}

// A group of LANES lanes packs the key and the value of one token and head: two independent 32-byte (bf16) loads per lane in
// flight, minimum and maximum by shuffles, 8 bytes of codes per lane.  One pass over the data; bound by its bytes.  Groups share
// nothing, so CTAs are small: with 256 threads the last group to end kept the place of the others (30.2 us, not 28.7).
constexpr int kAppendThreads = 64;

template <int D, bool BF16>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(AppendParams a) {
    constexpr int LANES = D <= 64 ? 4 : D <= 128 ? 8 : 16;
    const int lane = threadIdx.x & (LANES - 1);
    const long long row = ((long long)blockIdx.x * kAppendThreads + threadIdx.x) / LANES;
    const bool there = row < a.rows;
    const unsigned token = there ? (unsigned)row / (unsigned)a.heads : 0u;
    const int head = there ? (int)((unsigned)row - token * (unsigned)a.heads) : 0;
    const bool real = there && (!a.tokens_dev || (int)token < *a.tokens_dev);
    const bool active = real && lane < D / 16;
    Values16<BF16> k, v;
    if (active) {
        k.load(a.k, token * a.k_ts + head * a.k_hs + lane * 16);
        v.load(a.v, token * a.v_ts + head * a.v_hs + lane * 16);
    }
    const long long slot = real ? a.slot_map[token] : -1;
    if (slot >= a.slots && lane == 0 && head == 0) atomicOr(a.status, 1);
    const bool write = slot >= 0 && slot < a.slots;
    const long long page = write ? slot >> a.page_shift : 0, place = write ? slot & ((1ll << a.page_shift) - 1) : 0;
    const long long at = page * a.ps + head * a.hs + place * a.ts, mat = page * a.mps + head * a.mhs + place * a.mts;
    const long long stored_at = row * D;
    pack_vector<D, LANES, BF16>(k, active, write, a.k_codes + at, a.k_meta + mat, a.k_stored, stored_at);
    pack_vector<D, LANES, BF16>(v, active, write, a.v_codes + at, a.v_meta + mat, a.v_stored, stored_at);
}

template <int D>
void append_dispatch(const AppendParams &p, bool bf16, cudaStream_t stream) {
    constexpr int LANES = D <= 64 ? 4 : D <= 128 ? 8 : 16;
    const unsigned grid = (unsigned)((p.rows * LANES + kAppendThreads - 1) / kAppendThreads);
    if (bf16) kv_append_kernel<D, true><<<grid, kAppendThreads, 0, stream>>>(p);
    else kv_append_kernel<D, false><<<grid, kAppendThreads, 0, stream>>>(p);
}

int log2_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}

constexpr long long kKvWaitLimit = 8000000000ll;   // about 4 s

bool page_size_ok(int p) { return p >= 16 && p <= 1024 && (p & (p - 1)) == 0; }

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace
}  // namespace fi

using namespace fi;

extern "C" {

fi_status_t fi_pages_destroy(fi_pages_t *p) {
    if (!p) return FI_OK;
    DeviceGuard guard(p->cfg.device);
    cudaDeviceSynchronize();
    cudaFree(p->ticket);
    cudaFree(p->segments);
    delete p;
    return FI_OK;
}

fi_status_t fi_pages_create(const fi_pages_config_t *cfg, fi_pages_t **out) {
    if (out) *out = nullptr;
    if (!cfg || !out) {
        set_error("fi_pages_create: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (!page_size_ok(cfg->page_size) || cfg->max_blocks < 1 || (long long)cfg->max_blocks * cfg->page_size > 2147483647ll ||
        cfg->max_batch < 1 || cfg->max_batch > kPageMaxBatch || cfg->device < 0) {
        set_error("fi_pages_create: page_size a power of two in 16..1024, max_blocks >= 1 with max_blocks * page_size < 2^31, "
                  "max_batch in 1..%d", kPageMaxBatch);
        return FI_ERR_INVALID_ARG;
    }
    fi_pages *p = new (std::nothrow) fi_pages();
    if (!p) {
        set_error("fi_pages_create: out of host memory");
        return FI_ERR_OOM;
    }
    p->cfg = *cfg;
    DeviceGuard guard(cfg->device);
    cudaError_t e = guard.ok ? cudaSuccess : cudaErrorInvalidDevice;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&p->sm_count, cudaDevAttrMultiProcessorCount, cfg->device);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(pages_extend_kernel<kPageItems>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPageMaxBatch * 16);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(pages_release_kernel<kPageItems>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPageMaxBatch * 8);
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&p->ticket), sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMemset(p->ticket, 0, sizeof(uint32_t));
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&p->segments), kPageSegments * sizeof(int32_t));
    if (e == cudaSuccess) e = cudaMemset(p->segments, 0, kPageSegments * sizeof(int32_t));
    if (e == cudaSuccess) e = prepare_pages_share();
    if (e == cudaSuccess) e = cudaDeviceSynchronize();
    if (e != cudaSuccess) {
        const fi_status_t st = cuda_fail(e, "fi_pages_create");
        fi_pages_destroy(p);
        return st;
    }
    *out = p;
    return FI_OK;
}

fi_status_t fi_pages_extend(fi_pages_t *p, const fi_pages_extend_t *s, void *cuda_stream) {
    if (!p || !s) {
        set_error("fi_pages_extend: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (s->batch_max < 0 || s->batch_max > p->cfg.max_batch || s->max_tokens < 0 || s->rows < 0 || s->num_pages < 0 ||
        s->table_ld < p->cfg.max_blocks || (!s->row_idx && s->batch_max > s->rows)) {
        set_error("fi_pages_extend: batch %d outside 0..%d, a negative size, table_ld below max_blocks, or more requests than rows",
                  s->batch_max, p->cfg.max_batch);
        return FI_ERR_INVALID_ARG;
    }
    if ((s->rows > 0 && (!s->lens || !s->lens_out || !s->block_table)) || (s->num_pages > 0 && !s->free_pages) || !s->free_count ||
        !s->free_count_out || !s->cu_tokens || (s->batch_max > 0 && !s->granted) ||
        (s->max_tokens > 0 && (!s->slot_map || !s->positions))) {
        set_error("fi_pages_extend: null pointer (only row_idx, batch_count and new_lens may be)");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(p->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_pages_extend");
    int grid = s->max_tokens / 4096;   // below that the sums cost more than the tokens
    grid = grid < 1 ? 1 : grid > p->sm_count ? p->sm_count : grid;
    // a decode step of up to 256 requests: eight warps form the sums faster than 32
    const int threads = s->batch_max <= 256 && s->max_tokens <= 1024 && s->rows <= 1024 ? 256 : kPageThreads;
    const bool wide = aligned16(s->slot_map) && aligned16(s->positions);
    if (s->batch_max <= threads)
        pages_extend_kernel<1><<<grid, threads, (size_t)s->batch_max * 16, static_cast<cudaStream_t>(cuda_stream)>>>(
            *s, log2_of(p->cfg.page_size), p->cfg.max_blocks, wide, p->ticket);
    else
        pages_extend_kernel<kPageItems><<<grid, threads, (size_t)s->batch_max * 16, static_cast<cudaStream_t>(cuda_stream)>>>(
            *s, log2_of(p->cfg.page_size), p->cfg.max_blocks, wide, p->ticket);
    count_launch();
    return check_launch("fi_pages_extend");
}

fi_status_t fi_pages_release(fi_pages_t *p, const int32_t *row_idx, int32_t batch_max, const int32_t *batch_count,
                             const int32_t *lens, int32_t rows, const int32_t *block_table, int64_t table_ld,
                             int32_t *free_pages, int32_t num_pages, const int32_t *free_count, int32_t *lens_out,
                             int32_t *free_count_out, void *cuda_stream) {
    if (!p || (rows > 0 && (!lens || !block_table || !lens_out)) || (num_pages > 0 && !free_pages) || !free_count || !free_count_out ||
        (batch_max > 0 && !row_idx)) {
        set_error("fi_pages_release: null argument (only batch_count may be)");
        return FI_ERR_INVALID_ARG;
    }
    if (batch_max < 0 || batch_max > p->cfg.max_batch || rows < 0 || num_pages < 0 || table_ld < p->cfg.max_blocks) {
        set_error("fi_pages_release: batch %d outside 0..%d, a negative size, or table_ld below max_blocks", batch_max, p->cfg.max_batch);
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(p->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_pages_release");
    ReleaseParams a = {row_idx, batch_count, lens, block_table, free_count, free_pages, lens_out, free_count_out, table_ld,
                       batch_max, rows, num_pages, p->cfg.max_blocks, log2_of(p->cfg.page_size)};
    long long grid = (long long)batch_max * p->cfg.max_blocks / 16384;   // an upper bound of the pages, rarely met
    grid = grid < 1 ? 1 : grid > p->sm_count ? p->sm_count : grid;
    const int threads = batch_max <= 256 && rows <= 1024 ? 256 : kPageThreads;
    if (batch_max <= threads)
        pages_release_kernel<1><<<(int)grid, threads, (size_t)batch_max * 8, static_cast<cudaStream_t>(cuda_stream)>>>(a, p->ticket);
    else
        pages_release_kernel<kPageItems><<<(int)grid, threads, (size_t)batch_max * 8, static_cast<cudaStream_t>(cuda_stream)>>>(a, p->ticket);
    count_launch();
    return check_launch("fi_pages_release");
}

fi_status_t fi_kv_destroy(fi_kv_t *kv) {
    if (!kv) return FI_OK;
    DeviceGuard guard(kv->cfg.device);
    cudaDeviceSynchronize();
    cudaFree(kv->status_dev);
    cudaFree(kv->scratch);
    delete kv;
    return FI_OK;
}

fi_status_t fi_kv_create(const fi_kv_config_t *cfg, fi_kv_t **out) {
    if (out) *out = nullptr;
    if (!cfg || !out || !cfg->k_codes || !cfg->v_codes || !cfg->k_meta || !cfg->v_meta) {
        set_error("fi_kv_create: null argument");
        return FI_ERR_INVALID_ARG;
    }
    const int d = cfg->head_dim;
    if (!page_size_ok(cfg->page_size) || cfg->num_pages < 1 || (d != 64 && d != 128 && d != 192 && d != 256) ||
        cfg->kv_heads < 1 || cfg->q_heads < cfg->kv_heads || cfg->q_heads % cfg->kv_heads != 0 || cfg->q_heads > 65535 ||
        cfg->device < 0) {
        set_error("fi_kv_create: page_size a power of two in 16..1024, num_pages >= 1, head_dim 64, 128, 192 or 256, q_heads a "
                  "multiple of kv_heads");
        return FI_ERR_INVALID_ARG;
    }
    if (!aligned16(cfg->k_codes) || !aligned16(cfg->v_codes) || (reinterpret_cast<uintptr_t>(cfg->k_meta) & 3) != 0 ||
        (reinterpret_cast<uintptr_t>(cfg->v_meta) & 3) != 0 || cfg->page_stride % 16 != 0 || cfg->head_stride % 16 != 0 ||
        cfg->token_stride % 16 != 0 || cfg->page_stride < 0 || cfg->head_stride < 0 || cfg->token_stride < d / 2 ||
        cfg->meta_page_stride < 0 || cfg->meta_head_stride < 0 || cfg->meta_token_stride < 1 || cfg->page_stride > 2147483647ll ||
        cfg->token_stride > 2147483647ll / cfg->page_size || cfg->meta_page_stride > 2147483647ll ||
        cfg->meta_token_stride > 2147483647ll / cfg->page_size ||
        (double)cfg->num_pages * (double)cfg->page_stride + (double)cfg->page_size * (double)cfg->token_stride >= 16.0 * 4294967296.0 ||
        (double)cfg->num_pages * (double)cfg->meta_page_stride + (double)cfg->page_size * (double)cfg->meta_token_stride >= 4294967296.0) {
        set_error("fi_kv_create: codes and their strides must be multiples of 16 bytes, meta of 4, strides not negative, tokens "
                  "not overlapping, strides of pages and of page_size tokens below 2^31, pools of at most 64 GiB of codes and "
                  "16 GiB of meta");
        return FI_ERR_INVALID_ARG;
    }
    fi_kv *kv = new (std::nothrow) fi_kv();
    if (!kv) {
        set_error("fi_kv_create: out of host memory");
        return FI_ERR_OOM;
    }
    kv->cfg = *cfg;
    kv->wait_limit = kKvWaitLimit;
    kv->page_shift = log2_of(cfg->page_size);
    DeviceGuard guard(cfg->device);
    cudaError_t e = guard.ok ? cudaSuccess : cudaErrorInvalidDevice;
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&kv->sm_count, cudaDevAttrMultiProcessorCount, cfg->device);
    if (e == cudaSuccess) e = cudaMalloc(reinterpret_cast<void **>(&kv->status_dev), sizeof(int32_t));
    if (e == cudaSuccess) e = cudaMemset(kv->status_dev, 0, sizeof(int32_t));
    fi_status_t st = e == cudaSuccess ? prepare_attend(kv) : cuda_fail(e, "fi_kv_create");
    if (st == FI_OK) {
        e = cudaDeviceSynchronize();
        if (e != cudaSuccess) st = cuda_fail(e, "fi_kv_create");
    }
    if (st != FI_OK) {
        fi_kv_destroy(kv);
        return st;
    }
    *out = kv;
    return FI_OK;
}

fi_status_t fi_kv_set_wait_limit(fi_kv_t *kv, int64_t limit_cycles) {
    if (!kv || limit_cycles < 0 || limit_cycles > kKvWaitLimit) {
        set_error("fi_kv_set_wait_limit: null handle or limit outside 0..%lld cycles", kKvWaitLimit);
        return FI_ERR_INVALID_ARG;
    }
    kv->wait_limit = limit_cycles ? limit_cycles : kKvWaitLimit;
    return FI_OK;
}

fi_status_t fi_kv_poll_status(fi_kv_t *kv) {
    if (!kv) {
        set_error("fi_kv_poll_status: null handle");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(kv->cfg.device);
    int32_t word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpy(&word, kv->status_dev, sizeof word, cudaMemcpyDeviceToHost);
    if (e == cudaSuccess && word) e = cudaMemset(kv->status_dev, 0, sizeof word);
    if (e != cudaSuccess) return cuda_fail(e, "fi_kv_poll_status");
    if (word & 4) {
        set_error("fi_kv_poll_status: a bounded wait inside an attention kernel ran out");
        return FI_ERR_TIMEOUT;
    }
    if (word) {
        set_error("fi_kv_poll_status:%s%s", word & 1 ? " a slot past the pool was skipped by fi_kv_append;" : "",
                  word & 2 ? " a page number outside the pool was met by fi_kv_attend or fi_kv_copy_pages" : "");
        return FI_ERR_INVALID_ARG;
    }
    return FI_OK;
}

fi_status_t fi_kv_append(fi_kv_t *kv, const fi_kv_append_t *a, void *cuda_stream) {
    if (!kv || !a) {
        set_error("fi_kv_append: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (a->dtype != FI_F32 && a->dtype != FI_BF16) {
        set_error("fi_kv_append: dtype must be FI_F32 or FI_BF16");
        return FI_ERR_INVALID_ARG;
    }
    const long long rows = a->tokens * (long long)kv->cfg.kv_heads;
    if (a->tokens < 0 || a->tokens > 2147483647ll || rows > 2147483647ll) {
        set_error("fi_kv_append: tokens * kv_heads must lie in 0..2^31 - 1");
        return FI_ERR_INVALID_ARG;
    }
    if (a->tokens == 0) return FI_OK;
    if (!a->k || !a->v || !a->slot_map) {
        set_error("fi_kv_append: null pointer (only tokens_dev, k_stored and v_stored may be)");
        return FI_ERR_INVALID_ARG;
    }
    const int unit = a->dtype == FI_BF16 ? 8 : 4;
    const auto bad = [&](int64_t stride, int64_t count) { return count > 1 && (stride < 0 || stride % unit != 0); };
    if (!aligned16(a->k) || !aligned16(a->v) || !aligned16(a->k_stored) || !aligned16(a->v_stored) || bad(a->k_token_stride, a->tokens) ||
        bad(a->v_token_stride, a->tokens) || bad(a->k_head_stride, kv->cfg.kv_heads) || bad(a->v_head_stride, kv->cfg.kv_heads)) {
        set_error("fi_kv_append: vectors must start on 16-byte boundaries, strides must not be negative");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(kv->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_kv_append");
    const fi_kv_config_t &c = kv->cfg;
    AppendParams p = {a->k, a->v, a->slot_map, a->tokens_dev, a->k_stored, a->v_stored, a->k_token_stride, a->k_head_stride,
                      a->v_token_stride, a->v_head_stride, static_cast<unsigned char *>(c.k_codes),
                      static_cast<unsigned char *>(c.v_codes), static_cast<uint32_t *>(c.k_meta), static_cast<uint32_t *>(c.v_meta),
                      c.page_stride, c.head_stride, c.token_stride, c.meta_page_stride, c.meta_head_stride, c.meta_token_stride,
                      rows, (long long)c.num_pages << kv->page_shift, c.kv_heads, kv->page_shift, kv->status_dev};
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    const bool bf16 = a->dtype == FI_BF16;
    switch (c.head_dim) {
        case 64: append_dispatch<64>(p, bf16, stream); break;
        case 128: append_dispatch<128>(p, bf16, stream); break;
        case 192: append_dispatch<192>(p, bf16, stream); break;
        default: append_dispatch<256>(p, bf16, stream); break;
    }
    count_launch();
    return check_launch("fi_kv_append");
}

}  // extern "C"

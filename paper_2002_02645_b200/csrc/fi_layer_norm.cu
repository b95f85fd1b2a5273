// Norm of whole rows, by mean and variance or by root mean square, and its gradients.
//
//   n = (x - mean) r, r = 1 / sqrt(mean((x - mean)^2) + eps);  y = n w + b        (rms: mean taken as 0)
//   backward:  g = dy w;  dx = r (g - mean(g) - n mean(g n));  dw = sum dy n, db = sum dy        (rms: without mean(g))
//
// A row is held in registers by a warp or a part of one (up to 1,024 values) or by a CTA, so that it is read once, its deviations are squared after the
// mean is known, and it is written once: the bound is the traffic.  Nothing of the forward pass is kept for the gradients; mean
// and r come again from x, which they read anyway.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "fi_internal.cuh"

namespace fi {
namespace {

constexpr int kMaxDim = 16384;
// CTAs of a backward pass, at most: so many sums of both weight gradients are in the workspace
constexpr int max_partials(int dim) { return dim <= 2048 ? 640 : dim <= 4096 ? 320 : 160; }

__device__ int32_t g_layer_norm_status;   // 1: a bounded wait ran out

struct RowNormParams {
    const void *x, *dy;
    void *out;                         // y, or dx
    const float *weight, *bias;
    const int32_t *rows, *count;
    float *partial;                    // backward: [CTAs][2][dim]; nullable
    long long x_stride, dy_stride, out_stride, tokens, x_rows, wait_limit;
    int dim, rms;
    float eps, inv_dim;
};

// 8 values of a row (VEC), widened to fp32
template <bool F32>
struct Raw8 {
    uint4 w[F32 ? 2 : 1];
};
template <bool F32>
__device__ __forceinline__ Raw8<F32> fetch8(const void *base, long long at) {
    Raw8<F32> r;
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + at * (F32 ? 4 : 2));
    r.w[0] = __ldcs(p);
    if constexpr (F32) r.w[1] = __ldcs(p + 1);
    return r;
}
template <bool F32>
__device__ __forceinline__ void widen8(const Raw8<F32> &r, float *x) {
    const uint32_t u[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
    if constexpr (F32) {
        const uint32_t v[4] = {r.w[1].x, r.w[1].y, r.w[1].z, r.w[1].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = __uint_as_float(u[i]);
            x[4 + i] = __uint_as_float(v[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(u[i] << 16);
            x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
        }
    }
}
template <bool F32>
__device__ __forceinline__ void store8(void *base, long long at, const float *x) {
    if constexpr (F32) {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + at);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = reinterpret_cast<const uint32_t &>(h);
        }
        *reinterpret_cast<uint4 *>(static_cast<__nv_bfloat16 *>(base) + at) = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
// The value, or 0; asked for in program order, so that those of a row are on their way together (65,536 rows of 1,500 values: 182 us, in the
// order that the compiler finds 247)
template <bool F32>
__device__ __forceinline__ float load1_if(const void *base, long long at, bool there) {
    const char *const from = static_cast<const char *>(base) + at * (F32 ? 4 : 2);
    if constexpr (F32) {
        float v;
        asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\nmov.b32 %0, 0;\n@q ld.global.f32 %0, [%1];\n}" : "=f"(v) : "l"(from), "r"((int)there));
        return v;
    } else {
        unsigned short v;
        asm volatile("{\n.reg .pred q;\nsetp.ne.b32 q, %2, 0;\nmov.b16 %0, 0;\n@q ld.global.u16 %0, [%1];\n}" : "=h"(v) : "l"(from), "r"((int)there));
        return __uint_as_float((uint32_t)v << 16);
    }
}
template <bool F32>
__device__ __forceinline__ void store1(void *base, long long at, float v) {
    if constexpr (F32) static_cast<float *>(base)[at] = v;
    else static_cast<__nv_bfloat16 *>(base)[at] = __float2bfloat16_rn(v);
}
// 8 floats of a weight, which stay in L1: loaded where they are used, so that they do not hold registers in between.  (Plain loads: the kernel
// before this one, which may still run when this one starts, may be what writes them.)
__device__ __forceinline__ void load8_again(const float *p, float *x) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("ld.global.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[4 * i]), "=f"(x[4 * i + 1]), "=f"(x[4 * i + 2]), "=f"(x[4 * i + 3])
                     : "l"(p + 4 * i));
}

// The values of a row that a thread of a group of `group` threads holds: P pieces of 8 neighbours (VEC), or 8 P values that lie
// `group` apart, for rows that start on no 16-byte boundary.
template <bool VEC, int P>
struct Place {
    int t, group, dim;
    __device__ __forceinline__ int piece(int p) const { return (t + p * group) * 8; }
    __device__ __forceinline__ int value(int i) const { return VEC ? piece(i >> 3) + (i & 7) : t + i * group; }
    __device__ __forceinline__ bool has(int i) const { return (VEC ? piece(i >> 3) : value(i)) < dim; }
};

template <bool F32, bool VEC, int P>
__device__ __forceinline__ void load_row(const Place<VEC, P> &l, const void *base, long long at, float (&v)[8 * P]) {
    if constexpr (VEC) {
        Raw8<F32> raw[P];
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (l.piece(p) < l.dim) raw[p] = fetch8<F32>(base, at + l.piece(p));
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (l.piece(p) < l.dim) widen8<F32>(raw[p], v + 8 * p);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) v[8 * p + i] = 0.f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) v[i] = load1_if<F32>(base, at + l.value(i), l.has(i));
    }
}
template <bool F32, bool VEC, int P>
__device__ __forceinline__ void store_row(const Place<VEC, P> &l, void *base, long long at, const float (&v)[8 * P]) {
    if constexpr (VEC) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (l.piece(p) < l.dim) store8<F32>(base, at + l.piece(p), v + 8 * p);
    } else {
#pragma unroll
        for (int i = 0; i < 8 * P; ++i)
            if (l.has(i)) store1<F32>(base, at + l.value(i), v[i]);
    }
}
// f(index into the registers, weight of that value).  TOGETHER: without 16-byte boundaries all weights are asked for before the first is used.  So
// for gradients (100,000 rows of 300 values in float32: 83 us, one at a time 98) and for 32 values a thread (5,000 rows of 15,001: 210 and 298), else
// not (100,000 rows of 300: 54 and 49).
template <bool TOGETHER = false, bool VEC, int P, typename F>
__device__ __forceinline__ void with_weight(const Place<VEC, P> &l, const float *w, F &&f) {
    if constexpr (VEC) {
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (l.piece(p) < l.dim) {
                float x[8];
                load8_again(w + l.piece(p), x);
#pragma unroll
                for (int i = 0; i < 8; ++i) f(8 * p + i, x[i]);
            }
    } else if constexpr (TOGETHER) {
        float x[8 * P];
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) x[i] = load1_if<true>(w, l.value(i), l.has(i));
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) f(i, x[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8 * P; ++i)
            if (l.has(i)) f(i, w[l.value(i)]);
    }
}

// sums over neighbouring lanes, a power of two of them
template <int LANES = 32>
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
// sums over the group: LANES of a warp, or (0) the CTA (every warp adds up the warps' sums in the same order).  `slot`: one of four places in
// turn, so that one barrier a sum is enough
template <int LANES, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float (*s)[32][2], int &slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum<LANES ? LANES : 32>(v[i]);
    if constexpr (!LANES) {
        const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
        if (lane == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) s[slot][warp][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = warp_sum(lane < warps ? s[slot][lane][i] : 0.f);
        slot = (slot + 1) & 3;
    }
}

// mean and r of the row in v; v becomes x - mean
template <int LANES, bool VEC, int P>
__device__ __forceinline__ float deviations(const RowNormParams &p, const Place<VEC, P> &l, float (&v)[8 * P], float (*s)[32][2], int &slot) {
    if (!p.rms) {
        float sum[1] = {0.f};
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) sum[0] += v[i];
        group_sum<LANES>(sum, s, slot);
        const float mean = sum[0] / (float)p.dim;           // (divided: equal values have no deviation)
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) v[i] = l.has(i) ? v[i] - mean : 0.f;
    }
    float sq[1] = {0.f};
#pragma unroll
    for (int i = 0; i < 8 * P; ++i) sq[0] = fmaf(v[i], v[i], sq[0]);
    group_sum<LANES>(sq, s, slot);
    return rsqrtf(fmaf(sq[0], p.inv_dim, p.eps));
}

__device__ __forceinline__ long long actual_tokens(const RowNormParams &p) {
    if (!p.count) return p.tokens;
    const long long c = *p.count;
    return c < 0 ? 0 : c > p.tokens ? p.tokens : c;
}

// Kernels here are launched while the one before them in the stream still runs; nothing that it may write is read, and nothing that it may
// read is written, before this.  The next one may begin at once.
__device__ __forceinline__ void in_turn() {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
}

// A row per group of LANES lanes (few enough that a short row leaves none of them idle: 262,144 rows of 64 values in bfloat16 take 20 us, with a
// warp each 70), or (0) of the CTA's threads.  Groups without a row take part in the sums.
template <bool X32, bool Y32, int LANES, bool VEC, int P>
__global__ void __launch_bounds__(LANES ? 128 : 512) layer_norm_kernel(const RowNormParams p) {
    __shared__ float s[4][32][2];
    in_turn();
    int slot = 0;
    const Place<VEC, P> l = {LANES ? (int)threadIdx.x & (LANES - 1) : (int)threadIdx.x, LANES ? LANES : (int)blockDim.x, p.dim};
    const long long token = LANES ? (long long)blockIdx.x * (128 / (LANES ? LANES : 1)) + threadIdx.x / (LANES ? LANES : 1) : blockIdx.x;
    long long row = -1;
    if (token < actual_tokens(p)) row = p.rows ? p.rows[token] : token;
    const bool there = row >= 0 && row < p.x_rows;
    if ((LANES == 0 || LANES == 32) && !there) return;
    float v[8 * P] = {};
    if (there) load_row<X32>(l, p.x, row * p.x_stride, v);
    const float r = deviations<LANES>(p, l, v, s, slot);
    if (!there) return;
    constexpr bool kTogether = LANES == 0 && P == 4;
    if (p.weight) with_weight<kTogether>(l, p.weight, [&](int i, float w) { v[i] = v[i] * r * w; });
    else
#pragma unroll
        for (int i = 0; i < 8 * P; ++i) v[i] *= r;
    if (p.bias) with_weight<kTogether>(l, p.bias, [&](int i, float b) { v[i] += b; });
    store_row<Y32>(l, p.out, token * p.out_stride, v);
}

// Rows are dealt out to the groups of the grid in turn; a thread gathers its columns of both weight gradients over all of them.
template <bool X32, bool Y32, int LANES, bool VEC, int P>
__global__ void __launch_bounds__(LANES ? 256 : 512) layer_norm_backward_kernel(const RowNormParams p) {
    constexpr int V = 8 * P;
    __shared__ float s[4][32][2];
    extern __shared__ float sums[];                         // LANES: [groups][dim]
    in_turn();
    int slot = 0;
    const Place<VEC, P> l = {LANES ? (int)threadIdx.x & (LANES - 1) : (int)threadIdx.x, LANES ? LANES : (int)blockDim.x, p.dim};
    const int groups_here = LANES ? 256 / (LANES ? LANES : 1) : 1, mine = LANES ? threadIdx.x / (LANES ? LANES : 1) : 0;
    const int warp_first = LANES ? (threadIdx.x >> 5) * (32 / (LANES ? LANES : 32)) : 0;
    float dw[V] = {}, db[V] = {};
    // Rows off 16-byte boundaries: a warp's long ones keep their weights, 32 a lane (65,536 rows of 1,023 values: 165 us, loaded again for each row 183)
    constexpr bool kKept = !VEC && LANES && P == 4;
    float kept[kKept ? V : 1];
    if constexpr (kKept)
#pragma unroll
        for (int i = 0; i < V; ++i) kept[i] = p.weight ? load1_if<true>(p.weight, l.value(i), l.has(i)) : 1.f;
    for (long long row0 = (long long)blockIdx.x * groups_here; row0 + warp_first < p.tokens; row0 += (long long)gridDim.x * groups_here) {
        const long long row = row0 + mine;
        const bool there = LANES == 0 || LANES == 32 || row < p.tokens;
        float v[V] = {}, g[V] = {};
        if (there) {
            load_row<X32>(l, p.x, row * p.x_stride, v);
            load_row<Y32>(l, p.dy, row * p.dy_stride, g);
        }
        float r = deviations<LANES>(p, l, v, s, slot);
        if (!there) r = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] *= r;                                      // n
            dw[i] = fmaf(g[i], v[i], dw[i]);
            db[i] += g[i];
        }
        if constexpr (kKept) {
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] *= kept[i];
        } else if (p.weight) {
            with_weight<true>(l, p.weight, [&](int i, float w) { g[i] *= w; });
        }
        float both[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < V; ++i) {
            both[0] += g[i];
            both[1] = fmaf(g[i], v[i], both[1]);
        }
        group_sum<LANES>(both, s, slot);
        const float less = p.rms ? 0.f : both[0] * p.inv_dim, along = both[1] * p.inv_dim;
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = r * (g[i] - less - v[i] * along);
        if (there) store_row<X32>(l, p.out, row * p.out_stride, g);
    }
    if (!p.partial) return;
    float *const to = p.partial + (long long)blockIdx.x * 2 * p.dim;
    if constexpr (!LANES) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (l.has(i)) {
                to[l.value(i)] = dw[i];
                to[p.dim + l.value(i)] = db[i];
            }
    } else {
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (which) __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (l.has(i)) sums[mine * p.dim + l.value(i)] = which ? db[i] : dw[i];
            __syncthreads();
            for (int c = threadIdx.x; c < p.dim; c += blockDim.x) {
                float total = 0.f;
                for (int g = 0; g < groups_here; ++g) total += sums[g * p.dim + c];
                to[which * p.dim + c] = total;
            }
        }
    }
}

// ---- long rows on 16-byte boundaries ----
//
// A CTA walks over the rows, R at a time.  A warp of its own brings them by bulk copies into a ring of stages in shared memory, as many
// ahead of the ones that are worked on as there is room for: up to 5 of 2,048 values, of 16,384 values in bfloat16 1 (gradients) to 5, of more
// than 11,160 float32 values with a float32 gradient none (issued by a thread that works on them they hold up all the others: 100 us, not 59, for 16,384
// rows of 4,096).  Weights stay in registers, of the gradients in shared memory: the ring leaves L1 too small for them.
// Values are worked on in pairs.
constexpr int kMaxRing = 6;

__device__ __forceinline__ uint64_t pair(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t both(float a) { return pair(a, a); }
__device__ __forceinline__ void unpair(uint64_t p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ float total(uint64_t p) {
    float a, b;
    unpair(p, a, b);
    return a + b;
}
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
// 8 values as four pairs: from shared memory, from a weight in global memory (which stays in L1), and to global memory
template <bool F32>
__device__ __forceinline__ void pairs_in(const unsigned char *at, uint64_t *v) {
    const uint4 a = *reinterpret_cast<const uint4 *>(at);
    if constexpr (F32) {
        const uint4 b = *reinterpret_cast<const uint4 *>(at + 16);
        v[0] = pair(__uint_as_float(a.x), __uint_as_float(a.y));
        v[1] = pair(__uint_as_float(a.z), __uint_as_float(a.w));
        v[2] = pair(__uint_as_float(b.x), __uint_as_float(b.y));
        v[3] = pair(__uint_as_float(b.z), __uint_as_float(b.w));
    } else {
        const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
}
__device__ __forceinline__ void pairs_weight(const float *p, uint64_t *v) {
    float x[8];
    load8_again(p, x);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pair(x[2 * i], x[2 * i + 1]);
}
template <bool F32>
__device__ __forceinline__ void pairs_out(void *base, long long at, const uint64_t *v) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) unpair(v[i], x[2 * i], x[2 * i + 1]);
    store8<F32>(base, at, x);
}

constexpr long long kWaitLimit = 8000000000ll;   // SM cycles (about 4 s)
constexpr long long kShortLimit = 1 << 20;       // limits below it are a test's
constexpr long long kDrainLimit = 200000000ll;   // (about 0.1 s)

struct RingBars {
    uint64_t full[kMaxRing], empty[kMaxRing], never;
    volatile int gave_up;
};

// The ring of a CTA, seen by one of its warps.  Waits have a limit in SM cycles; once one ran out, no row is asked for any more, every later
// wait of the CTA gives up at once, the kernel runs to its end with whatever is in its buffers, and the status word says that the results are
// not valid.
struct Ring {
    RingBars *bars;
    uint32_t base, stage_bytes;
    int stages;
    long long limit;
    int stage = 0;
    uint32_t phase = 0;

    static __device__ __forceinline__ uint32_t at(const uint64_t *bar) { return (uint32_t)__cvta_generic_to_shared(bar); }
    __device__ __forceinline__ void set_up(int readers) const {
        for (int i = 0; i < stages; ++i) {
            asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(at(bars->full + i)) : "memory");
            asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(at(bars->empty + i)), "r"(readers) : "memory");
        }
        asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(at(&bars->never)) : "memory");
        bars->gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    static __device__ __forceinline__ bool there(const uint64_t *bar, uint32_t parity) {
        uint32_t yes;
        asm volatile(
            "{\n"
            ".reg .pred q;\n"
            "mbarrier.try_wait.parity.shared::cta.b64 q, [%1], %2;\n"
            "selp.u32 %0, 1, 0, q;\n"
            "}\n"
            : "=r"(yes)
            : "r"(at(bar)), "r"(parity)
            : "memory");
        return yes != 0;
    }
    __device__ __forceinline__ bool wait(const uint64_t *bar, uint32_t parity) const {
        if (there(bar, parity)) return true;
        for (const long long t0 = clock64(); !there(bar, parity);) {
            if (bars->gave_up) return false;
            if (clock64() - t0 > limit) {
                bars->gave_up = 1;
                atomicOr(&g_layer_norm_status, 1);
                return false;
            }
        }
        return true;
    }
    __device__ __forceinline__ void wait_full() const { wait(bars->full + stage, phase); }
    // false: nothing is to be asked for any more
    __device__ __forceinline__ bool wait_empty() const { return wait(bars->empty + stage, phase ^ 1) && !bars->gave_up; }
    // so that a wait runs out for certain
    __device__ __forceinline__ void short_limit() const {
        if (limit < kShortLimit && threadIdx.x == 0) wait(&bars->never, 0);
    }
    // The end of the warp that asks for rows: all that it has started lands before it leaves, so that none of it comes down where another
    // CTA is by then.  `issued`: stages in use since the ring began, up to all of them
    __device__ __forceinline__ void drain(int issued) {
        for (; issued > 0; --issued) {
            if (stage == 0) {
                stage = stages;
                phase ^= 1;
            }
            --stage;
            for (const long long t0 = clock64(); !there(bars->full + stage, phase);)
                if (clock64() - t0 > (bars->gave_up ? kDrainLimit : kWaitLimit)) {
                    atomicOr(&g_layer_norm_status, 1);
                    return;
                }
        }
    }
    __device__ __forceinline__ void next() {
        if (++stage == stages) {
            stage = 0;
            phase ^= 1;
        }
    }
    // the warp has the stage's values
    __device__ __forceinline__ void release() {
        __syncwarp();
        if ((threadIdx.x & 31) == 0) asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(at(bars->empty + stage)) : "memory");
        next();
    }
};
__device__ __forceinline__ void ring_expect(uint32_t bar, int bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ring_copy(uint32_t to, const void *from, int bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to), "l"(from), "r"(bytes), "r"(bar)
                 : "memory");
}

// Sums over the CTA of N values, always in the same order.  s: [4][N][16]; `slot`: one of four places in turn, so that one barrier is enough.
// Of the working warps.
template <int THREADS, int N>
__device__ __forceinline__ void cta_sums(float (&v)[N], float *s, int &slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    float *const here = s + slot * (N * 16);
    if ((threadIdx.x & 31) == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) here[i * 16 + (threadIdx.x >> 5)] = v[i];
    asm volatile("bar.sync 1, %0;" ::"n"(THREADS) : "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < THREADS / 32; w += 4) {
            const float4 x = *reinterpret_cast<const float4 *>(here + i * 16 + w);
            t += (x.x + x.y) + (x.z + x.w);
        }
        v[i] = t;
    }
    slot = (slot + 1) & 3;
}

// FULL: every thread has all its pieces, as with rows of 2,048 or 4,096 values.
// what a step reads, widened to pairs: row i of the stage, `skip` bytes behind its start
template <bool F32, bool FULL, int P>
__device__ __forceinline__ void stage_row(const Place<true, P> &l, const unsigned char *at, bool there, uint64_t (&v)[4 * P]) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
        if (there && (FULL || l.piece(q) < l.dim)) pairs_in<F32>(at + l.piece(q) * (F32 ? 4 : 2), v + 4 * q);
        else
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = 0;
    }
}

// v becomes x - mean (0 where there is no value), from the sum of the row
template <bool FULL, int P>
__device__ __forceinline__ void less_mean(const Place<true, P> &l, uint64_t (&v)[4 * P], float sum) {
    const uint64_t less = both(-(sum / (float)l.dim));
#pragma unroll
    for (int e = 0; e < 4 * P; ++e) v[e] = add2(v[e], less);
    if (!FULL)                                              // (not all threads have all pieces)
#pragma unroll
        for (int q = 0; q < P; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * q + e] = l.piece(q) < l.dim ? v[4 * q + e] : 0;
}

template <bool X32, bool Y32, bool RMS, bool FULL, int THREADS, int P, int R>
__global__ void __launch_bounds__(THREADS + 32, 512 / THREADS) layer_norm_ring_kernel(const RowNormParams p, int stages) {
    __shared__ __align__(16) float s[4 * R * 16];
    __shared__ RingBars bars;
    extern __shared__ __align__(128) unsigned char ring[];
    const Place<true, P> l = {(int)threadIdx.x, THREADS, p.dim};
    const int row_bytes = p.dim * (X32 ? 4 : 2);
    long long tokens = 0;
    const auto row_at = [&](long long token) {               // -1: none
        if (token >= tokens) return -1ll;
        const long long row = p.rows ? p.rows[token] : token;
        return row >= 0 && row < p.x_rows ? row : -1ll;
    };
    Ring r = {&bars, (uint32_t)__cvta_generic_to_shared(ring), (uint32_t)(R * row_bytes), stages, p.wait_limit};
    if (threadIdx.x == 0) r.set_up(THREADS / 32);
    in_turn();
    tokens = actual_tokens(p);
    const long long steps = (tokens + R - 1) / R;
    __syncthreads();
    if (threadIdx.x >= THREADS) {
        if (threadIdx.x == THREADS) {
            int issued = 0;
            for (long long step = blockIdx.x; step < steps; step += gridDim.x) {
                long long row[R];
                int n = 0;
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    row[i] = row_at(step * R + i);
                    n += row[i] >= 0;
                }
                if (!r.wait_empty()) break;
                const uint32_t bar = Ring::at(bars.full + r.stage), to = r.base + r.stage * r.stage_bytes;
                ring_expect(bar, n * row_bytes);
#pragma unroll
                for (int i = 0; i < R; ++i)
                    if (row[i] >= 0) ring_copy(to + i * row_bytes, static_cast<const char *>(p.x) + row[i] * p.x_stride * (X32 ? 4 : 2), row_bytes, bar);
                r.next();
                issued = min(issued + 1, stages);
            }
            r.drain(issued);
        }
        return;
    }
    r.short_limit();
    uint64_t w[4 * P], b[4 * P];
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            w[4 * q + e] = both(1.f);
            b[4 * q + e] = 0;
        }
        if (FULL || l.piece(q) < p.dim) {
            if (p.weight) pairs_weight(p.weight + l.piece(q), w + 4 * q);
            if (p.bias) pairs_weight(p.bias + l.piece(q), b + 4 * q);
        }
    }
    int slot = 0;
    for (long long step = blockIdx.x; step < steps; step += gridDim.x) {
        uint64_t v[R][4 * P];
        bool there[R];
        r.wait_full();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            there[i] = row_at(step * R + i) >= 0;
            stage_row<X32, FULL>(l, ring + (r.stage * R + i) * row_bytes, there[i], v[i]);
        }
        float sum[R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            uint64_t t = 0;
#pragma unroll
            for (int e = 0; e < 4 * P; ++e) t = RMS ? fma2(v[i][e], v[i][e], t) : add2(t, v[i][e]);
            sum[i] = total(t);
        }
        r.release();
        cta_sums<THREADS>(sum, s, slot);
        if (!RMS) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                less_mean<FULL>(l, v[i], sum[i]);
                uint64_t t = 0;
#pragma unroll
                for (int e = 0; e < 4 * P; ++e) t = fma2(v[i][e], v[i][e], t);
                sum[i] = total(t);
            }
            cta_sums<THREADS>(sum, s, slot);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const uint64_t scale = both(rsqrtf(fmaf(sum[i], p.inv_dim, p.eps)));
            if (there[i])
#pragma unroll
                for (int q = 0; q < P; ++q)
                    if (FULL || l.piece(q) < p.dim) {
                        uint64_t y[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) y[e] = fma2(mul2(v[i][4 * q + e], scale), w[4 * q + e], b[4 * q + e]);
                        pairs_out<Y32>(p.out, (step * R + i) * p.out_stride + l.piece(q), y);
                    }
        }
    }
}

// Gradients.  With d = x - mean and t = dy d the sums of a row are those of d^2, g = dy w and t w, all at once:
//   along = mean(g n) = r mean(t w);  dw += r t;  dx = r g - r mean(g) - r along d r
// 8,191 rows of 4,096 take 53 us with the sums' kernel, 3.8 TB/s.  What bounds it: latency.  Issue slots are 53 % full; a warp waits for shared memory and
// shuffles most of the time between two of its 430 instructions a row, in two rounds of sums one after the other, at 16 working warps per SM, which
// 96 registers leave.  (Without the checks for rows that do not fill the threads: 60 us.)  Rows of more than 8,192 values, 32 of each array a
// thread, spill 464 to 480 bytes.
template <bool X32, bool Y32, bool RMS, int THREADS, int P, int R>
__global__ void __launch_bounds__(THREADS + 32, 512 / THREADS) layer_norm_backward_ring_kernel(const RowNormParams p, int stages) {
    __shared__ __align__(16) float s1[4 * R * 16], s3[4 * 3 * R * 16];
    __shared__ RingBars bars;
    extern __shared__ __align__(128) unsigned char raw[];
    float *const weight = reinterpret_cast<float *>(raw);    // [2][dim / 8][4]: halves of eight neighbours, apart for the banks' sake
    unsigned char *const ring = raw + p.dim * 4;
    const Place<true, P> l = {(int)threadIdx.x, THREADS, p.dim};
    const int x_bytes = p.dim * (X32 ? 4 : 2), y_bytes = p.dim * (Y32 ? 4 : 2), row_bytes = x_bytes + y_bytes;
    const long long steps = (p.tokens + R - 1) / R;
    Ring r = {&bars, (uint32_t)__cvta_generic_to_shared(ring), (uint32_t)(R * row_bytes), stages, p.wait_limit};
    if (threadIdx.x == 0) r.set_up(THREADS / 32);
    in_turn();
    for (int i = threadIdx.x; i < p.dim / 4; i += THREADS + 32)
        *reinterpret_cast<float4 *>(weight + (i & 1) * (p.dim / 2) + (i >> 1) * 4) =
            p.weight ? *reinterpret_cast<const float4 *>(p.weight + 4 * i) : make_float4(1.f, 1.f, 1.f, 1.f);
    const auto weights = [&](int q, uint64_t (&w)[4]) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 x = *reinterpret_cast<const float4 *>(weight + h * (p.dim / 2) + (l.t + q * THREADS) * 4);
            w[2 * h] = pair(x.x, x.y);
            w[2 * h + 1] = pair(x.z, x.w);
        }
    };
    __syncthreads();
    if (threadIdx.x >= THREADS) {
        if (threadIdx.x == THREADS) {
            int issued = 0;
            for (long long step = blockIdx.x; step < steps; step += gridDim.x) {
                const int rows = (int)min((long long)R, p.tokens - step * R);
                if (!r.wait_empty()) break;
                const uint32_t bar = Ring::at(bars.full + r.stage), to = r.base + r.stage * r.stage_bytes;
                ring_expect(bar, rows * row_bytes);
                for (int i = 0; i < rows; ++i) {
                    const long long row = step * R + i;
                    ring_copy(to + i * row_bytes, static_cast<const char *>(p.x) + row * p.x_stride * (X32 ? 4 : 2), x_bytes, bar);
                    ring_copy(to + i * row_bytes + x_bytes, static_cast<const char *>(p.dy) + row * p.dy_stride * (Y32 ? 4 : 2), y_bytes, bar);
                }
                r.next();
                issued = min(issued + 1, stages);
            }
            r.drain(issued);
        }
        return;
    }
    r.short_limit();
    int slot = 0, slot3 = 0;
    uint64_t dw[4 * P] = {}, db[4 * P] = {};
    for (long long step = blockIdx.x; step < steps; step += gridDim.x) {
        r.wait_full();
        const int rows = (int)min((long long)R, p.tokens - step * R);
        uint64_t v[R][4 * P], g[R][4 * P];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const unsigned char *const at = ring + (r.stage * R + i) * row_bytes;
            stage_row<X32, false>(l, at, i < rows, v[i]);
            stage_row<Y32, false>(l, at + x_bytes, i < rows, g[i]);
        }
        r.release();
        if (!RMS) {
            float sum[R];
#pragma unroll
            for (int i = 0; i < R; ++i) {
                uint64_t t = 0;
#pragma unroll
                for (int e = 0; e < 4 * P; ++e) t = add2(t, v[i][e]);
                sum[i] = total(t);
            }
            cta_sums<THREADS>(sum, s1, slot);
#pragma unroll
            for (int i = 0; i < R; ++i) less_mean<false>(l, v[i], sum[i]);
        }
        uint64_t sq[R] = {}, sg[R] = {}, st[R] = {};
#pragma unroll
        for (int q = 0; q < P; ++q)
            if (l.piece(q) < p.dim) {
                uint64_t w[4];
                weights(q, w);
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t d = v[i][4 * q + e], dy = g[i][4 * q + e];
                        db[4 * q + e] = add2(db[4 * q + e], dy);
                        sq[i] = fma2(d, d, sq[i]);
                        if (!RMS) sg[i] = fma2(dy, w[e], sg[i]);
                        st[i] = fma2(mul2(dy, d), w[e], st[i]);
                    }
            }
        float sums[3 * R];
#pragma unroll
        for (int i = 0; i < R; ++i) {
            sums[3 * i] = total(sq[i]);
            sums[3 * i + 1] = total(sg[i]);
            sums[3 * i + 2] = total(st[i]);
        }
        cta_sums<THREADS>(sums, s3, slot3);
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (i >= rows) continue;                        // (a row that is not there: 1 / 0)
            const float k = rsqrtf(fmaf(sums[3 * i], p.inv_dim, p.eps)), less = RMS ? 0.f : sums[3 * i + 1] * p.inv_dim;
            const float along = sums[3 * i + 2] * p.inv_dim * k;
            const uint64_t k2 = both(k), less2 = both(-less * k), along2 = both(-along * k * k);
#pragma unroll
            for (int q = 0; q < P; ++q)
                if (l.piece(q) < p.dim) {
                    uint64_t w[4], out[4];
                    weights(q, w);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint64_t d = v[i][4 * q + e], dy = g[i][4 * q + e];
                        dw[4 * q + e] = fma2(mul2(dy, d), k2, dw[4 * q + e]);
                        out[e] = fma2(d, along2, fma2(mul2(dy, w[e]), k2, less2));
                    }
                    pairs_out<X32>(p.out, (step * R + i) * p.out_stride + l.piece(q), out);
                }
        }
    }
    if (!p.partial) return;
    float *const to = p.partial + (long long)blockIdx.x * 2 * p.dim;
#pragma unroll
    for (int q = 0; q < P; ++q)
        if (l.piece(q) < p.dim) {
            pairs_out<true>(to, l.piece(q), dw + 4 * q);
            pairs_out<true>(to, p.dim + l.piece(q), db + 4 * q);
        }
}

// Weight gradients from the CTAs' sums, 32 columns per CTA, always in the same order.  Launched while the CTAs that write them still run.
__global__ void __launch_bounds__(1024) layer_norm_sum_kernel(const float *partial, int parts, int dim, float *dweight, float *dbias) {
    in_turn();
    __shared__ float s[32][33];
    float *const out = blockIdx.y ? dbias : dweight;
    if (!out) return;
    const int lane = threadIdx.x & 31, part = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    float sum = 0.f;
    if (col < dim)
        for (int b = part; b < parts; b += 32) sum += partial[((long long)b * 2 + blockIdx.y) * dim + col];
    s[part][lane] = sum;
    __syncthreads();
    if (part == 0 && col < dim) {
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += s[i][lane];
        out[col] = total;
    }
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// see in_turn
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

// once for a device and kernel
template <typename Kernel>
cudaError_t ring_ready(Kernel kernel, std::atomic<unsigned long long> &done) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    const unsigned long long bit = device >= 0 && device < 64 ? 1ull << device : 0;
    if (e != cudaSuccess || (done.load(std::memory_order_acquire) & bit)) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024);
    if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
    return e;
}
int ring_stages(int room, int stage) { return room / stage < kMaxRing ? room / stage : kMaxRing; }

// `which`: rows of up to (-1, gradients only: 1,024) 2,048, 4,096, 8,192 and 16,384 values.  512 working threads an SM; a row's warps have all
// pieces of the row or nearly: four CTAs of 128 threads for 2,048 values take 48 us for 32,768 rows, two of 256 threads 70.
template <bool X32, bool Y32, bool RMS, bool FULL>
auto ring_forward(int which) {
    return which == 0   ? layer_norm_ring_kernel<X32, Y32, RMS, FULL, 128, 2, 2>
           : which == 1 ? layer_norm_ring_kernel<X32, Y32, RMS, FULL, 256, 2, 2>
           : which == 2 ? layer_norm_ring_kernel<X32, Y32, RMS, FULL, 512, 2, 2>
                        : layer_norm_ring_kernel<X32, Y32, RMS, FULL, 512, 4, 1>;
}
template <bool X32, bool Y32>
auto ring_forward(bool rms, bool full, int which) {
    if (rms) return full ? ring_forward<X32, Y32, true, true>(which) : ring_forward<X32, Y32, true, false>(which);
    return full ? ring_forward<X32, Y32, false, true>(which) : ring_forward<X32, Y32, false, false>(which);
}
template <bool X32, bool Y32, bool RMS>
auto ring_backward(int which) {
    return which < 0    ? layer_norm_backward_ring_kernel<X32, Y32, RMS, 128, 1, 2>
           : which == 0 ? layer_norm_backward_ring_kernel<X32, Y32, RMS, 128, 2, 1>
           : which == 1 ? layer_norm_backward_ring_kernel<X32, Y32, RMS, 256, 2, 1>
           : which == 2 ? layer_norm_backward_ring_kernel<X32, Y32, RMS, 512, 2, 1>
                        : layer_norm_backward_ring_kernel<X32, Y32, RMS, 512, 4, 1>;
}

// lanes that have a row's values, 8 each (up to 256 values), 16 or 32
int lanes_of(int dim) { return dim <= 32 ? 4 : dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }
// threads that have them, 8 `pieces` each
int threads_of(int dim, int pieces) { return (dim + pieces * 256 - 1) / (pieces * 256) * 32; }

template <bool X32, bool Y32, bool VEC>
cudaError_t launch_forward(const RowNormParams &p, int sms, cudaStream_t stream) {
    if constexpr (VEC) {
        // more rows than are worked on at one time: a few CTAs that stay, with the next rows on their way
        if (p.dim > 1024 && p.tokens > 8ll * sms) {
            static std::atomic<unsigned long long> done[4][4];
            const int which = p.dim <= 2048 ? 0 : p.dim <= 4096 ? 1 : p.dim <= 8192 ? 2 : 3, threads = which < 2 ? 128 << which : 512, rows = which == 3 ? 1 : 2;
            const int per_sm = 512 / threads, stage = rows * p.dim * (X32 ? 4 : 2);
            const bool full = p.dim == threads * 8 * (which == 3 ? 4 : 2);
            const auto kernel = ring_forward<X32, Y32>(p.rms, full, which);
            const cudaError_t e = ring_ready(kernel, done[which][p.rms + 2 * full]);
            if (e != cudaSuccess) return e;
            const int stages = ring_stages((220 / per_sm - 1) * 1024, stage);
            return launch_early(kernel, dim3((unsigned)(sms * per_sm)), threads + 32, (size_t)stages * stage, stream, p, stages);
        }
    }
    if (p.dim <= 1024) {
        const int lanes = lanes_of(p.dim);
        const auto kernel = lanes == 4      ? layer_norm_kernel<X32, Y32, 4, VEC, 1>
                            : lanes == 8    ? layer_norm_kernel<X32, Y32, 8, VEC, 1>
                            : lanes == 16   ? layer_norm_kernel<X32, Y32, 16, VEC, 1>
                            : p.dim <= 256  ? layer_norm_kernel<X32, Y32, 32, VEC, 1>
                            : p.dim <= 512  ? layer_norm_kernel<X32, Y32, 32, VEC, 2>
                                            : layer_norm_kernel<X32, Y32, 32, VEC, 4>;
        const int rows = 128 / lanes;
        return launch_early(kernel, dim3((unsigned)((p.tokens + rows - 1) / rows)), 128, 0, stream, p);
    }
    if constexpr (!VEC) {
        const int pieces = p.dim <= 4096 ? 1 : p.dim <= 8192 ? 2 : 4;
        return launch_early(pieces == 1   ? layer_norm_kernel<X32, Y32, 0, VEC, 1>
                            : pieces == 2 ? layer_norm_kernel<X32, Y32, 0, VEC, 2>
                                          : layer_norm_kernel<X32, Y32, 0, VEC, 4>,
                            dim3((unsigned)p.tokens), threads_of(p.dim, pieces), 0, stream, p);
    } else {
        const int threads = p.dim <= 4096 ? 128 : p.dim <= 8192 ? 256 : 512;
        return launch_early(layer_norm_kernel<X32, Y32, 0, VEC, 4>, dim3((unsigned)p.tokens), threads, 0, stream, p);
    }
}

template <bool X32, bool Y32, bool VEC>
cudaError_t launch_backward(const RowNormParams &p, int sms, int *parts, cudaStream_t stream) {
    // Short rows: a warp's or a part of one's.  From 513 values on the ring is faster where rows lie on 16-byte boundaries (65,536 of 1,024: 103 us,
    // with a warp each, whose 64 sums a lane leave room for 8 warps an SM, 115).
    if (p.dim <= (VEC ? 512 : 1024)) {
        // no more CTAs than run at one time
        const int lanes = lanes_of(p.dim), rows = 256 / lanes, per_sm = p.dim <= 256 ? 3 : p.dim <= 512 ? 2 : 1;
        const long long want = (p.tokens + rows - 1) / rows, most = per_sm * sms < max_partials(p.dim) ? per_sm * sms : max_partials(p.dim);
        const unsigned grid = (unsigned)(want < 1 ? 1 : want < most ? want : most);
        const size_t smem = (size_t)rows * p.dim * sizeof(float);
        const auto kernel = lanes == 4      ? layer_norm_backward_kernel<X32, Y32, 4, VEC, 1>
                            : lanes == 8    ? layer_norm_backward_kernel<X32, Y32, 8, VEC, 1>
                            : lanes == 16   ? layer_norm_backward_kernel<X32, Y32, 16, VEC, 1>
                            : p.dim <= 256  ? layer_norm_backward_kernel<X32, Y32, 32, VEC, 1>
                            : VEC || p.dim <= 512 ? layer_norm_backward_kernel<X32, Y32, 32, VEC, 2>
                                                  : layer_norm_backward_kernel<X32, Y32, 32, false, 4>;
        *parts = (int)grid;
        return launch_early(kernel, dim3(grid), 256, smem, stream, p);
    }
    if constexpr (VEC) {
        static std::atomic<unsigned long long> done[5][2];
        const int which = p.dim <= 1024 ? -1 : p.dim <= 2048 ? 0 : p.dim <= 4096 ? 1 : p.dim <= 8192 ? 2 : 3, threads = which < 0 ? 128 : which < 2 ? 128 << which : 512;
        const int per_sm = 512 / threads, rows = which < 0 ? 2 : 1, stage = rows * p.dim * ((X32 ? 4 : 2) + (Y32 ? 4 : 2));
        const auto kernel = p.rms ? ring_backward<X32, Y32, true>(which) : ring_backward<X32, Y32, false>(which);
        const int stages = ring_stages((220 / per_sm - 2) * 1024 - p.dim * 4, stage);
        const long long most = sms * per_sm < max_partials(p.dim) ? sms * per_sm : max_partials(p.dim);
        const long long want = (p.tokens + rows - 1) / rows;
        const unsigned grid = (unsigned)(want < 1 ? 1 : want < most ? want : most);
        *parts = (int)grid;
        const cudaError_t e = ring_ready(kernel, done[which + 1][p.rms]);
        if (e != cudaSuccess) return e;
        return launch_early(kernel, dim3(grid), threads + 32, (size_t)stages * stage + p.dim * 4, stream, p, stages);
    }
    if constexpr (!VEC) {
        const int threads = p.dim <= 2048 ? 128 : p.dim <= 4096 ? 256 : 512;
        const long long most = sms * (512 / threads) < max_partials(p.dim) ? sms * (512 / threads) : max_partials(p.dim);
        const unsigned grid = (unsigned)(p.tokens < 1 ? 1 : p.tokens < most ? p.tokens : most);
        *parts = (int)grid;
        return launch_early(p.dim <= 8192 ? layer_norm_backward_kernel<X32, Y32, 0, VEC, 2> : layer_norm_backward_kernel<X32, Y32, 0, VEC, 4>, dim3(grid),
                            threads, 0, stream, p);
    }
}

template <typename F>
void with_types(bool x32, bool y32, bool vec, F &&f) {
    const auto types = [&](auto x, auto y) {
        if (vec) f(x, y, std::true_type{});
        else f(x, y, std::false_type{});
    };
    if (x32 && y32) types(std::true_type{}, std::true_type{});
    else if (x32) types(std::true_type{}, std::false_type{});
    else if (y32) types(std::false_type{}, std::true_type{});
    else types(std::false_type{}, std::false_type{});
}

fi_status_t check_args(const fi_layer_norm_t *a, bool backward, const char *name) {
    if (!a) {
        set_error("%s: null argument", name);
        return FI_ERR_INVALID_ARG;
    }
    if ((a->x_dtype != FI_F32 && a->x_dtype != FI_BF16) || (a->y_dtype != FI_F32 && a->y_dtype != FI_BF16)) {
        set_error("%s: types must be FI_F32 or FI_BF16", name);
        return FI_ERR_INVALID_ARG;
    }
    if (a->dim < 1 || a->dim > kMaxDim || a->tokens < 0 || a->tokens > 2147483647ll || (a->rows && a->x_rows < 0)) {
        set_error("%s: 1 <= dim <= %d, 0 <= tokens < 2^31 (got %lld rows of %d)", name, kMaxDim, (long long)a->tokens, a->dim);
        return FI_ERR_INVALID_ARG;
    }
    if (a->tokens > 0 && ((!a->x && !(a->rows && a->x_rows == 0)) || !a->out || (backward && !a->dy))) {
        set_error("%s: null pointer", name);
        return FI_ERR_INVALID_ARG;
    }
    if (backward && (a->rows || a->tokens_dev)) {
        set_error("%s: gradients of all rows only", name);
        return FI_ERR_INVALID_ARG;
    }
    if (backward && (a->dweight || a->dbias) && !a->workspace) {
        set_error("%s: weight gradients need a workspace", name);
        return FI_ERR_INVALID_ARG;
    }
    const uintptr_t x_size = a->x_dtype == FI_F32 ? 4 : 2, y_size = a->y_dtype == FI_F32 ? 4 : 2;
    const long long x_rows = a->rows ? a->x_rows : a->tokens;
    const auto off = [](const void *p, uintptr_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1)) != 0; };
    if (off(a->x, x_size) || off(a->out, backward ? x_size : y_size) || (backward && off(a->dy, y_size)) || off(a->weight, 4) || off(a->bias, 4) ||
        off(a->workspace, 16) || a->wait_limit < 0 || (x_rows > 1 && a->x_stride < a->dim) || (a->tokens > 1 && (a->out_stride < a->dim || (backward && a->dy_stride < a->dim)))) {
        set_error("%s: rows must not overlap; pointers must be aligned to their types", name);
        return FI_ERR_INVALID_ARG;
    }
    return FI_OK;
}

RowNormParams row_norm_params(const fi_layer_norm_t *a, bool backward, bool *vec) {
    RowNormParams p = {};
    p.x = a->x;
    p.dy = a->dy;
    p.out = a->out;
    p.weight = a->weight;
    p.bias = a->bias;
    p.rows = a->rows;
    p.count = a->tokens_dev;
    p.partial = backward && (a->dweight || a->dbias) ? static_cast<float *>(a->workspace) : nullptr;
    p.x_stride = a->x_stride;
    p.dy_stride = a->dy_stride;
    p.out_stride = a->out_stride;
    p.tokens = a->tokens;
    p.x_rows = a->rows ? a->x_rows : a->tokens;
    p.wait_limit = a->wait_limit > 0 && a->wait_limit < kWaitLimit ? a->wait_limit : kWaitLimit;
    p.dim = a->dim;
    p.rms = a->rms != 0;
    p.eps = a->eps;
    p.inv_dim = 1.f / (float)a->dim;
    const auto unit = [](int dtype) { return dtype == FI_F32 ? 4 : 8; };
    const int out_unit = unit(backward ? a->x_dtype : a->y_dtype);
    *vec = a->dim % 8 == 0 && aligned16(a->x) && aligned16(a->out) && aligned16(a->weight) && aligned16(a->bias) &&
           (p.x_rows <= 1 || a->x_stride % unit(a->x_dtype) == 0) && (a->tokens <= 1 || a->out_stride % out_unit == 0) &&
           (!backward || (aligned16(a->dy) && (a->tokens <= 1 || a->dy_stride % unit(a->y_dtype) == 0)));
    return p;
}

}  // namespace
}  // namespace fi

using namespace fi;

extern "C" {

int64_t fi_layer_norm_workspace(int32_t dim) { return dim < 1 || dim > kMaxDim ? 0 : (int64_t)max_partials(dim) * 2 * dim * sizeof(float); }

fi_status_t fi_layer_norm(const fi_layer_norm_t *a, void *cuda_stream) {
    fi_status_t st = check_args(a, false, "fi_layer_norm");
    if (st != FI_OK || a->tokens == 0) return st;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_fail(e, "fi_layer_norm");
    bool vec;
    const RowNormParams p = row_norm_params(a, false, &vec);
    with_types(a->x_dtype == FI_F32, a->y_dtype == FI_F32, vec, [&](auto x, auto y, auto v) {
        e = launch_forward<decltype(x)::value, decltype(y)::value, decltype(v)::value>(p, sms, static_cast<cudaStream_t>(cuda_stream));
    });
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_layer_norm");
}

fi_status_t fi_layer_norm_backward(const fi_layer_norm_t *a, void *cuda_stream) {
    fi_status_t st = check_args(a, true, "fi_layer_norm_backward");
    if (st != FI_OK) return st;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_fail(e, "fi_layer_norm_backward");
    bool vec;
    const RowNormParams p = row_norm_params(a, true, &vec);
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int parts = 0;
    with_types(a->x_dtype == FI_F32, a->y_dtype == FI_F32, vec, [&](auto x, auto y, auto v) {
        e = launch_backward<decltype(x)::value, decltype(y)::value, decltype(v)::value>(p, sms, &parts, stream);
    });
    if (e == cudaSuccess && p.partial)
        e = launch_early(layer_norm_sum_kernel, dim3((a->dim + 31) / 32, 2), 1024, 0, stream, p.partial, parts, a->dim, a->dweight, a->dbias);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_layer_norm_backward");
}

fi_status_t fi_layer_norm_poll_status(void) {
    int32_t word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&word, g_layer_norm_status, sizeof word);
    if (e == cudaSuccess && word) {
        const int32_t zero = 0;
        e = cudaMemcpyToSymbol(g_layer_norm_status, &zero, sizeof zero);
    }
    if (e != cudaSuccess) return cuda_fail(e, "fi_layer_norm_poll_status");
    if (word) {
        set_error("fi_layer_norm, fi_layer_norm_backward: a wait inside a kernel ran out; its results are not valid");
        return FI_ERR_TIMEOUT;
    }
    return FI_OK;
}

}  // extern "C"

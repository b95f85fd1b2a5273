// Norm of each query and key head with the position rotation in the same pass, and its gradients.
//
//   n = x r, r = 1 / sqrt(mean(x^2) + eps);  z = n w;  y = R z
//   backward:  g = R^T dy;  dx = r (g w - n mean(g w n));  dw = sum over tokens and heads of g n
//
// One head of one token (a row) is held by a group of 1..16 neighbouring lanes, 16 values each, in two pieces of 8 that
// lie half a rotation apart, so that both members of every pair are in one lane and the rotation needs no exchange.  The
// sums over a row are shuffles inside the group.  Everything is read once and written once: the bound is the traffic.
#include <cuda_bf16.h>

#include "fi_internal.cuh"

namespace fi {
namespace {

constexpr int kNormThreads = 64;      // of the forward pass: groups share nothing, and small CTAs leave no hole when they end
constexpr int kBackwardThreads = 256;
constexpr int kMaxPartials = 1024;   // CTAs of a backward pass, at most

// rows of one operand: (token, head) pairs
struct NormSide {
    const void *x;
    const void *dy;
    void *out;
    const float *weight;
    long long x_ts, x_hs, dy_ts, dy_hs, out_ts, out_hs;   // elements
    int heads;
};

struct NormParams {
    NormSide q, k;
    const float *rope;
    const int32_t *positions;
    const int32_t *tokens_dev;
    float *partial;        // backward: [CTAs][head_dim]
    int q_ctas;            // backward: CTAs that work on the queries, the others on the keys
    long long tokens;
    int head_dim, rot, max_pos, interleaved;
    float eps, inv_dim;
};

// 8 values as they are in memory, and as fp32
template <bool BF16>
struct Raw8 {
    uint4 w[BF16 ? 1 : 2];
};

template <bool BF16>
__device__ __forceinline__ Raw8<BF16> fetch8(const void *base, long long elem) {
    Raw8<BF16> r;
    const uint4 *p = reinterpret_cast<const uint4 *>(static_cast<const char *>(base) + elem * (BF16 ? 2 : 4));
    r.w[0] = p[0];
    if constexpr (!BF16) r.w[1] = p[1];
    return r;
}

template <bool BF16>
__device__ __forceinline__ void widen8(const Raw8<BF16> &r, float *x) {
    if constexpr (BF16) {
        const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(r.w[i].x); x[4 * i + 1] = __uint_as_float(r.w[i].y);
            x[4 * i + 2] = __uint_as_float(r.w[i].z); x[4 * i + 3] = __uint_as_float(r.w[i].w);
        }
    }
}

template <bool BF16>
__device__ __forceinline__ void load8(const void *base, long long elem, float *x) {
    widen8<BF16>(fetch8<BF16>(base, elem), x);
}

// 8 floats that stay in L1: loaded where they are used, so that they do not hold registers in between
__device__ __forceinline__ void load8_again(const float *p, float *x) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
        asm volatile("ld.global.nc.v4.f32 {%0, %1, %2, %3}, [%4];"
                     : "=f"(x[4 * i]), "=f"(x[4 * i + 1]), "=f"(x[4 * i + 2]), "=f"(x[4 * i + 3])
                     : "l"(p + 4 * i));
}

// ONCE: not to be kept in L2 in the place of what is still to be read
template <bool BF16, bool ONCE = false>
__device__ __forceinline__ void store8(void *base, long long elem, const float *x) {
    if constexpr (BF16) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
            w[i] = reinterpret_cast<const uint32_t &>(h);
        }
        uint4 *p = reinterpret_cast<uint4 *>(static_cast<char *>(base) + elem * 2);
        const uint4 v = make_uint4(w[0], w[1], w[2], w[3]);
        if constexpr (ONCE) __stcs(p, v);
        else *p = v;
    } else {
        float4 *p = reinterpret_cast<float4 *>(static_cast<float *>(base) + elem);
        p[0] = make_float4(x[0], x[1], x[2], x[3]);
        p[1] = make_float4(x[4], x[5], x[6], x[7]);
    }
}

// Where a lane's two pieces start, and the first of the 8 angles it turns by (turned = false: its values pass unturned).
struct LanePlace {
    int a, b, angle;
    bool there, turned;
};

__device__ __forceinline__ LanePlace lane_place(const NormParams &p, int lane) {
    LanePlace l;
    l.there = lane < p.head_dim / 16;
    l.turned = lane < p.rot / 16;
    l.angle = lane * 8;
    if (p.interleaved) {
        l.a = lane * 16;
        l.b = l.a + 8;
    } else if (l.turned) {
        l.a = lane * 8;
        l.b = p.rot / 2 + lane * 8;
    } else {
        l.a = lane * 16;   // the rest behind the rotated values starts at a multiple of 16 too
        l.b = l.a + 8;
    }
    return l;
}

// turn v[0..7], v[8..15] by the lane's angles (dir = -1: back)
__device__ __forceinline__ void turn(float (&v)[16], const float (&c)[8], const float (&s)[8], int interleaved, float dir) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = v[2 * i], b = v[2 * i + 1], t = s[i] * dir;
            v[2 * i] = a * c[i] - b * t;
            v[2 * i + 1] = b * c[i] + a * t;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = v[i], b = v[8 + i], t = s[i] * dir;
            v[i] = a * c[i] - b * t;
            v[8 + i] = b * c[i] + a * t;
        }
    }
}

__device__ __forceinline__ void load_angles(const NormParams &p, const LanePlace &l, int pos, float (&c)[8], float (&s)[8]) {
    if (pos < 0 || pos >= p.max_pos) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
        return;
    }
    const float *row = p.rope + (long long)pos * p.rot;
    load8<false>(row, l.angle, c);
    load8<false>(row, p.rot / 2 + l.angle, s);
}

template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

__device__ __forceinline__ long long actual_tokens(const NormParams &p) {
    if (!p.tokens_dev) return p.tokens;
    const long long t = *p.tokens_dev;
    return t < 0 ? 0 : t > p.tokens ? p.tokens : t;
}

// A group takes R heads of one token, of the queries or of the keys: their loads are all on the way at once, and the angles
// and the weight are loaded once for them.  R = 4 keeps 64 bytes per thread in flight and reads the table a quarter as
// often: 16,384 tokens of 32 + 8 heads of 128 (bf16) took 103 us with one head per group and take 65.5, 5.3 TB/s (68.3 in
// CTAs of 256 threads, where the last group to end keeps the place of the others).  Small calls take R = 1, which has the
// shorter chain (launch_norm).
template <int LANES, bool BF16, int R>
__global__ void __launch_bounds__(kNormThreads, R == 1 ? 16 : 12) head_norm_rope_kernel(NormParams p) {
    const int lane = threadIdx.x & (LANES - 1);
    const unsigned q_parts = (p.q.heads + R - 1) / R, parts = q_parts + (p.k.heads + R - 1) / R;
    const unsigned item = blockIdx.x * (unsigned)(kNormThreads / LANES) + threadIdx.x / LANES;
    const unsigned token = item / parts, part = item - token * parts;
    const LanePlace l = lane_place(p, lane);
    const bool active = (long long)token < actual_tokens(p) && l.there;
    const bool is_k = part >= q_parts;
    const NormSide &side = is_k ? p.k : p.q;
    const int head0 = (int)(is_k ? part - q_parts : part) * R, heads = min(side.heads - head0, R);
    Raw8<BF16> raw[R][2];
    float c[8], s[8];
    const bool turned = active && l.turned;
    if (active) {
        const long long at = (long long)token * side.x_ts + (long long)head0 * side.x_hs;
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i < heads) {
                raw[i][0] = fetch8<BF16>(side.x, at + i * side.x_hs + l.a);
                raw[i][1] = fetch8<BF16>(side.x, at + i * side.x_hs + l.b);
            }
        if (turned) load_angles(p, l, p.positions[token], c, s);
    }
    const long long to = (long long)token * side.out_ts + (long long)head0 * side.out_hs;
#pragma unroll
    for (int i = 0; i < R; ++i) {
        float v[16], sum = 0.f;
        if (active && i < heads) {
            widen8<BF16>(raw[i][0], v);
            widen8<BF16>(raw[i][1], v + 8);
#pragma unroll
            for (int e = 0; e < 16; ++e) sum = fmaf(v[e], v[e], sum);
        }
        sum = group_sum<LANES>(sum);
        if (active && i < heads) {
            const float r = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
            if (side.weight) {
                float w[16];
                load8_again(side.weight + l.a, w);
                load8_again(side.weight + l.b, w + 8);
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] = v[e] * r * w[e];
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] *= r;
            }
            if (turned) turn(v, c, s, p.interleaved, 1.f);
            store8<BF16>(side.out, to + i * side.out_hs + l.a, v);
            store8<BF16>(side.out, to + i * side.out_hs + l.b, v + 8);
        }
    }
}

// Gradients of the rows of one operand, dealt out to the groups of the grid in turn; `dw` gathers the lane's 16 columns of the
// weight gradient over all its rows.
template <int LANES, bool BF16>
__device__ __forceinline__ void backward_rows(const NormParams &p, const NormSide &side, long long tokens, unsigned cta, unsigned ctas,
                                              float (&dw)[16]) {
    const int lane = threadIdx.x & (LANES - 1);
    const LanePlace l = lane_place(p, lane);
    const long long rows = tokens * side.heads;
    const long long groups = (long long)ctas * (kBackwardThreads / LANES);
    const long long rounds = (rows + groups - 1) / groups;
    // row of a round, its token and head
    struct Row {
        bool active;
        unsigned token;
        int head;
    };
    const auto row_of = [&](long long round) {
        const long long row = round * groups + (long long)cta * (kBackwardThreads / LANES) + threadIdx.x / LANES;
        Row o;
        o.active = row < rows && l.there;
        o.token = o.active ? (unsigned)row / (unsigned)side.heads : 0u;
        o.head = o.active ? (int)((unsigned)row - o.token * (unsigned)side.heads) : 0;
        return o;
    };
    Raw8<BF16> rx[2], rg[2];
    float nc[8], ns[8];
    const auto fetch = [&](const Row &o, int pos) {
        if (!o.active) return;
        const long long at = (long long)o.token * side.x_ts + (long long)o.head * side.x_hs;
        const long long dat = (long long)o.token * side.dy_ts + (long long)o.head * side.dy_hs;
        rx[0] = fetch8<BF16>(side.x, at + l.a);
        rx[1] = fetch8<BF16>(side.x, at + l.b);
        rg[0] = fetch8<BF16>(side.dy, dat + l.a);
        rg[1] = fetch8<BF16>(side.dy, dat + l.b);
        if (l.turned) load_angles(p, l, pos, nc, ns);
    };
    const auto position_of = [&](const Row &o) { return o.active && l.turned ? p.positions[o.token] : 0; };
    Row now = row_of(0), next = row_of(1);
    fetch(now, position_of(now));
    int next_pos = position_of(next);
    for (long long round = 0; round < rounds; ++round) {   // the whole warp stays: the sums below are its shuffles
        const bool active = now.active;
        const unsigned token = now.token;
        const int head = now.head;
        float x[16], g[16], c[8], s[8];
        float sum = 0.f;
        if (active) {
            widen8<BF16>(rx[0], x);
            widen8<BF16>(rx[1], x + 8);
            widen8<BF16>(rg[0], g);
            widen8<BF16>(rg[1], g + 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                c[i] = nc[i];
                s[i] = ns[i];
            }
        }
        // the next row and its angles are on their way while this one is worked on
        now = next;
        fetch(now, next_pos);
        next = row_of(round + 2);
        next_pos = position_of(next);
        if (active) {
            if (l.turned) turn(g, c, s, p.interleaved, -1.f);
#pragma unroll
            for (int i = 0; i < 16; ++i) sum = fmaf(x[i], x[i], sum);
        }
        sum = group_sum<LANES>(sum);
        const float r = rsqrtf(fmaf(sum, p.inv_dim, p.eps));
        float dot = 0.f;
        if (active) {
            float w[16];
            if (side.weight) {
                load8_again(side.weight + l.a, w);
                load8_again(side.weight + l.b, w + 8);
            } else {
#pragma unroll
                for (int i = 0; i < 16; ++i) w[i] = 1.f;
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                x[i] *= r;                       // n
                dw[i] = fmaf(g[i], x[i], dw[i]);
                g[i] *= w[i];
                dot = fmaf(g[i], x[i], dot);
            }
        }
        dot = group_sum<LANES>(dot) * p.inv_dim;
        if (active) {
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = r * (g[i] - x[i] * dot);
            const long long to = (long long)token * side.out_ts + (long long)head * side.out_hs;
            store8<BF16, true>(side.out, to + l.a, g);
            store8<BF16, true>(side.out, to + l.b, g + 8);
        }
    }
}

// Each CTA leaves its sums of the weight gradients in `partial`; the groups of the CTA are added in a fixed order.
// 8,191 tokens of 16 + 4 heads of 128 (bf16, 64 values turned) take 33 us with the sums' kernel, 3.9 TB/s.  What bounds it: 128
// registers leave two CTAs per SM, so 32 KB of loads in flight; with three the registers spill (57 us).
template <int LANES, bool BF16>
__global__ void __launch_bounds__(kBackwardThreads, 2) head_norm_rope_backward_kernel(NormParams p) {
    constexpr int GROUPS = kBackwardThreads / LANES;
    __shared__ float s_dw[GROUPS][LANES * 16 + 1];
    const long long tokens = actual_tokens(p);
    const LanePlace l = lane_place(p, threadIdx.x & (LANES - 1));
    const bool is_k = blockIdx.x >= (unsigned)p.q_ctas;
    float dw[16] = {};
    if (is_k) backward_rows<LANES, BF16>(p, p.k, tokens, blockIdx.x - p.q_ctas, gridDim.x - p.q_ctas, dw);
    else backward_rows<LANES, BF16>(p, p.q, tokens, blockIdx.x, p.q_ctas, dw);
    if (!p.partial) return;
    if (l.there) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s_dw[threadIdx.x / LANES][l.a + i] = dw[i];
            s_dw[threadIdx.x / LANES][l.b + i] = dw[8 + i];
        }
    }
    __syncthreads();
    for (int d = threadIdx.x; d < p.head_dim; d += kBackwardThreads) {
        float sum = 0.f;
#pragma unroll 8
        for (int g = 0; g < GROUPS; ++g) sum += s_dw[g][d];
        p.partial[(long long)blockIdx.x * p.head_dim + d] = sum;
    }
}

// Weight gradients from the CTAs' sums, 32 columns per CTA (of the queries' gradient, then of the keys'), always in the same order.
__global__ void __launch_bounds__(1024) norm_weight_sum_kernel(const float *partial, int q_ctas, int ctas, int head_dim, float *dq_weight,
                                                               float *dk_weight) {
    cudaGridDependencySynchronize();     // launched while the CTAs that write the sums still run
    __shared__ float s[32][33];
    const int half = gridDim.x / 2;
    const bool is_k = (int)blockIdx.x >= half;
    const int col = ((int)blockIdx.x - (is_k ? half : 0)) * 32 + (threadIdx.x & 31), part = threadIdx.x >> 5;
    float *const out = is_k ? dk_weight : dq_weight;
    if (!out) return;
    float sum = 0.f;
    if (col < head_dim)
        for (int b = (is_k ? q_ctas : 0) + part; b < (is_k ? ctas : q_ctas); b += 32) sum += partial[(long long)b * head_dim + col];
    s[part][threadIdx.x & 31] = sum;
    __syncthreads();
    if (part == 0 && col < head_dim) {
        float total = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += s[i][threadIdx.x];
        out[col] = total;
    }
}

bool norm_aligned(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int lanes_for(int head_dim) { return head_dim <= 16 ? 1 : head_dim <= 32 ? 2 : head_dim <= 64 ? 4 : head_dim <= 128 ? 8 : 16; }

template <int LANES>
void launch_norm(const NormParams &p, bool bf16, bool backward, unsigned grid, int sms, cudaStream_t stream) {
    if (backward) {
        if (bf16) head_norm_rope_backward_kernel<LANES, true><<<grid, kBackwardThreads, 0, stream>>>(p);
        else head_norm_rope_backward_kernel<LANES, false><<<grid, kBackwardThreads, 0, stream>>>(p);
        return;
    }
    const int per_cta = kNormThreads / LANES;
    const auto ctas = [&](int r) {
        const long long parts = (p.q.heads + r - 1) / r + (p.k.heads + r - 1) / r;
        return (unsigned)((p.tokens * parts + per_cta - 1) / per_cta);
    };
    if (ctas(1) <= (unsigned)sms * 16) {     // all groups are resident at once even with a head each
        if (bf16) head_norm_rope_kernel<LANES, true, 1><<<ctas(1), kNormThreads, 0, stream>>>(p);
        else head_norm_rope_kernel<LANES, false, 1><<<ctas(1), kNormThreads, 0, stream>>>(p);
    } else {
        if (bf16) head_norm_rope_kernel<LANES, true, 4><<<ctas(4), kNormThreads, 0, stream>>>(p);
        else head_norm_rope_kernel<LANES, false, 2><<<ctas(2), kNormThreads, 0, stream>>>(p);
    }
}

void launch_norm_lanes(int lanes, const NormParams &p, bool bf16, bool backward, unsigned grid, int sms, cudaStream_t stream) {
    switch (lanes) {
        case 1: launch_norm<1>(p, bf16, backward, grid, sms, stream); break;
        case 2: launch_norm<2>(p, bf16, backward, grid, sms, stream); break;
        case 4: launch_norm<4>(p, bf16, backward, grid, sms, stream); break;
        case 8: launch_norm<8>(p, bf16, backward, grid, sms, stream); break;
        default: launch_norm<16>(p, bf16, backward, grid, sms, stream); break;
    }
}

fi_status_t current_sms(int *sms, const char *name) {
    int device = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(sms, cudaDevAttrMultiProcessorCount, device);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, name);
}

fi_status_t check_norm_args(const fi_head_norm_rope_t *a, bool backward, const char *name) {
    if (!a) {
        set_error("%s: null argument", name);
        return FI_ERR_INVALID_ARG;
    }
    if (a->dtype != FI_F32 && a->dtype != FI_BF16) {
        set_error("%s: dtype must be FI_F32 or FI_BF16", name);
        return FI_ERR_INVALID_ARG;
    }
    if (a->head_dim < 16 || a->head_dim > 256 || a->head_dim % 16 || a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 16 ||
        a->q_heads < 1 || a->k_heads < 0 || a->tokens < 0 || a->max_pos < 0 ||
        a->tokens * ((long long)a->q_heads + a->k_heads) > 2147483647ll || a->tokens > 2147483647ll) {
        set_error("%s: head_dim and rot_dim multiples of 16 with rot_dim <= head_dim <= 256, q_heads >= 1, k_heads >= 0, and "
                  "tokens * heads below 2^31 (got head_dim %d, rot_dim %d, heads %d + %d)", name, a->head_dim, a->rot_dim, a->q_heads,
                  a->k_heads);
        return FI_ERR_INVALID_ARG;
    }
    const bool k = a->k_heads > 0;
    if (a->tokens > 0 && (!a->q || !a->q_out || (k && (!a->k || !a->k_out)) || (a->rot_dim > 0 && (!a->rope || !a->positions)) ||
                          (backward && (!a->dq_out || (k && !a->dk_out))))) {
        set_error("%s: null pointer", name);
        return FI_ERR_INVALID_ARG;
    }
    if (backward && (a->dq_weight || a->dk_weight) && !a->workspace) {
        set_error("%s: weight gradients need a workspace", name);
        return FI_ERR_INVALID_ARG;
    }
    const int unit = a->dtype == FI_BF16 ? 8 : 4;
    const int64_t strides[12] = {a->q_token_stride, a->q_head_stride, k ? a->k_token_stride : 0, k ? a->k_head_stride : 0,
                                 a->q_out_token_stride, a->q_out_head_stride, k ? a->k_out_token_stride : 0, k ? a->k_out_head_stride : 0,
                                 backward ? a->dq_out_token_stride : 0, backward ? a->dq_out_head_stride : 0,
                                 backward && k ? a->dk_out_token_stride : 0, backward && k ? a->dk_out_head_stride : 0};
    bool ok = norm_aligned(a->q) && norm_aligned(a->q_out) && (!k || (norm_aligned(a->k) && norm_aligned(a->k_out))) &&
              norm_aligned(a->q_weight) && norm_aligned(a->k_weight) && norm_aligned(a->rope) &&
              (!backward || (norm_aligned(a->dq_out) && (!k || norm_aligned(a->dk_out)) && norm_aligned(a->workspace)));
    for (int i = 0; i < 12; ++i) {     // (strides between tokens and between heads in turn; of a single one it may be anything)
        const int64_t count = i % 2 == 0 ? a->tokens : i % 4 == 1 ? a->q_heads : a->k_heads;
        ok = ok && (count <= 1 || (strides[i] >= 0 && strides[i] % unit == 0));
    }
    if (!ok) {
        set_error("%s: heads, weights and the rope table must start on 16-byte boundaries, strides must not be negative", name);
        return FI_ERR_INVALID_ARG;
    }
    return FI_OK;
}

NormParams norm_params(const fi_head_norm_rope_t *a, bool backward) {
    NormParams p = {};
    p.q = {a->q, a->dq_out, a->q_out, a->q_weight, a->q_token_stride, a->q_head_stride, a->dq_out_token_stride,
           a->dq_out_head_stride, a->q_out_token_stride, a->q_out_head_stride, a->q_heads};
    p.k = {a->k, a->dk_out, a->k_out, a->k_weight, a->k_token_stride, a->k_head_stride, a->dk_out_token_stride,
           a->dk_out_head_stride, a->k_out_token_stride, a->k_out_head_stride, a->k_heads};
    p.rope = a->rope;
    p.positions = a->positions;
    p.tokens_dev = a->tokens_dev;
    p.partial = backward && (a->dq_weight || a->dk_weight) ? static_cast<float *>(a->workspace) : nullptr;
    p.tokens = a->tokens;
    p.head_dim = a->head_dim;
    p.rot = a->rot_dim;
    p.max_pos = a->max_pos;
    p.interleaved = a->interleaved != 0;
    p.eps = a->eps;
    p.inv_dim = 1.f / (float)a->head_dim;
    return p;
}

}  // namespace
}  // namespace fi

using namespace fi;

extern "C" {

int64_t fi_head_norm_rope_workspace(int32_t head_dim) {
    return head_dim < 16 || head_dim > 256 ? 0 : (int64_t)kMaxPartials * head_dim * sizeof(float);
}

fi_status_t fi_head_norm_rope(const fi_head_norm_rope_t *a, void *cuda_stream) {
    fi_status_t st = check_norm_args(a, false, "fi_head_norm_rope");
    if (st != FI_OK || a->tokens == 0) return st;
    int sms = 0;
    st = current_sms(&sms, "fi_head_norm_rope");
    if (st != FI_OK) return st;
    launch_norm_lanes(lanes_for(a->head_dim), norm_params(a, false), a->dtype == FI_BF16, false, 0, sms, static_cast<cudaStream_t>(cuda_stream));
    count_launch();
    return check_launch("fi_head_norm_rope");
}

fi_status_t fi_head_norm_rope_backward(const fi_head_norm_rope_t *a, void *cuda_stream) {
    fi_status_t st = check_norm_args(a, true, "fi_head_norm_rope_backward");
    if (st != FI_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    NormParams p = norm_params(a, true);
    int sms = 0;
    st = current_sms(&sms, "fi_head_norm_rope_backward");
    if (st != FI_OK) return st;
    // as many CTAs as are resident at once, dealt out to queries and keys by their numbers of rows
    const int lanes = lanes_for(a->head_dim), per_cta = kBackwardThreads / lanes;
    const long long most = sms * 2 < kMaxPartials ? sms * 2 : kMaxPartials;
    const long long q_rows = a->tokens * (long long)a->q_heads, k_rows = a->tokens * (long long)a->k_heads;
    long long q_ctas = (q_rows + per_cta - 1) / per_cta, k_ctas = (k_rows + per_cta - 1) / per_cta;
    if (q_ctas + k_ctas > most) {
        k_ctas = k_rows ? (most * k_rows + (q_rows + k_rows) / 2) / (q_rows + k_rows) : 0;
        if (k_rows && k_ctas < 1) k_ctas = 1;
        q_ctas = most - k_ctas;
    }
    if (q_ctas < 1) q_ctas = 1;                       // no tokens: the sums are zero
    if (a->k_heads > 0 && k_ctas < 1) k_ctas = 1;
    const int grid = (int)(q_ctas + k_ctas);
    p.q_ctas = (int)q_ctas;
    launch_norm_lanes(lanes, p, a->dtype == FI_BF16, true, (unsigned)grid, sms, stream);
    count_launch();
    if (p.partial) {   // launched before the first kernel ends, which it waits for: the call takes 36.2 us, not 38.6
        cudaLaunchAttribute early;
        early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
        early.val.programmaticStreamSerializationAllowed = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(2 * ((a->head_dim + 31) / 32));
        cfg.blockDim = dim3(1024);
        cfg.stream = stream;
        cfg.attrs = &early;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaLaunchKernelEx(&cfg, norm_weight_sum_kernel, (const float *)p.partial, p.q_ctas, grid, (int)a->head_dim,
                                                 a->dq_weight, a->k_heads > 0 ? a->dk_weight : (float *)nullptr);
        if (e != cudaSuccess) return cuda_fail(e, "fi_head_norm_rope_backward");
        count_launch();
    }
    return check_launch("fi_head_norm_rope_backward");
}

}  // extern "C"

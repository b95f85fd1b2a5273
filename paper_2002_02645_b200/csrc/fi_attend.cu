// Attention over keys and values held in 4 bits.
//
// With k = n s_k + m_k and v = n' s_v + m_v (codes n, n' in 0..15; one scale and offset per token and key head)
//   x_t = scale log2(e) (s_k (q . n) + m_k sum(q)),   out = sum_t p_t (s_v n' + m_v) / sum_t p_t,   p_t = 2^(x_t - max)
// so scales and offsets never touch the codes: the products run on the codes themselves, and the offset of v is one
// sum per query row.  The scale of v goes into the exponent: with y_t = x_t + log2(s_v) and M = max y - 7 as it was when a y last
// went over M + 15, the weight P_t = 2^(y_t - M) multiplies n' directly, sum p_t = sum P_t / s_v and the offset's part is
// sum P_t m_v / s_v.  So the largest weight is between 2^7 and 2^15 as a half, whose last place is 2^-24 for all weights below
// 2^-14: a weight is off by 2^-12 of itself or 2^-32 of the largest (float32 queries, with two halves: 2^-22 or 2^-32).  With weights up
// to 1 instead, 32,763 float32 weights 8 nats below the largest were off by 2^-12 of themselves.
//
// A code is a half-precision number without any conversion: a 16-bit word that holds only the four bits n is the
// subnormal n 2^-24 (n 2^-20 when it sits in the next four bits), which the tensor cores multiply exactly.  Eight codes
// cost one shift and four masks; the powers of two are taken back once per row.
//
// Codes are all positive, so the product part and the offset part are larger than what they add up to.  The offset part
// therefore takes the weights as they were rounded for the product, and float32 queries, which must not lose what the parts have in
// common, take the codes less 7.5 (one more instruction per two codes) and offsets moved by 7.5 scales.
// Tensor cores cut what they add, so a sum kept there shrinks with every product (bf16 queries over 100,000 keys of a warp: by more
// than the result's rounding).  So they add up 32 keys, and long sums are kept outside of them, which takes 5 % longer (64 requests of
// 800 to 8,192 keys: 86.7 -> 91.5 us).  Taking them out every 16 steps only, into scratch of 16 KB per CTA, took 89.4 us; into tensor
// memory 169 us, because fewer CTAs of a kernel that has some run per SM.
// A value vector of hardly any spread (a constant one has the smallest scale there is) is all offset: its P_t is far below the
// others' and may round to nothing, although its p_t is like theirs.  Where the offset is more than kMostlyOffset scales, the
// offset part takes the weight as it was before the rounding: what the two parts then differ in, 2^-12 of 15 scales, is below
// 2^-13 of the value.  Up to there a weight that rounds to nothing loses 2^-25 of the largest product at most.
#include "fi_attend.cuh"

namespace fi {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kStages = 2;                 // steps of a warp in its ring: the one it works on and the next
constexpr float kMostlyOffset = 64.f;      // offset over scale of a value vector that is its offset more than its codes

__device__ __forceinline__ float lg2(float x) {
    float y;
    asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// log2 of a scale, off by 2^-22 whatever its size (lg2 alone: of the result's size, and a scale of 2^-40 is a weight off by 4e-6)
__device__ __forceinline__ float log2_scale(float x) {
    const uint32_t bits = __float_as_uint(x);
    return (float)((int)(bits >> 23) - 127) + lg2(__uint_as_float((bits & 0x7fffffu) | 0x3f800000u));
}

__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(h);
}

// what pack_half left over
__device__ __forceinline__ uint32_t pack_rest(uint32_t packed, float lo, float hi) {
    const float2 f = __half22float2(reinterpret_cast<const __half2 &>(packed));
    return pack_half(lo - f.x, hi - f.y);
}

// Two codes as halves: n 2^-24 (ROW 0) or n 2^-20 (ROW 1) as they are, or 2^10 (n - 7.5) times that when CENTRED.
template <bool CENTRED, int ROW>
__device__ __forceinline__ uint32_t codes(uint32_t w) {
    if constexpr (CENTRED) {
        const uint32_t grow = 0x64006400u;                                  // 2^10
        const uint32_t less = ROW ? 0x9f809f80u : 0x8f808f80u;              // -7.5 2^-10, -7.5 2^-14
        const __half2 h = __hfma2(reinterpret_cast<const __half2 &>(w), reinterpret_cast<const __half2 &>(grow),
                                  reinterpret_cast<const __half2 &>(less));
        return reinterpret_cast<const uint32_t &>(h);
    } else {
        return w;
    }
}

// N words of shared memory from an address that is a multiple of 4 * (largest power of two in N) bytes
template <int N>
__device__ __forceinline__ void load_words(const unsigned char *p, uint32_t *w) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = *(reinterpret_cast<const uint4 *>(p) + i);
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
    } else if constexpr (N % 2 == 0) {
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const uint2 v = *(reinterpret_cast<const uint2 *>(p) + i);
            w[2 * i] = v.x; w[2 * i + 1] = v.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = *(reinterpret_cast<const uint32_t *>(p) + i);
    }
}

template <int BYTES>
__device__ __forceinline__ void async_copy(uint32_t dst, const void *src) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

__device__ __forceinline__ void async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }

template <int N>
__device__ __forceinline__ void async_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// One request as the kernel sees it.
struct Request {
    int row, len, queries, first_token;   // queries = 0: nothing to do
    int unit0, units, row_tiles;          // key units it reads, tiles of query rows per key head
};

// blocks of 16 keys a warp takes per step, and keys a CTA does (a unit): with 8 rows there are registers for four blocks,
// whose products, exponentials and copies overlap; two blocks take 7 % longer on 64 requests of 800 to 8,192 keys
template <int D, int NT>
__host__ __device__ constexpr int blocks() { return D <= 128 && NT == 1 ? 4 : 2; }

template <int D, int NT>
__host__ __device__ constexpr int unit_keys() { return kWarps * 16 * blocks<D, NT>(); }

template <int ROWS, int UNIT>
__device__ __forceinline__ Request request_of(const AttendParams &p, int i) {
    Request r;
    r.first_token = p.cu_tokens ? p.cu_tokens[i] : i;
    r.queries = p.cu_tokens ? p.cu_tokens[i + 1] - r.first_token : 1;
    r.row = p.row_idx ? p.row_idx[i] : i;
    if (r.row < 0 || r.row >= p.rows || r.first_token < 0 || r.queries < 0 || r.queries > p.max_tokens - r.first_token) r.queries = 0;
    r.len = r.queries > 0 ? p.lens[r.row] : 0;
    const long long most = (long long)p.max_blocks << p.page_shift;
    if (r.len > most) r.len = (int)most;
    if (r.len < 0 || (p.granted && p.granted[i] < r.queries)) r.len = 0;     // (a refused request sees nothing)
    long long lo = 0;
    if (p.window > 0) {
        lo = (long long)max(r.len - r.queries, 0) - p.window + 1;
        if (lo < 0) lo = 0;
    }
    r.unit0 = (int)(lo / UNIT);
    const int end = (r.len + UNIT - 1) / UNIT;
    r.units = end > r.unit0 ? end - r.unit0 : 1;      // a request without keys still gets its zeros
    r.row_tiles = (int)(((long long)r.queries * p.group + ROWS - 1) / ROWS);
    return r;
}

// One step of a warp: the codes and the meta of 16 NB keys.
template <int D, int NB>
struct Stage {
    unsigned char k[NB * 8 * D], v[NB * 8 * D];
    uint32_t meta[NB][2][16];         // block of 16 keys; keys, values
};

// What the weights need of a key, worked out once per key.
template <int NB>
struct KeyFactors {
    float4 f[16 * NB];                // scale and offset of the key, log2 of the value's scale and its reciprocal
    float off[16 * NB];               // the value's offset over its scale
};

constexpr uint32_t kNoPage = 0xffffffffu;

// The walk over a CTA's share of the (request, tile of query rows, key head, unit of keys) units, in that order.
struct Walk {
    long long u, u_end, request_start;
    int request;
};

// A piece of the walk: consecutive units of one request, tile and head.
struct Piece {
    Request r;
    int head, tile, unit, steps;
    long long item_begin, item_end;   // all units of that request, tile and head
};

// a * b / c without a 64-bit division where 32 bits hold the product
__device__ __forceinline__ long long mul_div(long long a, long long b, long long c) {
    const unsigned long long m = (unsigned long long)a * (unsigned long long)b;
    return m >> 32 ? (long long)(m / (unsigned long long)c) : (long long)((uint32_t)m / (uint32_t)c);
}

// the CTA whose share [total i / ctas, total (i + 1) / ctas) holds unit u
__device__ __forceinline__ long long owner_of(long long u, long long ctas, long long total) {
    const unsigned long long m = (unsigned long long)(u + 1) * (unsigned long long)ctas - 1;
    return m >> 32 || total >> 32 ? (long long)(m / (unsigned long long)total) : (long long)((uint32_t)m / (uint32_t)total);
}

template <int ROWS, int UNIT>
__device__ __forceinline__ bool next_piece(const AttendParams &p, Walk &w, Piece &x) {
    while (w.u < w.u_end) {
        x.r = request_of<ROWS, UNIT>(p, w.request);
        const long long here = x.r.queries > 0 ? (long long)x.r.units * x.r.row_tiles * p.kv_heads : 0;
        if (w.u >= w.request_start + here) {
            w.request_start += here;
            ++w.request;
            continue;
        }
        const long long in_request = mul_div(w.u - w.request_start, 1, x.r.units);
        x.unit = (int)((w.u - w.request_start) - in_request * x.r.units);
        x.tile = (int)mul_div(in_request, 1, p.kv_heads);
        x.head = (int)(in_request - (long long)x.tile * p.kv_heads);
        x.item_begin = w.u - x.unit;
        x.item_end = x.item_begin + x.r.units;
        x.steps = (int)((x.item_end < w.u_end ? x.item_end : w.u_end) - w.u);
        return true;
    }
    return false;
}

// Result of a query row from its sums: weights' total, offsets' part, maximum.
template <bool F32>
__device__ __forceinline__ void store_out(void *out, long long at, const float *o, int n) {
    if constexpr (F32) {
        float4 *d = reinterpret_cast<float4 *>(static_cast<float *>(out) + at);
        for (int i = 0; i < n / 4; ++i) d[i] = make_float4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    } else {
        uint2 *d = reinterpret_cast<uint2 *>(static_cast<__nv_bfloat16 *>(out) + at);
        for (int i = 0; i < n / 4; ++i) {
            const __nv_bfloat162 a = __floats2bfloat162_rn(o[4 * i], o[4 * i + 1]), b = __floats2bfloat162_rn(o[4 * i + 2], o[4 * i + 3]);
            d[i] = make_uint2(reinterpret_cast<const uint32_t &>(a), reinterpret_cast<const uint32_t &>(b));
        }
    }
}

template <int D, int NT>
__host__ __device__ constexpr int slot_floats() { return 8 * NT * (D + 4); }

// CTAs per SM the registers are cut to
template <int D, int NT>
__host__ __device__ constexpr int min_ctas() { return D * NT <= 192 ? 3 : 2; }

// shared memory: the warps' rings, later the warps' results; then the statistics and the queries
template <int D, int NT>
__host__ __device__ constexpr int ring_bytes() {
    return kWarps * kStages * (int)sizeof(Stage<D, blocks<D, NT>()>) > kWarps * 8 * (D + 4) * 4
               ? kWarps * kStages * (int)sizeof(Stage<D, blocks<D, NT>()>) : kWarps * 8 * (D + 4) * 4;
}

template <int D, int NT, bool F32>
constexpr int attend_smem() {
    return ring_bytes<D, NT>() + kWarps * 8 * NT * 16 + NT * (D / 16) * 32 * 8 * (F32 ? 2 : 1);
}

// A CTA takes an equal share of all (request, tile of query rows, key head, unit of keys) units, whatever requests they
// belong to; each of its four warps works on a quarter of a unit at a time against the tile's 8 NT rows.  A warp fetches its
// own codes, a step ahead, with 16-byte asynchronous copies into its own ring (every byte of a code row is used by one lane
// only, so warps have nothing to share, and they never wait for each other until a request is done).  Keys are the rows of the products
// (m16), query rows their columns (n8), so that the usual 4 to 8 query heads of a key head fill a tile:
//   S^T[key, row] = K Q^T,  O^T[dim, row] += V^T P^T
// The product over head_dim runs in the order in which lanes hold the codes; q is laid out to match.
// 8 key heads of 128 over 262,143 keys of one request take 76 us, 3.8 TB/s; 64 requests of 800 to 8,192 keys 93 us.
// What bounds it: the loop's instructions (a further 131,072 keys of 8 heads take 27 us, 5.3 TB/s: 7 cycles per key and SM); the
// start of a CTA (2 us to the first request for codes), the SMs' unequal speeds on equal shares, the partial results and their join
// come on top, and so does the start of each further piece, which overlaps with the other CTAs of the SM only in part.
template <int D, int NT, bool F32>
__global__ void __launch_bounds__(kThreads, (min_ctas<D, NT>())) kv_attend_kernel(const AttendParams p) {
    constexpr int ROWS = 8 * NT;
    constexpr int KS = D / 16;              // steps of 16 in the product over head_dim
    constexpr int WV = D / 64;              // words of a value row per lane
    constexpr int CH = D / 32;              // 16-byte pieces of a code row
    constexpr int LD = D + 4;
    constexpr int NB = blocks<D, NT>(), UNIT = unit_keys<D, NT>(), WARP_KEYS = 16 * NB;
    constexpr float kBack = F32 ? 0x1p14f : 0x1p24f;   // takes back the powers of two of codes<F32, 0>()
    extern __shared__ __align__(128) unsigned char smem[];
    float *const s_o = reinterpret_cast<float *>(smem);        // [warps][8][LD]
    float *const s_stat = reinterpret_cast<float *>(smem + ring_bytes<D, NT>());    // [warps][ROWS][4]: maximum, sum, offset sum
    uint2 *const s_q = reinterpret_cast<uint2 *>(s_stat + kWarps * ROWS * 4);   // [1 or 2][NT][KS][32]
    __shared__ long long s_sum[kWarps];
    __shared__ long long s_start;
    __shared__ int s_request;
    __shared__ bool s_last;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, c = lane & 3;
    Stage<D, NB> *const ring = reinterpret_cast<Stage<D, NB> *>(smem) + warp * kStages;
    const uint32_t ring_at = smem_at(ring);
    // ---- this CTA's share ----
    int n = p.batch_max;
    if (p.batch_count) n = min(max(*p.batch_count, 0), p.batch_max);
    const int per_thread = (p.batch_max + kThreads - 1) / kThreads;
    long long mine = 0;
    for (int e = 0; e < per_thread; ++e) {
        const int i = tid * per_thread + e;
        if (i < p.batch_max) {      // all entries are read, so that their loads need not wait for the count
            const Request r = request_of<ROWS, UNIT>(p, i);
            if (i < n && r.queries > 0) mine += (long long)r.units * r.row_tiles * p.kv_heads;
        }
    }
    long long before = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long o = __shfl_up_sync(0xffffffffu, before, d);
        if (lane >= d) before += o;
    }
    if (lane == 31) s_sum[warp] = before;
    __syncthreads();
    long long total = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        const long long s = s_sum[w];
        if (w < warp) before += s;
        total += s;
    }
    before -= mine;
    if (total == 0) return;
    const long long ctas = total < gridDim.x ? total : gridDim.x;
    if (blockIdx.x >= ctas) return;
    Walk walk;
    walk.u = mul_div(total, blockIdx.x, ctas);
    walk.u_end = mul_div(total, blockIdx.x + 1, ctas);
    if (before <= walk.u && walk.u < before + mine) {
        int i = tid * per_thread;
        long long at = before;
        for (;; ++i) {
            const Request r = request_of<ROWS, UNIT>(p, i);
            const long long here = r.queries > 0 ? (long long)r.units * r.row_tiles * p.kv_heads : 0;
            if (walk.u < at + here) break;
            at += here;
        }
        s_request = i;
        s_start = at;
    }
    __syncthreads();
    walk.request = s_request;
    walk.request_start = s_start;

    const long long u_first = walk.u;
    Piece x;
    while (next_piece<ROWS, UNIT>(p, walk, x)) {
        const Request &r = x.r;
        const int head = x.head, tile = x.tile, steps = x.steps;
        const long long item_begin = x.item_begin, item_end = x.item_end;
        const int total_rows = r.queries * p.group;
        const int row0 = tile * ROWS;

        // ---- the first keys and values on their way ----
        const int32_t *const table = p.block_table + (long long)r.row * p.table_ld;
        int first_key = 0;                                // that any query sees
        if (p.window > 0) first_key = max(max(r.len - r.queries, 0) - p.window + 1, 0);
        // a 16-key block of codes is CH / 2 pieces of 16 bytes per lane; where they are in a page's first block:
        const unsigned char *k_from[CH / 2], *v_from[CH / 2];
#pragma unroll
        for (int i = 0; i < CH / 2; ++i) {
            const int piece = lane + 32 * i, key = piece / CH, part = piece - key * CH;
            const long long at = head * p.hs + ((long long)key * p.ts + part) * 16;
            k_from[i] = p.k_codes + at;
            v_from[i] = p.v_codes + at;
        }
        const uint32_t *const meta_from = (lane < 16 ? p.k_meta : p.v_meta) + head * p.mhs + (lane & 15) * p.mts;
        const int place_mask = (1 << p.page_shift) - 1;
        int tok = (r.unit0 + x.unit) * UNIT + warp * WARP_KEYS;
        // lane l looks up the page of block l mod NB, kNoPage past the end
        const auto page_at = [&](int t) {
            t += 16 * (lane & (NB - 1));
            return t < r.len ? min((uint32_t)__ldg(table + (t >> p.page_shift)), kNoPage - 1) : kNoPage;
        };
        uint32_t brought = 0;                             // NB bits per step on the way, the latest lowest: its blocks
        uint32_t fill = ring_at + lane * 16;
        // fetches the warp's keys at t, whose pages the lanes hold
        const auto fetch = [&](int t, uint32_t page_l) {
            brought <<= NB;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const uint32_t page = __shfl_sync(0xffffffffu, page_l, b);
                const int at = t + 16 * b;
                if (page < (uint32_t)p.num_pages) {
                    if (at + 16 > first_key) {
                        brought |= 1u << b;
                        const uint32_t place = at & place_mask, off = page * p.ps + place * p.ts, moff = page * p.mps + place * p.mts;
#pragma unroll
                        for (int i = 0; i < CH / 2; ++i) {
                            async_copy<16>(fill + b * 8 * D + i * 512, k_from[i] + off * 16ull);
                            async_copy<16>(fill + (NB + b) * 8 * D + i * 512, v_from[i] + off * 16ull);
                        }
                        async_copy<4>(fill - lane * 12 + NB * 16 * D + b * 128, meta_from + moff);
                    }
                } else if (page != kNoPage && at + 16 > first_key && lane == 0) {
                    atomicOr(p.status, 2);
                }
            }
            async_commit();
            fill = fill >= ring_at + (uint32_t)sizeof(Stage<D, NB>) ? ring_at + lane * 16 : fill + (uint32_t)sizeof(Stage<D, NB>);
        };
        fetch(tok, page_at(tok));
        uint32_t next_page = steps > 1 ? page_at(tok + UNIT) : kNoPage;

        // ---- the tile's queries, as halves, laid out as the products take them ----
        float cq[NT][2], sq[NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int row = row0 + nt * 8 + g;
            const bool real = row < total_rows;
            const int j = real ? row / p.group : 0, qh = real ? head * p.group + row - j * p.group : 0;
            const long long at = (long long)(r.first_token + j) * p.q_ts + (long long)qh * p.q_hs + c * (D / 4);
            float x[D / 4];
            float top = 0.f, sum = 0.f;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                float *const v = x + 8 * i;
                if (!real) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = 0.f;
                } else if constexpr (F32) {
                    const float4 *s = reinterpret_cast<const float4 *>(static_cast<const float *>(p.q) + at + 8 * i);
                    const float4 lo = __ldg(s), hi = __ldg(s + 1);
                    v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w; v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
                } else {
                    const uint4 s = __ldg(reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) + at + 8 * i));
                    const uint32_t w[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[2 * e] = __uint_as_float(w[e] << 16);
                        v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    top = fmaxf(top, fabsf(v[e]));
                    sum += v[e];
                }
            }
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                sum += __shfl_xor_sync(0xffffffffu, sum, d);
            }
            // the row's largest value goes to 2^14 .. 2^15: bf16 values stay exact as halves
            int up = 0;
            if (top > 0.f && top < INFINITY) {
                up = 141 - (int)(__float_as_uint(top) >> 23);
                up = up < -110 ? -110 : up > 110 ? 110 : up;
            }
            const float f = __uint_as_float((uint32_t)(127 + up) << 23);
            if (warp == nt % kWarps) {
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const float *const v = x + 8 * i;
                    // codes in the upper four bits of a byte count 16 times as much
                    const float f16 = f * 0.0625f;
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float a0 = v[2 * h] * f, a1 = v[2 * h + 4] * f, b0 = v[2 * h + 1] * f16, b1 = v[2 * h + 5] * f16;
                        const uint2 w = make_uint2(pack_half(a0, a1), pack_half(b0, b1));
                        s_q[(nt * KS + 2 * i + h) * 32 + lane] = w;
                        if constexpr (F32)
                            s_q[((NT + nt) * KS + 2 * i + h) * 32 + lane] = make_uint2(pack_rest(w.x, a0, a1), pack_rest(w.y, b0, b1));
                    }
                }
            }
            const float back = p.scale_log2 * __uint_as_float((uint32_t)(127 - up) << 23) * kBack;
            sum *= p.scale_log2;
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // columns of the products: rows 2c, 2c + 1
                cq[nt][h] = __shfl_sync(0xffffffffu, back, (2 * c + h) * 4);
                sq[nt][h] = __shfl_sync(0xffffffffu, sum, (2 * c + h) * 4);
            }
        }
        // keys a row sees: [low, high).  Rows past the last query see what the last one sees; they are never stored.
        int high[NT][2], low[NT][2];
        int all_high, any_high, all_low, any_low;   // keys every row, any row of the tile sees
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int row = min(row0 + nt * 8 + 2 * c + h, total_rows - 1);
                const int pos = r.len - r.queries + row / p.group;
                high[nt][h] = pos + 1;
                low[nt][h] = p.window > 0 ? max(pos, 0) - p.window + 1 : 0;
            }
        {
            const int first = r.len - r.queries + row0 / p.group, last = r.len - r.queries + (min(row0 + ROWS, total_rows) - 1) / p.group;
            all_high = first + 1;
            any_high = last + 1;
            all_low = p.window > 0 ? max(last, 0) - p.window + 1 : 0;
            any_low = p.window > 0 ? max(first, 0) - p.window + 1 : 0;
        }
        __syncthreads();

        float o[KS][NT][4];
        float top[NT][2], sum[NT][2], lost[NT][2], off[NT][2];
#pragma unroll
        for (int i = 0; i < KS; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][nt][e] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                top[nt][h] = kNoMax;
                sum[nt][h] = lost[nt][h] = off[nt][h] = 0.f;
            }

        Stage<D, NB> *drain = ring;
        for (int step = 0; step < steps; ++step, tok += UNIT) {
            fetch(tok + UNIT, next_page);
            next_page = step + 2 < steps ? page_at(tok + 2 * UNIT) : kNoPage;
            async_wait<1>();
            __syncwarp();
            Stage<D, NB> &st = *drain;
            const uint32_t valid = (brought >> NB) & ((1u << NB) - 1);
            const bool work = tok < any_high && tok + WARP_KEYS > any_low;
            const bool whole = tok + WARP_KEYS <= all_high && tok >= all_low && valid == (1u << NB) - 1;

            if (work) {
                // ---- S^T = K Q^T: lane (g, c) holds the c-th quarter of keys g and g + 8 of each block of 16 ----
                float s[NB][NT][4];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[b][nt][e] = 0.f;
                uint32_t kw[NB][2][D / 32];
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int e = 0; e < 2; ++e)
                        load_words<D / 32>(st.k + (16 * b + 8 * e + g) * (D / 2) + c * (D / 8), kw[b][e]);
                // the codes of the keys are in registers: their place takes the keys' factors
                KeyFactors<NB> &my_key = *reinterpret_cast<KeyFactors<NB> *>(st.k);
                static_assert(sizeof(KeyFactors<NB>) <= sizeof(st.k), "factors must fit");
                __syncwarp();
                bool flat = false;     // a value vector of the step is mostly offset
#pragma unroll
                for (int k = lane; k < WARP_KEYS; k += 32) {
                    const uint32_t km = st.meta[k >> 4][0][k & 15], vm = st.meta[k >> 4][1][k & 15];
                    // (a scale below 2^-30 of the offset counts as that: codes times it are nothing to the value, and the quotient of the
                    // two stays finite)
                    const float sk = meta_scale(km), sv = fmaxf(fmaxf(meta_scale(vm), kMinScale), fabsf(meta_offset(vm)) * 0x1p-30f);
                    float mk = meta_offset(km), mv = meta_offset(vm), inv;
                    if constexpr (F32) {
                        mk = fmaf(7.5f, sk, mk);
                        mv = fmaf(7.5f, sv, mv);
                        inv = __frcp_rn(sv);
                    } else {
                        inv = rcp(sv);
                    }
                    my_key.f[k] = make_float4(sk, mk, log2_scale(sv), inv);
                    my_key.off[k] = mv * inv;
                    flat = flat || fabsf(mv * inv) > kMostlyOffset;
                }
                const bool ordinary = whole && !__any_sync(0xffffffffu, flat);
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    uint2 q[NT], q2[NT];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        q[nt] = s_q[(nt * KS + ks) * 32 + lane];
                        if constexpr (F32) q2[nt] = s_q[((NT + nt) * KS + ks) * 32 + lane];
                    }
#pragma unroll
                    for (int b = 0; b < NB; ++b) {
                        const uint32_t w0 = kw[b][0][ks >> 1] >> ((ks & 1) * 8), w1 = kw[b][1][ks >> 1] >> ((ks & 1) * 8);
                        const uint32_t a[4] = {codes<F32, 0>(w0 & 0x000f000fu), codes<F32, 0>(w1 & 0x000f000fu),
                                               codes<F32, 1>(w0 & 0x00f000f0u), codes<F32, 1>(w1 & 0x00f000f0u)};
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            mma(s[b][nt], a, q[nt].x, q[nt].y);
                            if constexpr (F32) mma(s[b][nt], a, q2[nt].x, q2[nt].y);
                        }
                    }
                }
                __syncwarp();     // the keys' factors are there
                uint32_t pb[NB][NT][2], pb2[NB][NT][2];
                // ordinary: every row of the tile sees all keys of the step, and no value vector is mostly offset
                auto weights = [&](auto ordinary_) {
                    constexpr bool ORDINARY = decltype(ordinary_)::value;
                    float inv[NB][2];
#pragma unroll
                    for (int b = 0; b < NB; ++b)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {      // keys g and g + 8
                            const float4 f = my_key.f[16 * b + 8 * e + g];
                            inv[b][e] = f.w;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    float &x = s[b][nt][2 * e + h];
                                    x = fmaf(x * cq[nt][h], f.x, fmaf(f.y, sq[nt][h], f.z));
                                    if constexpr (!ORDINARY) {
                                        const int t = tok + 16 * b + 8 * e + g;
                                        if (t >= high[nt][h] || t < low[nt][h] || !((valid >> b) & 1)) x = -INFINITY;
                                    }
                                }
                        }
                    bool grow = false;
                float most[NT][2];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        most[nt][h] = s[0][nt][h];
#pragma unroll
                        for (int b = 0; b < NB; ++b) most[nt][h] = fmaxf(fmaxf(most[nt][h], s[b][nt][h]), s[b][nt][2 + h]);
                        grow = grow || most[nt][h] - top[nt][h] > kMost;     // (the difference is exact where it matters)
                    }
                if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float m = most[nt][h];
#pragma unroll
                            for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                            m = fmaxf(m - kStart, top[nt][h]);
                            const float f = ex2(top[nt][h] - m);
                            top[nt][h] = m;
                            sum[nt][h] *= f;
                            lost[nt][h] *= f;
                            off[nt][h] *= f;
#pragma unroll
                            for (int i = 0; i < KS; ++i) {
                                o[i][nt][h] *= f;
                                o[i][nt][2 + h] *= f;
                            }
                        }
                }
                // a step's weights are added up by themselves first: long sums are rounded once a step and lane, and what the
                // softmax sum loses there is kept (32,768 keys of one CTA, nearly all alike: the logarithm of the sum was off by
                // 2e-5, and by 9e-6 with steps alone)
                float part_sum[NT][2] = {}, part_off[NT][2] = {};
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const float offv = my_key.off[16 * b + 8 * e + g];
                            const float x0 = s[b][nt][2 * e], x1 = s[b][nt][2 * e + 1];
                            const float w0 = ex2(x0 - top[nt][0]), w1 = ex2(x1 - top[nt][1]);
                            const uint32_t packed = pack_half(w0, w1);
                            float2 w = __half22float2(reinterpret_cast<const __half2 &>(packed));
                            pb[b][nt][e] = transpose8x8(packed);
                            if constexpr (F32) {
                                const uint32_t rest = pack_half(w0 - w.x, w1 - w.y);
                                pb2[b][nt][e] = transpose8x8(rest);
                                const float2 w2 = __half22float2(reinterpret_cast<const __half2 &>(rest));
                                w.x += w2.x;
                                w.y += w2.y;
                            }
                            if constexpr (!ORDINARY) {
                                if (fabsf(offv) > kMostlyOffset) w = make_float2(w0, w1);
                            }
                            // a hidden key adds nothing, even when its scale or offset is no number
                            if (ORDINARY || !(x0 == -INFINITY)) {
                                part_sum[nt][0] = fmaf(w0, inv[b][e], part_sum[nt][0]);
                                part_off[nt][0] = fmaf(w.x, offv, part_off[nt][0]);
                            }
                            if (ORDINARY || !(x1 == -INFINITY)) {
                                part_sum[nt][1] = fmaf(w1, inv[b][e], part_sum[nt][1]);
                                part_off[nt][1] = fmaf(w.y, offv, part_off[nt][1]);
                            }
                        }
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const float both = sum[nt][h] + part_sum[nt][h];
                        lost[nt][h] += part_sum[nt][h] - (both - sum[nt][h]);
                        sum[nt][h] = both;
                        off[nt][h] += part_off[nt][h];
                    }
            };
                if (ordinary) weights(Bool<true>{});
                else weights(Bool<false>{});

                // ---- O^T += V^T P^T, two blocks at a time: lane (g, c) holds the g-th eighth of keys 2c, 2c + 1, 2c + 8, 2c + 9 of each ----
#pragma unroll
                for (int b0 = 0; b0 < NB; b0 += 2) {
                    uint32_t vw[2][4][WV];
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            load_words<WV>(st.v + (16 * (b0 + b) + 2 * c + (e & 1) + 8 * (e >> 1)) * (D / 2) + g * (D / 16), vw[b][e]);
#pragma unroll
                    for (int w = 0; w < WV; ++w) {
                        uint32_t x[2][4];   // block; (keys 2c, 2c + 1 | keys 2c + 8, 2c + 9) x (first | last four dims of the word)
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            x[b][0] = __byte_perm(vw[b][0][w], vw[b][1][w], 0x5410);
                            x[b][1] = __byte_perm(vw[b][0][w], vw[b][1][w], 0x7632);
                            x[b][2] = __byte_perm(vw[b][2][w], vw[b][3][w], 0x5410);
                            x[b][3] = __byte_perm(vw[b][2][w], vw[b][3][w], 0x7632);
                        }
                        float part[4][NT][4];
#pragma unroll
                        for (int b = 0; b < 2; ++b)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t lo = x[b][i >> 1] >> ((i & 1) * 8), hi = x[b][2 + (i >> 1)] >> ((i & 1) * 8);
                                const uint32_t a[4] = {codes<F32, 0>(lo & 0x000f000fu), codes<F32, 1>(lo & 0x00f000f0u),
                                                       codes<F32, 0>(hi & 0x000f000fu), codes<F32, 1>(hi & 0x00f000f0u)};
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    if (b == 0) part[i][nt][0] = part[i][nt][1] = part[i][nt][2] = part[i][nt][3] = 0.f;
                                    mma(part[i][nt], a, pb[b0 + b][nt][0], pb[b0 + b][nt][1]);
                                    if constexpr (F32) mma(part[i][nt], a, pb2[b0 + b][nt][0], pb2[b0 + b][nt][1]);
                                }
                            }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[4 * w + i][nt][e] += part[i][nt][e];
                    }
                }
            }
            __syncwarp();     // the next fetch fills what was read here
            drain = drain == ring + kStages - 1 ? ring : drain + 1;
        }
        async_wait<0>();
        __syncthreads();      // the rings become the place of the results

        // ---- the four warps' results together ----
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                sum[nt][h] += lost[nt][h];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) {
                    sum[nt][h] += __shfl_xor_sync(0xffffffffu, sum[nt][h], d);
                    off[nt][h] += __shfl_xor_sync(0xffffffffu, off[nt][h], d);
                }
                if (g == 0) {
                    float *const st = s_stat + (warp * ROWS + nt * 8 + 2 * c + h) * 4;
                    st[0] = top[nt][h];
                    st[1] = sum[nt][h];
                    st[2] = off[nt][h];
                }
            }
        const bool complete = item_begin >= u_first && item_end <= walk.u_end;
        const long long slot = 2 * (long long)blockIdx.x + (walk.u == u_first ? 0 : 1);
        float *const part = p.partial + slot * slot_floats<D, NT>();
        constexpr int PER = D / 16;      // dims per thread: 16 threads to a row
        const int my_row = tid >> 4, my_dim = (tid & 15) * 4;
        const auto store_row = [&](int row, float m, float l, float b, float (&acc)[PER]) {
            const int abs_row = row0 + row;
            if (abs_row >= total_rows) return;
            const int j = abs_row / p.group, qh = head * p.group + abs_row - j * p.group;
            const float scale = l != 0.f ? 1.f / l : 0.f;
            const long long token = r.first_token + j;
#pragma unroll
            for (int i = 0; i < PER; ++i) acc[i] = l != 0.f ? (acc[i] + b) * scale : 0.f;
#pragma unroll
            for (int i = 0; i < PER / 4; ++i)
                store_out<F32>(p.out, token * p.out_ts + (long long)qh * p.out_hs + my_dim + 64 * i, acc + 4 * i, 4);
            if (p.lse && (tid & 15) == 0)
                p.lse[token * (p.kv_heads * p.group) + qh] = log_sum(m, l);
        };
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            if (nt > 0) __syncthreads();
#pragma unroll
            for (int i = 0; i < KS; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    *reinterpret_cast<float2 *>(s_o + (warp * 8 + 2 * c + h) * LD + g * (D / 8) + 2 * i) =
                        make_float2(o[i][nt][h] * kBack, o[i][nt][2 + h] * (kBack / 16));
            __syncthreads();
            const int row = nt * 8 + my_row;
            float m = kNoMax, f[kWarps], l = 0.f, b = 0.f, acc[PER];
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m = fmaxf(m, s_stat[(w * ROWS + row) * 4]);
#pragma unroll
            for (int i = 0; i < PER; ++i) acc[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) {
                const float *const st = s_stat + (w * ROWS + row) * 4;
                f[w] = ex2(st[0] - m);
                l = fmaf(st[1], f[w], l);
                b = fmaf(st[2], f[w], b);
#pragma unroll
                for (int i = 0; i < PER / 4; ++i) {
                    const float4 x = *reinterpret_cast<const float4 *>(s_o + (w * 8 + my_row) * LD + my_dim + 64 * i);
                    acc[4 * i] = fmaf(x.x, f[w], acc[4 * i]);
                    acc[4 * i + 1] = fmaf(x.y, f[w], acc[4 * i + 1]);
                    acc[4 * i + 2] = fmaf(x.z, f[w], acc[4 * i + 2]);
                    acc[4 * i + 3] = fmaf(x.w, f[w], acc[4 * i + 3]);
                }
            }
            if (complete) {
                store_row(row, m, l, b, acc);
            } else {
                float *const d = part + row * LD;
#pragma unroll
                for (int i = 0; i < PER / 4; ++i)
                    __stcg(reinterpret_cast<float4 *>(d + my_dim + 64 * i), make_float4(acc[4 * i], acc[4 * i + 1], acc[4 * i + 2], acc[4 * i + 3]));
                if ((tid & 15) == 0) __stcg(reinterpret_cast<float4 *>(d + D), make_float4(m, l, b, 0.f));
            }
        }
        if (!complete) {
            // the last of the CTAs that share this item adds up what they left, in the order of the keys
            const int c0 = (int)owner_of(item_begin, ctas, total), c1 = (int)owner_of(item_end - 1, ctas, total);
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                s_last = atomicAdd(p.tickets + c0, 1u) == (uint32_t)(c1 - c0);
                __threadfence();
                if (s_last) p.tickets[c0] = 0;
            }
            __syncthreads();
            if (s_last) {
                // the item opens the share of every CTA but the first, and of that one when the share begins with it
                const int first_slot = mul_div(total, c0, ctas) == item_begin ? 0 : 1;
                constexpr long long APART = 2 * slot_floats<D, NT>();
                const int parts = c1 - c0 + 1;
                const float *const at = p.partial + c0 * APART + my_row * LD, *const at0 = at + first_slot * slot_floats<D, NT>();
                // rows 2 warp, 2 warp + 1 of how many tiles of 8 are there at all
                const int tiles = min(NT, (total_rows - row0 - 2 * warp + 7) >> 3);
                constexpr int FEW = D <= 128 ? 8 : 4;
                // Few parts of several tiles are all loaded at once and added up by every thread for itself, which saves the
                // exchange of weights for each tile.  (16 requests of 5 queries, 25 rows a head, up to 6 parts: the call takes 25.5 us
                // so and 26.8 in the other way; 64 requests of 4 rows a head, mostly 2 or 3 parts: 91.3 us in both.)
                if (NT > 1 && parts <= FEW) {
#pragma unroll 1
                    for (int nt = 0; nt < tiles; ++nt) {
                        float4 st[FEW], v[FEW][PER / 4];
#pragma unroll
                        for (int e = 0; e < FEW; ++e) {
                            const int k = min(e, parts - 1);
                            const float *const d = (k ? at + k * APART : at0) + nt * 8 * LD;
                            st[e] = __ldcg(reinterpret_cast<const float4 *>(d + D));
#pragma unroll
                            for (int i = 0; i < PER / 4; ++i) v[e][i] = __ldcg(reinterpret_cast<const float4 *>(d + my_dim + 64 * i));
                        }
                        float m = kNoMax, l = 0.f, b = 0.f, acc[PER];
#pragma unroll
                        for (int i = 0; i < PER; ++i) acc[i] = 0.f;
#pragma unroll
                        for (int e = 0; e < FEW; ++e) m = fmaxf(m, st[e].x);
#pragma unroll
                        for (int e = 0; e < FEW; ++e) {
                            const float w = e < parts ? ex2(st[e].x - m) : 0.f;   // (the last part stands in past the end)
                            l = fmaf(st[e].y, w, l);
                            b = fmaf(st[e].z, w, b);
#pragma unroll
                            for (int i = 0; i < PER / 4; ++i) {
                                acc[4 * i] = fmaf(v[e][i].x, w, acc[4 * i]);
                                acc[4 * i + 1] = fmaf(v[e][i].y, w, acc[4 * i + 1]);
                                acc[4 * i + 2] = fmaf(v[e][i].z, w, acc[4 * i + 2]);
                                acc[4 * i + 3] = fmaf(v[e][i].w, w, acc[4 * i + 3]);
                            }
                        }
                        store_row(nt * 8 + my_row, m, l, b, acc);
                    }
                } else {
                    // One warp per scheduler is all that works here, so what counts is the number of instructions in a row.  The
                    // 16 threads of a row work out the weights of 32 parts at a time, two each; the parts themselves come through
                    // the rings, each thread fetching what it adds up, FLIGHT groups of 4 on their way.  (All 56 parts of 262,143 keys
                    // took 14,000 cycles with 8 at a time through registers, and take 9,500.)
                    constexpr int GROUP = 4, CHUNK = 32, ROOM = ring_bytes<D, NT>() / (GROUP * kThreads * PER * 4);
                    constexpr int FLIGHT = ROOM < 4 ? ROOM : 4;
                    static_assert(FLIGHT >= 1 && NT * KS * 32 * 8 >= 8 * CHUNK * 4, "");
                    const int t = tid & 15;
                    float *const s_w = reinterpret_cast<float *>(s_q) + my_row * CHUNK;     // the queries have been used
                    const uint32_t ring_first = smem_at(smem) + tid * 16;
                    float4 st[2];
                    const auto look = [&](int nt, int base) {
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const int k = base + t + 16 * i;
                            st[i] = make_float4(kNoMax, 0.f, 0.f, 0.f);
                            if (k < parts && nt < tiles)
                                st[i] = __ldcg(reinterpret_cast<const float4 *>((k ? at + k * APART : at0) + nt * 8 * LD + D));
                        }
                    };
                    look(0, 0);
                    int sent = 0, sent_nt = 0;
                    uint32_t to = ring_first;
                    const float *src = at0 + my_dim, *next = at + my_dim;
                    const auto bring = [&] {
                        if (sent_nt < tiles) {
#pragma unroll
                            for (int e = 0; e < GROUP; ++e) {
#pragma unroll
                                for (int i = 0; i < PER / 4; ++i)
                                    async_copy<16>(to + (e * (PER / 4) + i) * kThreads * 16, src + 64 * i);
                                if (++sent < parts) src = next += APART;    // (the last part again, past the end)
                            }
                            if (sent >= parts) {
                                ++sent_nt;
                                sent = 0;
                                next = at + my_dim + sent_nt * 8 * LD;
                                src = at0 + my_dim + sent_nt * 8 * LD;
                            }
                        }
                        async_commit();
                        to = to == ring_first + (FLIGHT - 1) * GROUP * kThreads * PER * 4 ? ring_first : to + GROUP * kThreads * PER * 4;
                    };
#pragma unroll 1
                    for (int i = 0; i < FLIGHT; ++i) bring();
                    int from = 0;
#pragma unroll 1
                    for (int nt = 0; nt < tiles; ++nt) {
                        const int row = nt * 8 + my_row;
                        float m = kNoMax, l = 0.f, b = 0.f, acc[PER];
#pragma unroll
                        for (int i = 0; i < PER; ++i) acc[i] = 0.f;
#pragma unroll 1
                        for (int base = 0; base < parts; base += CHUNK) {
                            float m2 = fmaxf(m, fmaxf(st[0].x, st[1].x));
#pragma unroll
                            for (int d = 1; d < 16; d <<= 1) m2 = fmaxf(m2, __shfl_xor_sync(0xffffffffu, m2, d));
                            const float w0 = ex2(st[0].x - m2), w1 = ex2(st[1].x - m2), f = ex2(m - m2);
                            float l2 = st[0].y * w0 + st[1].y * w1, b2 = st[0].z * w0 + st[1].z * w1;
#pragma unroll
                            for (int d = 1; d < 16; d <<= 1) {
                                l2 += __shfl_xor_sync(0xffffffffu, l2, d);
                                b2 += __shfl_xor_sync(0xffffffffu, b2, d);
                            }
                            m = m2;
                            l = fmaf(l, f, l2);
                            b = fmaf(b, f, b2);
#pragma unroll
                            for (int i = 0; i < PER; ++i) acc[i] *= f;
                            __syncwarp();
                            s_w[t] = base + t < parts ? w0 : 0.f;
                            s_w[t + 16] = base + t + 16 < parts ? w1 : 0.f;
                            __syncwarp();
                            if (base + CHUNK < parts) look(nt, base + CHUNK);
                            else look(nt + 1, 0);
                            const int here = min(CHUNK, parts - base);
#pragma unroll 1
                            for (int k = 0; k < here; k += GROUP) {
                                async_wait<FLIGHT - 1>();
                                const float4 *const v = reinterpret_cast<const float4 *>(smem) + from * (GROUP * kThreads * PER / 4) + tid;
                                const float4 w4 = *reinterpret_cast<const float4 *>(s_w + k);
                                const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                                for (int e = 0; e < GROUP; ++e)
#pragma unroll
                                    for (int i = 0; i < PER / 4; ++i) {
                                        const float4 x = v[(e * (PER / 4) + i) * kThreads];
                                        acc[4 * i] = fmaf(x.x, w[e], acc[4 * i]);
                                        acc[4 * i + 1] = fmaf(x.y, w[e], acc[4 * i + 1]);
                                        acc[4 * i + 2] = fmaf(x.z, w[e], acc[4 * i + 2]);
                                        acc[4 * i + 3] = fmaf(x.w, w[e], acc[4 * i + 3]);
                                    }
                                bring();
                                from = from == FLIGHT - 1 ? 0 : from + 1;
                            }
                        }
                        store_row(row, m, l, b, acc);
                    }
                    async_wait<0>();
                }
            }
        }
        __syncthreads();
        walk.u += steps;
    }
}

// One compiled variant: its kernel, shared memory and tile height.
struct Variant {
    const void *kernel;
    int smem, rows, slot, unit;
};

template <int D, int NT, bool F32>
Variant variant() { return {reinterpret_cast<const void *>(&kv_attend_kernel<D, NT, F32>), attend_smem<D, NT, F32>(), 8 * NT, slot_floats<D, NT>(),
            unit_keys<D, NT>()}; }

// Rows of queries that share a key head decide the tile: as few columns of 8 as hold them, so that no product is wasted on
// empty ones, up to what the registers of a thread hold (head_dim / 16 x 4 accumulators per 8 rows); more rows than the
// largest tile are walked tile by tile.
__host__ constexpr int tile_columns(int head_dim, long long rows) {
    return rows <= 8 || head_dim > 128 ? 1 : rows <= 16 || head_dim > 64 ? 2 : 4;
}

template <bool F32>
Variant pick(int head_dim, int nt) {
    switch (head_dim) {
        case 64: return nt == 1 ? variant<64, 1, F32>() : nt == 2 ? variant<64, 2, F32>() : variant<64, 4, F32>();
        case 128: return nt == 1 ? variant<128, 1, F32>() : variant<128, 2, F32>();
        case 192: return variant<192, 1, F32>();
        default: return variant<256, 1, F32>();
    }
}

}  // namespace

fi_status_t prepare_attend(fi_kv *kv) {
    size_t floats = 0;
    int most_ctas = 0;
    for (int f32 = 0; f32 < 2; ++f32)
        for (int i = 0; i < 3; ++i) {
            const int nt = 1 << i;
            if (nt > tile_columns(kv->cfg.head_dim, 1 << 30)) continue;
            const Variant v = f32 ? pick<true>(kv->cfg.head_dim, nt) : pick<false>(kv->cfg.head_dim, nt);
            int ctas = 0;
            cudaError_t e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, v.smem);
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&ctas, v.kernel, kThreads, v.smem);
            if (e == cudaSuccess && ctas < 1) e = cudaErrorInvalidConfiguration;
            if (e != cudaSuccess) return cuda_fail(e, "fi_kv_create: attention kernels");
            kv->attend_ctas[f32][i] = ctas * kv->sm_count;
            if (ctas * kv->sm_count > most_ctas) most_ctas = ctas * kv->sm_count;
            const size_t need = (size_t)ctas * kv->sm_count * 2 * v.slot;
            if (need > floats) floats = need;
        }
    most_ctas = (most_ctas + 3) / 4 * 4;   // the partial results behind the tickets stay 16-byte aligned
    kv->tickets = most_ctas;
    const fi_status_t st = prepare_attend_prompt(kv);
    if (st != FI_OK) return st;
    cudaError_t e = cudaMalloc(reinterpret_cast<void **>(&kv->scratch), floats * 4 + (size_t)most_ctas * 4);
    if (e == cudaSuccess) e = cudaMemset(kv->scratch, 0, (size_t)most_ctas * 4);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_kv_create: attention scratch");
}

}  // namespace fi

using namespace fi;

extern "C" fi_status_t fi_kv_attend(fi_kv_t *kv, const fi_kv_attend_t *a, void *cuda_stream) {
    if (!kv || !a) {
        set_error("fi_kv_attend: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (a->dtype != FI_F32 && a->dtype != FI_BF16) {
        set_error("fi_kv_attend: dtype must be FI_F32 or FI_BF16");
        return FI_ERR_INVALID_ARG;
    }
    const long long most_keys = (long long)a->max_blocks << kv->page_shift;
    if (a->batch_max < 0 || a->max_tokens < 0 || a->rows < 0 || a->max_blocks < 0 || a->window < 0 || a->max_query < 0 ||
        a->table_ld < a->max_blocks || most_keys > 2147483647ll - 1024 || (!a->row_idx && a->batch_max > a->rows) ||
        (!a->cu_tokens && a->batch_max > a->max_tokens) ||
        (long long)a->max_tokens * (kv->cfg.q_heads / kv->cfg.kv_heads) > 2147483647ll - 1024) {
        set_error("fi_kv_attend: negative size, table_ld below max_blocks, more keys or query rows than 2^31 - 1,024, or fewer rows "
                  "or tokens than requests");
        return FI_ERR_INVALID_ARG;
    }
    if (a->batch_max == 0 || a->max_tokens == 0) return FI_OK;
    if (!a->q || !a->out || !a->lens || (a->max_blocks > 0 && !a->block_table)) {
        set_error("fi_kv_attend: null pointer (only lse, row_idx, batch_count, cu_tokens and granted may be)");
        return FI_ERR_INVALID_ARG;
    }
    const int unit = a->dtype == FI_BF16 ? 8 : 4;
    const auto bad = [&](int64_t stride, int count) { return count > 1 && (stride < 0 || stride % unit != 0); };
    if ((reinterpret_cast<uintptr_t>(a->q) & 15) || (reinterpret_cast<uintptr_t>(a->out) & 15) || bad(a->q_token_stride, a->max_tokens) ||
        bad(a->out_token_stride, a->max_tokens) || bad(a->q_head_stride, kv->cfg.q_heads) || bad(a->out_head_stride, kv->cfg.q_heads)) {
        set_error("fi_kv_attend: heads must start on 16-byte boundaries, strides must not be negative");
        return FI_ERR_INVALID_ARG;
    }
    if (!(a->scale > -3e38f && a->scale < 3e38f)) {
        set_error("fi_kv_attend: scale must be finite");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(kv->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_kv_attend");
    const fi_kv_config_t &c = kv->cfg;
    AttendParams p;
    p.q = a->q;
    p.out = a->out;
    p.lse = a->lse;
    p.lens = a->lens;
    p.block_table = a->block_table;
    p.row_idx = a->row_idx;
    p.batch_count = a->batch_count;
    p.cu_tokens = a->cu_tokens;
    p.granted = a->granted;
    p.k_codes = static_cast<const unsigned char *>(c.k_codes);
    p.v_codes = static_cast<const unsigned char *>(c.v_codes);
    p.k_meta = static_cast<const uint32_t *>(c.k_meta);
    p.v_meta = static_cast<const uint32_t *>(c.v_meta);
    p.tickets = reinterpret_cast<uint32_t *>(kv->scratch);
    p.partial = reinterpret_cast<float *>(kv->scratch + (size_t)kv->tickets * 4);
    p.status = kv->status_dev;
    p.q_ts = a->q_token_stride;
    p.q_hs = a->q_head_stride;
    p.out_ts = a->out_token_stride;
    p.out_hs = a->out_head_stride;
    p.ps = (uint32_t)(c.page_stride / 16);
    p.hs = c.head_stride;
    p.ts = (uint32_t)(c.token_stride / 16);
    p.mps = (uint32_t)c.meta_page_stride;
    p.mhs = c.meta_head_stride;
    p.mts = (uint32_t)c.meta_token_stride;
    p.table_ld = a->table_ld;
    p.rows = a->rows;
    p.max_blocks = a->max_blocks;
    p.batch_max = a->batch_max;
    p.max_tokens = a->max_tokens;
    p.window = a->window < most_keys ? a->window : 0;
    p.num_pages = c.num_pages;
    p.page_shift = kv->page_shift;
    p.kv_heads = c.kv_heads;
    p.group = c.q_heads / c.kv_heads;
    p.scale_log2 = a->scale * kLog2e;
    p.wait_limit = kv->wait_limit;
    const bool f32 = a->dtype == FI_F32;
    const long long per_request = a->cu_tokens ? (a->max_query < 1 ? 1 : a->max_query) : 1;
    const long long rows = per_request * p.group;
    if (prompt_kernel_serves(kv, p, a->dtype, per_request)) return launch_attend_prompt(kv, p, rows, static_cast<cudaStream_t>(cuda_stream));
    const int nt = tile_columns(c.head_dim, rows);
    const Variant v = f32 ? pick<true>(c.head_dim, nt) : pick<false>(c.head_dim, nt);
    long long grid = kv->attend_ctas[f32 ? 1 : 0][nt >> 1];
    const long long units = (most_keys + v.unit - 1) / v.unit;
    const double most = (double)a->batch_max * c.kv_heads * (double)((rows + v.rows - 1) / v.rows) * (double)(units < 1 ? 1 : units);
    if (most < (double)grid) grid = (long long)most;
    void *args[] = {&p};
    const cudaError_t e = cudaLaunchKernel(v.kernel, dim3((unsigned)grid), dim3(kThreads), args, (size_t)v.smem,
                                           static_cast<cudaStream_t>(cuda_stream));
    count_launch();
    if (e != cudaSuccess) return cuda_fail(e, "fi_kv_attend");
    return check_launch("fi_kv_attend");
}

// Attention over the 4-bit store for many queries per request (prompts): tensor-bound, so it runs on tcgen05.
//
// A CTA takes 256 query rows of one request and key head (row = query x heads of the group), as two halves of 128, and walks
// the keys in tiles of 128.  Four warps unpack the keys of a tile to halves in shared memory and four its values; four warps
// per half, a thread per row, turn S into the weights P; and one thread of a warp of its own issues the products
//   S = Q K^T  (128 x 128, fp32 in TMEM)      O += P V  (128 x head_dim, fp32 in TMEM)
// for each half.  The halves take turns: while one forms weights the other's products run.  All meet at mbarriers.
//   Two chunks of 1,024 queries of 32 heads behind 8,192 keys take 382 us, 638 TFLOP/s, without the logarithm.  With one half only and everything
// unrolled it was 680 us, a third of the warps' time spent waiting for instructions; so every role's loop is short, and S is
// read from TMEM twice, 32 columns at a time, rather than held.  Products issued by a thread that forms weights hold it up by
// 2,000 cycles per tile.  Waiting for a tile's values, rather than only for their power, before forming its weights cost
// another 170 us.  What bounds it now: the exponentials (16 per cycle and SM: 2,048 cycles of about 5,700 per 256 x 128 tile),
// the operands in shared memory (about 3,000 cycles of reads and writes), and 256 such items on 148 SMs.
//
// Unlike in the kernel for few rows, codes are brought to their values here (128 rows share the work): k = n s + m as a half,
// rounded once (2^-11), after a power of two common to the tile has put the largest value of its 128 keys at 2^14 .. 2^15,
// so no size of keys runs over (they may reach the end of bf16); the power goes into the factor of the scores.  Values likewise, and their power F into the
// exponent: P = 2^(x + F - M) with M = max(x + F) - 7 as it was when one last went over M + 15 (so halves start at 2^7 and lose what is
// below 2^-32 of the largest, not 2^-25), and the sum takes P 2^-F.  A key whose scale or offset (or whose value's) is no
// number becomes NaN in its scores and zero in V: the rows that see it get NaN, the others lose nothing.
//
// Keys rounded to halves put a score off by up to 2^-11 of its parts.  The result, whose weights are halves anyway, may have that; the
// softmax sum's logarithm is a float32 number, which was off by up to 8e-4 where few keys count.  So when it is wanted, the
// codes go into the product as they are, less 7.5 (exact), and the scores take each key's scale and offset behind it:
//   y = (S c) s + (m + 7.5 s) (scale log2(e) sum(q)) + F
// The case above takes 467 us then: a thread loads 64 times 16 bytes of factors per tile, two scores take three more packed operations,
// and y is written back to TMEM.  (When it took 471: one pass over S instead of two, with the maximum checked afterwards, 489, as it has to
// wait for the product before; keys as two halves, in two products, 535.)
#include "fi_attend.cuh"

namespace fi {
namespace {

constexpr int kTile = 128;                 // keys of a tile, query rows of a half
constexpr int kRows = 2 * kTile;           // query rows of a CTA
constexpr int kSoftmaxWarps = 8;           // warp w reads TMEM lanes 32 (w mod 4) .. of half w / 4
constexpr int kUnpackWarps = 4;            // for the keys, and as many for the values
constexpr int kProductWarp = kSoftmaxWarps + 2 * kUnpackWarps;
constexpr int kPromptThreads = (kProductWarp + 1) * 32;
constexpr long long kShortLimit = 1 << 20;       // SM cycles (about 0.5 ms): limits below it are a test's
constexpr long long kDrainLimit = 200000000ll;   // (about 0.1 s)
constexpr int kTmemCols = 512;             // S of both halves, O of both

struct PromptCtl {
    uint64_t k_full, k_empty, v_full, v_empty, q_full;
    uint64_t k_info[4], v_info[4];         // a tile's powers (EXACT: scales and offsets): known before its keys and values have a place
    uint64_t s_full[2], p_full[2], pv_done[2];                      // of the halves
    uint64_t drained;                      // every product that was issued is over
    float k_power[4], v_power[4];          // 2^E of a tile's keys; F of its values
    uint32_t hidden[4][kUnpackWarps];      // keys of a tile whose page is not in the pool, a bit each
    uint32_t red[2][2][kUnpackWarps];      // largest key and value of a tile, by warp
    alignas(16) float k_scale[4][kTile], k_offset[4][kTile];   // EXACT: of a tile's keys, offsets moved by 7.5 scales
    alignas(16) uint32_t meta[kTile];      // scale and offset of a tile's values, as halves
    uint32_t tmem;
    volatile int gave_up;
};

template <int D>
struct PromptSmem {
    static constexpr int kQ = kTile * D * 2, kP = kTile * kTile * 2;   // of a half
    static constexpr int q = 0, k = 2 * kQ, v = k + kTile * D * 2, p = v + kTile * D * 2, ctl = p + 2 * kP;
    static constexpr int bytes = 1024 /* alignment */ + ctl + (int)sizeof(PromptCtl);
};

__device__ __forceinline__ void bar_init(uint64_t *bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(bar)), "r"(count) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint64_t *bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_at(bar)) : "memory");
}

__device__ __forceinline__ bool bar_try(uint64_t *bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(ok)
        : "r"(smem_at(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}

// Bounded wait.  When it gives up, every later wait of the CTA does so at once: no more products are issued, the kernel runs to its
// end with whatever is in its buffers, and the status word says that the results are not valid.  What a wait does when it is not over
// at once is one copy of code: in line it took the registers of the loops (399 us, not 385).
__device__ __noinline__ bool bar_wait_long(uint64_t *bar, uint32_t parity, PromptCtl *ctl, int32_t *status, long long limit) {
    const long long t0 = clock64();
    for (uint32_t spins = 1;; ++spins) {
        if (bar_try(bar, parity)) return true;
        if ((spins & 255) == 0) {
            if (ctl->gave_up) return false;
            if (clock64() - t0 > limit) {
                ctl->gave_up = 1;
                atomicOr(status, 4);
                return false;
            }
        }
    }
}

__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, PromptCtl *ctl, const AttendParams &p) {
    return bar_try(bar, parity) || bar_wait_long(bar, parity, ctl, p.status, p.wait_limit);
}

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(bar)) : "memory");
}

// operand in shared memory: rows of 128 bytes, 128-byte swizzle, groups of eight rows 1,024 bytes apart
__device__ __forceinline__ uint64_t operand(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// half x half -> fp32, M = 128
__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, int n, uint32_t accumulate) {
    const uint32_t idesc = (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n"
        "}\n" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}

// 16 columns of the thread's TMEM lane
__device__ __forceinline__ void tmem_load(uint32_t addr, uint32_t *v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]),
          "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15])
        : "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
        "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]),
        "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15])
        : "memory");
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// the 16 registers may only be used behind the wait above it
__device__ __forceinline__ void settle(uint32_t *v) {
    asm volatile("" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]),
                      "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])::"memory");
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

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(h);
}

// value of two codes: (n 2^-24) is made n exactly, then n scale + offset rounds once
template <int ROW>
__device__ __forceinline__ uint32_t value2(uint32_t codes, __half2 scale, __half2 offset) {
    // 1024 + n, or 1024 + 16 n
    const uint32_t big = codes | 0x64006400u;
    const __half2 n = ROW ? __hfma2(reinterpret_cast<const __half2 &>(big), __float2half2_rn(0.0625f), __float2half2_rn(-64.f))
                          : __hadd2(reinterpret_cast<const __half2 &>(big), __float2half2_rn(-1024.f));
    const __half2 v = __hfma2(n, scale, offset);
    return reinterpret_cast<const uint32_t &>(v);
}

// two codes n as (n - 7.5) 2^-9, exactly
constexpr float kCode = 0x1p-9f;
template <int ROW>
__device__ __forceinline__ uint32_t centred2(uint32_t codes) {
    const __half2 v = __hfma2(reinterpret_cast<const __half2 &>(codes), __float2half2_rn(kCode * (ROW ? 0x1p20f : 0x1p24f)),
                              __float2half2_rn(-7.5f * kCode));
    return reinterpret_cast<const uint32_t &>(v);
}

constexpr uint32_t kNone = 0xffffffffu;

// Scale and offset of a key and of its value; bad: one of the four is no finite number (y - y is not 0 then).
struct KeyMeta {
    uint32_t k, v;
    bool bad;
    __device__ __forceinline__ KeyMeta(uint32_t k_, uint32_t v_) : k(k_), v(v_) {
        const float ks = meta_scale(k), ko = meta_offset(k), vs = meta_scale(v), vo = meta_offset(v);
        bad = (ks - ks) + (ko - ko) + (vs - vs) + (vo - vo) != 0.f;
    }
};

// E of a tile, which puts the largest of its 128 values (one per thread of four warps) at 2^14 .. 2^15 when it is taken out; `red` is
// used again two tiles later.
__device__ __forceinline__ int tile_power(float most, uint32_t *red, int uw, int lane, int barrier) {
    const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(most));
    if (lane == 0) red[uw] = top;
    asm volatile("bar.sync %0, 128;" ::"r"(barrier) : "memory");
    uint32_t all = 0;
#pragma unroll
    for (int i = 0; i < kUnpackWarps; ++i) all = max(all, *reinterpret_cast<volatile uint32_t *>(red + i));
    const int e = all ? (int)(all >> 23) - 141 : 0;
    return e < -100 ? -100 : e;            // (114 at most)
}

// One tile of query rows as every role walks them: request by request, heads, row tiles from the last (most keys) to the first.
struct Item {
    int row, len, queries, first_token, head, row0, rows;   // rows: of the request and head
    int first_key, tiles[2];                                // tiles of 128 keys from first_key on that a half sees; the second sees more
};

struct ItemWalk {
    long long item, start;
    int request, n;
};

__device__ __forceinline__ bool next_item(const AttendParams &p, ItemWalk &w, Item &x) {
    for (; w.request < w.n; ++w.request) {
        const int i = w.request;
        x.first_token = p.cu_tokens ? p.cu_tokens[i] : i;
        x.queries = p.cu_tokens ? p.cu_tokens[i + 1] - x.first_token : 1;
        x.row = p.row_idx ? p.row_idx[i] : i;
        if (x.row < 0 || x.row >= p.rows || x.first_token < 0 || x.queries < 0 || x.queries > p.max_tokens - x.first_token) x.queries = 0;
        x.rows = x.queries * p.group;
        const int row_tiles = (int)(((long long)x.rows + kRows - 1) / kRows);
        const long long here = (long long)row_tiles * p.kv_heads;
        if (w.item >= w.start + here) {
            w.start += here;
            continue;
        }
        const int in_request = (int)(w.item - w.start);
        x.head = in_request / row_tiles;
        x.row0 = (row_tiles - 1 - (in_request - x.head * row_tiles)) * kRows;
        const long long most = (long long)p.max_blocks << p.page_shift;
        x.len = p.lens[x.row];
        if (x.len > most) x.len = (int)most;
        if (x.len < 0 || (p.granted && p.granted[i] < x.queries)) x.len = 0;     // (a refused request sees nothing)
        const int before = x.len - x.queries, first = before + x.row0 / p.group;
        x.first_key = p.window > 0 ? max(max(first, 0) - p.window + 1, 0) / kTile * kTile : 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row0 = x.row0 + h * kTile, last = before + (min(row0 + kTile, x.rows) - 1) / p.group;
            x.tiles[h] = row0 >= x.rows || last < 0 ? 0 : (last + 1 - x.first_key + kTile - 1) / kTile;
        }
        w.item += gridDim.x;
        return true;
    }
    return false;
}

// tiles that are unpacked for an item
__device__ __forceinline__ int tiles_of(const Item &x) { return max(x.tiles[0], x.tiles[1]); }

template <int D, bool EXACT>
__global__ void __launch_bounds__(kPromptThreads, 1) kv_attend_prompt_kernel(const __grid_constant__ AttendParams p) {
    using S = PromptSmem<D>;
    constexpr int PANEL = kTile * 128;     // 128 rows of 128 bytes
    extern __shared__ unsigned char raw_smem[];
    unsigned char *const smem = raw_smem + ((1024 - (smem_at(raw_smem) & 1023)) & 1023);
    PromptCtl *const ctl = reinterpret_cast<PromptCtl *>(smem + S::ctl);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        bar_init(&ctl->k_full, kUnpackWarps * 32);
        bar_init(&ctl->k_empty, 1);
        bar_init(&ctl->v_full, kUnpackWarps * 32);
        bar_init(&ctl->v_empty, 1);
        for (int i = 0; i < 4; ++i) {
            bar_init(&ctl->k_info[i], kUnpackWarps);
            bar_init(&ctl->v_info[i], 1);
        }
        bar_init(&ctl->q_full, kSoftmaxWarps * 32);
        bar_init(&ctl->drained, 1);
        for (int h = 0; h < 2; ++h) {
            bar_init(&ctl->s_full[h], 1);
            bar_init(&ctl->p_full[h], kSoftmaxWarps * 16);
            bar_init(&ctl->pv_done[h], 1);
        }
        ctl->gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&ctl->tmem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = ctl->tmem;
    ItemWalk walk = {(long long)blockIdx.x, 0, 0, p.batch_max};
    if (p.batch_count) walk.n = min(max(*p.batch_count, 0), p.batch_max);
    Item x;
    uint32_t tiles_before = 0;             // of the items before: parities follow from it

    // so that a wait runs out for certain: nothing completes this barrier yet, and the products wait for this thread
    if (p.wait_limit < kShortLimit && tid == 0) bar_wait(&ctl->drained, 0, ctl, p);

    if (warp < kSoftmaxWarps) {
        // ---- a thread per query row ----
        const int my_row = tid & (kTile - 1), half = tid >> 7;
        const uint32_t lanes_at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes_at + half * kTile, o_at = lanes_at + 2 * kTile + half * kTile;
        uint32_t steps = 0;                                   // tiles of this half so far
        while (next_item(p, walk, x)) {
            const int all = tiles_of(x), mine = x.tiles[half], row0 = x.row0 + half * kTile;
            const int row = row0 + my_row;
            const bool real = row < x.rows;
            const int shown = real ? row : x.rows - 1;        // rows past the last see what it sees; they are never stored
            const int j = shown / p.group, qh = x.head * p.group + shown - j * p.group;
            const int pos = x.len - x.queries + j;
            const int high = pos + 1, low = p.window > 0 ? max(pos, 0) - p.window + 1 : 0;
            const int first = x.len - x.queries + row0 / p.group, last = x.len - x.queries + (min(row0 + kTile, x.rows) - 1) / p.group;
            const int all_high = first + 1, all_low = p.window > 0 ? max(last, 0) - p.window + 1 : 0;
            float c = 0.f, q_sum = 0.f;                       // what S is worth; EXACT: the row's scale sum(q)
            if (all > 0) {
                // ---- the row's query as halves, its largest value at 2^14 .. 2^15 (exact for bf16), in the order of the codes ----
                const uint4 *q = reinterpret_cast<const uint4 *>(static_cast<const __nv_bfloat16 *>(p.q) +
                                                                 (long long)(x.first_token + j) * p.q_ts + (long long)qh * p.q_hs);
                float top = 0.f;
                const auto words = [&](int i, float (&v)[8]) {
                    const uint4 w = real ? __ldg(q + i) : make_uint4(0, 0, 0, 0);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[2 * e] = __uint_as_float(u[e] << 16);
                        v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u);
                    }
                };
#pragma unroll 4
                for (int i = 0; i < D / 8; ++i) {
                    float v[8];
                    words(i, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(v[e]));
                }
                int up = 0;
                if (top > 0.f && top < INFINITY) {
                    up = 141 - (int)(__float_as_uint(top) >> 23);
                    up = up > 110 ? 110 : up;            // (-113 at least)
                }
                float f = __uint_as_float((uint32_t)(127 + up) << 23);
                const float back = p.scale_log2 * __uint_as_float((uint32_t)(127 - up) << 23);
                if constexpr (!EXACT) {
                    // the factor of the scores is kept positive: its sign goes into the query (and a factor of zero makes it zero)
                    c = fabsf(back);
                    if (back < 0.f) f = -f;
                    if (!(c > 0.f)) {
                        f = 0.f;
                        c = 1.f;
                    }
                }
                float total[EXACT ? 8 : 1] = {};
#pragma unroll 4
                for (int i = 0; i < D / 8; ++i) {
                    float v[8];
                    words(i, v);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        v[e] *= f;
                        if constexpr (EXACT) total[e] += v[e];
                    }
                    *reinterpret_cast<uint4 *>(smem + S::q + half * S::kQ + (i >> 3) * PANEL + my_row * 128 + (((i & 7) ^ (my_row & 7)) << 4)) =
                        make_uint4(half2_bits(v[0], v[4]), half2_bits(v[1], v[5]), half2_bits(v[2], v[6]), half2_bits(v[3], v[7]));
                }
                if constexpr (EXACT) {
                    c = back / kCode;
                    q_sum = back * (((total[0] + total[4]) + (total[1] + total[5])) + ((total[2] + total[6]) + (total[3] + total[7])));
                }
                fence_async();
                bar_arrive(&ctl->q_full);
            }
            float top = kNoMax, sum = 0.f;
            for (int t = 0; t < all; ++t) {
                const uint32_t n = tiles_before + t;
                bar_wait(&ctl->k_info[n & 3], (n >> 2) & 1, ctl, p);   // the tile's powers
                bar_wait(&ctl->v_info[n & 3], (n >> 2) & 1, ctl, p);
                if (t >= mine) {
                    // A tile for the other half.  It is counted through here too, and not before its values are there: two phases of
                    // p_full completed ahead of the thread that waits for them would look like none.
                    bar_wait(&ctl->v_full, n & 1, ctl, p);
                    bar_arrive(&ctl->p_full[half]);
                    continue;
                }
                const int key0 = x.first_key + t * kTile;
                // (never 0: a hidden score is -infinity and has to stay so)
                const float ck = EXACT ? 1.f : fminf(fmaxf(c * ctl->k_power[n & 3], FLT_MIN), FLT_MAX), fv = ctl->v_power[n & 3];
                const uint32_t lost = ctl->hidden[n & 3][0] | ctl->hidden[n & 3][1] | ctl->hidden[n & 3][2] | ctl->hidden[n & 3][3];
                const bool edge = key0 + kTile > all_high || key0 < all_low || lost != 0;
                bar_wait(&ctl->s_full[half], steps & 1, ctl, p);
                tc_after();
                // 32 scores from column c0 on, hidden ones at -infinity
                uint32_t s[32];
                const auto read = [&](int c0) {
                    tmem_load(s_at + c0, s);
                    tmem_load(s_at + c0 + 16, s + 16);
                    tmem_load_wait();
                    settle(s);
                    settle(s + 16);
                };
                const auto hide = [&](int c0) {
                    if (edge) {
                        const int hi = high - key0 - c0, lo = low - key0 - c0;
                        const uint32_t gone = ctl->hidden[n & 3][c0 >> 5];
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (i >= hi || i < lo || ((gone >> i) & 1)) s[i] = 0xff800000u;
                    }
                };
                float most = -INFINITY;
#pragma unroll 1
                for (int c0 = 0; c0 < kTile; c0 += 32) {
                    read(c0);
                    if constexpr (EXACT) {
                        const uint64_t c2 = pair(c, c), sq2 = pair(q_sum, q_sum), fv2 = pair(fv, fv);
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            const float4 ks = *reinterpret_cast<const float4 *>(&ctl->k_scale[n & 3][c0 + i]),
                                         ko = *reinterpret_cast<const float4 *>(&ctl->k_offset[n & 3][c0 + i]);
                            float y[4];
                            unpair(fma2(mul2(pair(__uint_as_float(s[i]), __uint_as_float(s[i + 1])), c2), pair(ks.x, ks.y),
                                        fma2(pair(ko.x, ko.y), sq2, fv2)), y[0], y[1]);
                            unpair(fma2(mul2(pair(__uint_as_float(s[i + 2]), __uint_as_float(s[i + 3])), c2), pair(ks.z, ks.w),
                                        fma2(pair(ko.z, ko.w), sq2, fv2)), y[2], y[3]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[i + e] = __float_as_uint(y[e]);
                        }
                    }
                    hide(c0);
                    if constexpr (EXACT) {      // y takes the place of S
                        tmem_store(s_at + c0, s);
                        tmem_store(s_at + c0 + 16, s + 16);
                    }
#pragma unroll
                    for (int i = 0; i < 32; i += 2) most = fmaxf(fmaxf(most, __uint_as_float(s[i])), __uint_as_float(s[i + 1]));
                }
                if constexpr (EXACT) tmem_store_wait();
                else most = fmaf(most, ck, fv);
                // the products have read the weights before and added them up
                if (t > 0) bar_wait(&ctl->pv_done[half], (steps - 1) & 1, ctl, p);
                if (__any_sync(0xffffffffu, most - top > kMost)) {
                    const float m = fmaxf(most - kStart, top), shrink = ex2(top - m);
                    top = m;
                    sum *= shrink;
                    if (t > 0) {
                        tc_after();
#pragma unroll 1
                        for (int i = 0; i < D / 16; ++i) {
                            tmem_load(o_at + 16 * i, s);
                            tmem_load_wait();
                            settle(s);
#pragma unroll
                            for (int e = 0; e < 16; ++e) s[e] = __float_as_uint(__uint_as_float(s[e]) * shrink);
                            tmem_store(o_at + 16 * i, s);
                        }
                        tmem_store_wait();
                    }
                }
                const uint64_t ck2 = pair(ck, ck), fv2 = pair(fv, fv), less2 = pair(-top, -top), shift2 = pair(fv - top, fv - top);
                uint64_t part[2] = {0, 0};
                // Beside large scores y is rounded before the maximum is taken off it, as it was for the maximum: then no weight is above
                // 2^15 (in one step it might be, by the roundings of y).  ROUNDED costs one more operation for two scores.
                const auto weights = [&](auto rounded_) {
                    constexpr bool ROUNDED = decltype(rounded_)::value;
#pragma unroll 1
                    for (int c0 = 0; c0 < kTile; c0 += 32) {
                        read(c0);
                        if constexpr (!EXACT) hide(c0);
                        unsigned char *const to = smem + S::p + half * S::kP + (c0 >> 6) * PANEL + my_row * 128;
#pragma unroll
                        for (int i = 0; i < 32; i += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                float w0, w1;
                                const uint64_t s2 = pair(__uint_as_float(s[i + 2 * e]), __uint_as_float(s[i + 2 * e + 1]));
                                unpair(EXACT ? add2(s2, less2) : ROUNDED ? add2(fma2(s2, ck2, fv2), less2) : fma2(s2, ck2, shift2), w0, w1);
                                w0 = ex2(w0);
                                w1 = ex2(w1);
                                part[e & 1] = add2(part[e & 1], pair(w0, w1));
                                w[e] = half2_bits(w0, w1);
                            }
                            *reinterpret_cast<uint4 *>(to + ((((c0 & 32) + i) >> 3 ^ (my_row & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
                        }
                    }
                };
                if (!EXACT && __any_sync(0xffffffffu, fabsf(top) > 0x1p20f && top != kNoMax)) weights(Bool<true>{});
                else weights(Bool<false>{});
                fence_async();
                tc_before();
                bar_arrive(&ctl->p_full[half]);
                ++steps;
                float a0, a1;
                unpair(add2(part[0], part[1]), a0, a1);
                sum = fmaf(a0 + a1, ex2(-fv), sum);
            }
            tiles_before += all;
            if (mine > 0) {
                bar_wait(&ctl->pv_done[half], (steps - 1) & 1, ctl, p);
                tc_after();
            }
            const float scale = sum != 0.f ? 1.f / sum : 0.f;
            __nv_bfloat16 *const out = static_cast<__nv_bfloat16 *>(p.out) + (long long)(x.first_token + j) * p.out_ts + (long long)qh * p.out_hs;
#pragma unroll 1
            for (int i = 0; i < D / 16; ++i) {
                uint32_t o[16];
                if (mine > 0) {
                    tmem_load(o_at + 16 * i, o);
                    tmem_load_wait();
                    settle(o);
                }
                uint32_t w[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v0 = sum != 0.f ? __uint_as_float(o[2 * e]) * scale : 0.f, v1 = sum != 0.f ? __uint_as_float(o[2 * e + 1]) * scale : 0.f;
                    const __nv_bfloat162 h = __floats2bfloat162_rn(v0, v1);
                    w[e] = reinterpret_cast<const uint32_t &>(h);
                }
                if (real) {
                    reinterpret_cast<uint4 *>(out)[2 * i] = make_uint4(w[0], w[1], w[2], w[3]);
                    reinterpret_cast<uint4 *>(out)[2 * i + 1] = make_uint4(w[4], w[5], w[6], w[7]);
                }
            }
            if (real && p.lse)
                p.lse[(long long)(x.first_token + j) * (p.kv_heads * p.group) + qh] = log_sum(top, sum);
            tc_before();
        }
    } else if (warp < kSoftmaxWarps + kUnpackWarps) {
        // ---- keys: a thread per key; pages are looked up two tiles ahead, codes fetched one tile ahead ----
        const int u = tid - kSoftmaxWarps * 32, uw = u >> 5;
        const int mask = (1 << p.page_shift) - 1;
        while (next_item(p, walk, x)) {
            const int all = tiles_of(x);
            const int32_t *const table = p.block_table + (long long)x.row * p.table_ld;
            const unsigned char *const k_head = p.k_codes + x.head * p.hs;
            const uint32_t *const km_head = p.k_meta + x.head * p.mhs, *const vm_head = p.v_meta + x.head * p.mhs;
            uint32_t page = kNone, next[D / 8], next_km = 0, next_vm = 0;
            bool next_lost = false;
            const auto look_up = [&](int t) {
                const int key = x.first_key + t * kTile + u;
                page = t < all && key < x.len ? min((uint32_t)__ldg(table + (key >> p.page_shift)), kNone - 1) : kNone;
            };
            const auto fetch = [&](int t) {
                const int key = x.first_key + t * kTile + u;
                const bool there = page < (uint32_t)p.num_pages;
                next_lost = !there && page != kNone;
                next_km = next_vm = 0;
                const uint32_t place = key & mask, off = page * p.ps + place * p.ts, moff = page * p.mps + place * p.mts;
                const uint4 *from = reinterpret_cast<const uint4 *>(k_head + off * 16ull);
#pragma unroll
                for (int i = 0; i < D / 32; ++i) {
                    const uint4 a = there ? __ldg(from + i) : make_uint4(0, 0, 0, 0);
                    next[4 * i] = a.x; next[4 * i + 1] = a.y; next[4 * i + 2] = a.z; next[4 * i + 3] = a.w;
                }
                if (there) {
                    next_km = __ldg(km_head + moff);
                    next_vm = __ldg(vm_head + moff);
                }
            };
            look_up(0);
            fetch(0);
            look_up(1);
            for (int t = 0; t < all; ++t) {
                const uint32_t n = tiles_before + t;
                const KeyMeta meta(next_km, next_vm);
                const bool lost = next_lost;
                if (lost) atomicOr(p.status, 2);
                const float scale = meta.bad ? 0.f : meta_scale(meta.k), offset = meta.bad ? __uint_as_float(0x7fc00000u) : meta_offset(meta.k);
                // (S of tile n - 2 is there for both halves, so both have formed the weights of n - 3: the place of n - 4 is free)
                __half2 s2, o2;
                if constexpr (EXACT) {
                    ctl->k_scale[n & 3][u] = scale;
                    ctl->k_offset[n & 3][u] = fmaf(7.5f, scale, offset);
                } else {
                    const int e = tile_power(meta.bad ? 0.f : fmaxf(fabsf(offset), fabsf(fmaf(15.f, scale, offset))), ctl->red[n & 1][0], uw, lane, 1);
                    const float f = __uint_as_float((uint32_t)(127 - e) << 23);
                    s2 = __float2half2_rn(scale * f);
                    o2 = __float2half2_rn(offset * f);
                    if (u == 0) ctl->k_power[n & 3] = __uint_as_float((uint32_t)(127 + e) << 23);
                }
                const uint32_t gone = __ballot_sync(0xffffffffu, lost);
                if (lane == 0) ctl->hidden[n & 3][uw] = gone;
                __syncwarp();
                if (lane == 0) bar_arrive(&ctl->k_info[n & 3]);
                bar_wait(&ctl->k_empty, (n & 1) ^ 1, ctl, p);
                unsigned char *const to = smem + S::k + u * 128;
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    const uint32_t w = next[i], w8 = w >> 8;
                    uint4 v;
                    if constexpr (EXACT)
                        v = make_uint4(centred2<0>(w & 0x000f000fu), centred2<1>(w & 0x00f000f0u), centred2<0>(w8 & 0x000f000fu),
                                       centred2<1>(w8 & 0x00f000f0u));
                    else
                        v = make_uint4(value2<0>(w & 0x000f000fu, s2, o2), value2<1>(w & 0x00f000f0u, s2, o2),
                                       value2<0>(w8 & 0x000f000fu, s2, o2), value2<1>(w8 & 0x00f000f0u, s2, o2));
                    *reinterpret_cast<uint4 *>(to + (i >> 3) * PANEL + (((i & 7) ^ (u & 7)) << 4)) = v;
                }
                fence_async();
                bar_arrive(&ctl->k_full);
                fetch(t + 1);          // on their way while this thread waits for a free stage
                look_up(t + 2);
            }
            tiles_before += all;
        }
    } else if (warp < kProductWarp) {
        // ---- values, transposed: a row per dim, eight neighbouring keys are 16 bytes of it.  A thread takes D / 64 times a word
        // of eight dims of eight keys; pages are looked up two tiles ahead, codes fetched one tile ahead ----
        constexpr int NV = D / 64;
        const int u = tid - (kSoftmaxWarps + kUnpackWarps) * 32, uw = u >> 5;
        const int mask = (1 << p.page_shift) - 1;
        // eight lanes hold the groups of eight keys of half a tile, so that their 16-byte pieces of a row hit different banks
        const int group = (lane & 7) + 8 * (uw & 1), word0 = (lane >> 3) + 4 * (uw >> 1);
        while (next_item(p, walk, x)) {
            const int all = tiles_of(x);
            const int32_t *const table = p.block_table + (long long)x.row * p.table_ld;
            const unsigned char *const v_head = p.v_codes + x.head * p.hs + word0 * 4;
            const uint32_t *const km_head = p.k_meta + x.head * p.mhs, *const vm_head = p.v_meta + x.head * p.mhs;
            uint32_t page = kNone, group_page = kNone, next[NV][8], next_km = 0, next_vm = 0;   // of the thread's key, of its group
            const auto look_up = [&](int t) {
                const int key = x.first_key + t * kTile + u, first = x.first_key + t * kTile + 8 * group;
                page = t < all && key < x.len ? (uint32_t)__ldg(table + (key >> p.page_shift)) : kNone;
                group_page = t < all && first < x.len ? (uint32_t)__ldg(table + (first >> p.page_shift)) : kNone;
            };
            const auto fetch = [&](int t) {
                const int key = x.first_key + t * kTile + u, first = x.first_key + t * kTile + 8 * group;
                next_km = next_vm = 0;
                if (page < (uint32_t)p.num_pages) {
                    const uint32_t moff = page * p.mps + (uint32_t)(key & mask) * p.mts;
                    next_km = __ldg(km_head + moff);
                    next_vm = __ldg(vm_head + moff);
                }
                const bool there = group_page < (uint32_t)p.num_pages;
                const unsigned char *const from = v_head + (group_page * p.ps + (uint32_t)(first & mask) * p.ts) * 16ull;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        next[i][e] = there ? __ldg(reinterpret_cast<const uint32_t *>(from + i * 32 + (unsigned long long)(e * p.ts) * 16)) : 0u;
            };
            look_up(0);
            fetch(0);
            look_up(1);
            for (int t = 0; t < all; ++t) {
                const uint32_t n = tiles_before + t;
                const KeyMeta meta(next_km, next_vm);
                const float scale = meta.bad ? 0.f : meta_scale(meta.v), offset = meta.bad ? 0.f : meta_offset(meta.v);
                const int e = tile_power(fmaxf(fabsf(offset), fabsf(fmaf(15.f, scale, offset))), ctl->red[n & 1][1], uw, lane, 2);
                const float f = __uint_as_float((uint32_t)(127 - e) << 23);
                if (u == 0) {          // (the product of tile n - 2 is done: both halves have taken the power of n - 4)
                    ctl->v_power[n & 3] = (float)e;
                    bar_arrive(&ctl->v_info[n & 3]);
                }
                bar_wait(&ctl->v_empty, (n & 1) ^ 1, ctl, p);
                ctl->meta[u] = half2_bits(scale * f, offset * f);
                asm volatile("bar.sync 2, 128;" ::: "memory");
                unsigned char *const to = smem + S::v + (group >> 3) * (D * 128) + word0 * 1024;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {                        // four dims at a time: the registers hold no more
                        uint32_t v[4][4];                                // pairs of keys; dims
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const uint2 m = *reinterpret_cast<const uint2 *>(ctl->meta + 8 * group + 2 * q);
                            const uint32_t sc = __byte_perm(m.x, m.y, 0x5410), of = __byte_perm(m.x, m.y, 0x7632);
                            const __half2 s2 = reinterpret_cast<const __half2 &>(sc), o2 = reinterpret_cast<const __half2 &>(of);
                            const uint32_t c = __byte_perm(next[i][2 * q], next[i][2 * q + 1], h ? 0x7632 : 0x5410), c8 = c >> 8;
                            v[q][0] = value2<0>(c & 0x000f000fu, s2, o2);
                            v[q][1] = value2<1>(c & 0x00f000f0u, s2, o2);
                            v[q][2] = value2<0>(c8 & 0x000f000fu, s2, o2);
                            v[q][3] = value2<1>(c8 & 0x00f000f0u, s2, o2);
                        }
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            *reinterpret_cast<uint4 *>(to + i * 8192 + (4 * h + d) * 128 + (((group & 7) ^ (4 * h + d)) << 4)) =
                                make_uint4(v[0][d], v[1][d], v[2][d], v[3][d]);
                    }
                }
                fence_async();
                bar_arrive(&ctl->v_full);
                fetch(t + 1);
                look_up(t + 2);
            }
            tiles_before += all;
        }
    } else if (lane == 0) {
        // ---- the products ----
        const uint32_t q_at = smem_at(smem + S::q), k_at = smem_at(smem + S::k), v_at = smem_at(smem + S::v), p_at = smem_at(smem + S::p);
        uint32_t items_before = 0;
        bool go = true;                                       // no wait has been given up here
        // S of tile n for half h
        const auto scores = [&](int h) {
            tc_after();
#pragma unroll
            for (int i = 0; i < D / 16; ++i)
                mma_f16(tmem + h * kTile, operand(q_at + h * S::kQ + (i >> 2) * PANEL) + 2 * (i & 3), operand(k_at + (i >> 2) * PANEL) + 2 * (i & 3),
                        kTile, i != 0);
            tc_commit(&ctl->s_full[h]);
        };
        while (go && next_item(p, walk, x)) {
            const int all = tiles_of(x);
            if (all == 0) continue;
            go = bar_wait(&ctl->q_full, items_before & 1, ctl, p) && bar_wait(&ctl->k_full, tiles_before & 1, ctl, p);
            ++items_before;
            if (!go) break;
            if (x.tiles[0] > 0) scores(0);
            if (x.tiles[1] > 0) scores(1);
            tc_commit(&ctl->k_empty);
            for (int t = 0; t < all && go; ++t) {
                const uint32_t n = tiles_before + t;
                const bool more = t + 1 < all;
                go = bar_wait(&ctl->v_full, n & 1, ctl, p);
                if (more) go = bar_wait(&ctl->k_full, (n + 1) & 1, ctl, p) && go;
                // whichever half has its weights: its next S first, so that it goes on, then what the weights give
                bool open[2] = {true, true};
                for (uint32_t spins = 0; open[0] || open[1]; ++spins) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (!open[h]) continue;
                        // the last one open is waited for, with the limit; of two each is tried in turn, for a while
                        if (open[h ^ 1] && spins < (1u << 24)) {
                            if (!bar_try(&ctl->p_full[h], n & 1)) {
                                if (!ctl->gave_up) continue;
                                go = false;
                            }
                        } else {
                            go = bar_wait(&ctl->p_full[h], n & 1, ctl, p) && go;
                        }
                        open[h] = false;
                        if (t >= x.tiles[h] || !go) continue;
                        if (t + 1 < x.tiles[h]) scores(h);
                        tc_after();
#pragma unroll
                        for (int i = 0; i < kTile / 16; ++i)
                            mma_f16(tmem + 2 * kTile + h * kTile, operand(p_at + h * S::kP + (i >> 2) * PANEL) + 2 * (i & 3),
                                    operand(v_at + (i >> 2) * (D * 128)) + 2 * (i & 3), D, (t | i) != 0);
                        tc_commit(&ctl->pv_done[h]);
                    }
                }
                if (more) tc_commit(&ctl->k_empty);
                tc_commit(&ctl->v_empty);
            }
            tiles_before += all;
        }
        // no product is on its way when TMEM is freed, after a wait that was given up either
        tc_commit(&ctl->drained);
        const long long t0 = clock64();
        bool over = false;
        while (!(over = bar_try(&ctl->drained, 0)) && clock64() - t0 < kDrainLimit) {}
        if (!over) atomicOr(p.status, 4);
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
    }
}

template <int D>
constexpr int prompt_smem() { return PromptSmem<D>::bytes; }

const void *prompt_kernel(bool wide, bool exact) {
    if (wide) return exact ? reinterpret_cast<const void *>(&kv_attend_prompt_kernel<128, true>) : reinterpret_cast<const void *>(&kv_attend_prompt_kernel<128, false>);
    return exact ? reinterpret_cast<const void *>(&kv_attend_prompt_kernel<64, true>) : reinterpret_cast<const void *>(&kv_attend_prompt_kernel<64, false>);
}

}  // namespace

// Which kernel.  The one for few rows takes its time by tiles of 16 rows, however they are spread: it cuts long keys over CTAs.  This
// one takes its time by rounds of CTAs, whose keys are not cut.  Both grow with the keys, so the choice does not need their number:
// measured (bf16, head_dim 128, 4 heads to a key head, 8,192 keys) a tile of 16 rows takes 0.39 us, a round of 148 CTAs 167 to 204,
// with the logarithm 223 to 254: as long as 3.2 or 4.2 tiles per CTA (head_dim 64: 0.23 us, 143 to 171, 186 to 219: 4.2 or 5.4).  16 requests x 8 key heads x 64 rows: 199 us there, 167 (223) us
// here; 32 rows: 108 and 167 (223); one request of 2,048 rows: 368 and 204 (254); 512 rows: 104 and 200 (253).  Not every request has
// as many rows as the largest: all of them have no more than max_tokens tokens, and no more than one tile or item each that is
// not full.  One prompt of 1,024 tokens beside 255 single tokens, 2,000 keys each: 413 us there, 755 (964) here; four of 512
// beside 60, 4,000 keys: 838 and 482 (619).  Short keys leave the other kernel waiting for its starts and joins: at 512 keys and 256
// rows of one request it takes 37 us, this one 28 (31); at 128 rows 20 and 22.  (The table's columns stand for the keys, which are on the
// device.)  A hint of more queries than there are tokens asks for this kernel.
bool prompt_kernel_serves(const fi_kv *kv, const AttendParams &p, int dtype, long long queries) {
    if (dtype != FI_BF16 || (kv->cfg.head_dim != 64 && kv->cfg.head_dim != 128)) return false;
    if (queries > p.max_tokens) return true;
    const double rows = (double)queries * p.group, all_rows = (double)p.max_tokens * p.group, batch = p.batch_max;
    const auto blocks = [&](int size) {
        const double whole = batch * (double)(long long)((rows + size - 1) / size), packed = all_rows / size + batch;
        return kv->cfg.kv_heads * (whole < packed ? whole : packed);
    };
    const double rounds = (double)(long long)((blocks(kRows) + kv->sm_count - 1) / kv->sm_count);
    const double tiles_a_round = kv->cfg.head_dim == 64 ? (p.lse ? 5.4 : 4.2) : (p.lse ? 4.2 : 3.2);
    if (blocks(16) > tiles_a_round * kv->sm_count * rounds) return true;
    return rows >= 256 && all_rows >= 256 * batch && (long long)p.max_blocks << p.page_shift <= 1024;
}

fi_status_t prepare_attend_prompt(const fi_kv *kv) {
    const bool wide = kv->cfg.head_dim == 128;
    if (!wide && kv->cfg.head_dim != 64) return FI_OK;
    cudaError_t e = cudaSuccess;
    for (int exact = 0; exact < 2 && e == cudaSuccess; ++exact)
        e = cudaFuncSetAttribute(prompt_kernel(wide, exact != 0), cudaFuncAttributeMaxDynamicSharedMemorySize, wide ? prompt_smem<128>() : prompt_smem<64>());
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_kv_create: attention kernels");
}

fi_status_t launch_attend_prompt(const fi_kv *kv, const AttendParams &p, long long rows, cudaStream_t stream) {
    const double items = (double)p.batch_max * kv->cfg.kv_heads * (double)((rows + kRows - 1) / kRows);
    const int grid = items < kv->sm_count ? (int)items : kv->sm_count;
    const bool wide = kv->cfg.head_dim == 128;
    AttendParams args = p;
    void *list[] = {&args};
    const cudaError_t e = cudaLaunchKernel(prompt_kernel(wide, p.lse != nullptr), dim3((unsigned)grid), dim3(kPromptThreads), list,
                                           (size_t)(wide ? prompt_smem<128>() : prompt_smem<64>()), stream);
    count_launch();
    if (e != cudaSuccess) return cuda_fail(e, "fi_kv_attend");
    return check_launch("fi_kv_attend");
}

}  // namespace fi

// The products of a layer: y = act(x W^T + b) + r for a list of rows, and the gradients.
//
// All three products are one form, D[n][m] = sum_k A(m, k) B(n, k), with the output's contiguous dimension as the MMA's
// rows, so that the 32 lanes of a warp hold neighbouring values of one output row and store them side by side:
//   forward    D = y   [tokens][out]   A = W  (k contiguous)   B = x  (k contiguous)      k over in
//   dx         D = dx  [tokens][in]    A = W  (m contiguous)   B = dz (k contiguous)      k over out
//   dW         D = dW  [out][in]       A = x  (m contiguous)   B = dz (n contiguous)      k over tokens
// Operands come by TMA in blocks of 64 along k, 128-byte swizzle, as they lie in memory: the tensor cores take either order.
// Sums are fp32 in TMEM, long ones in pieces.
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "fi_internal.cuh"

namespace fi {
namespace {

constexpr int kM = 128;                   // output columns of a CTA (MMA rows)
constexpr int kKb = 64;                   // reduction values of a block: 128 bytes, a line of the swizzle
constexpr int kABytes = kM * kKb * 2;     // of a block
constexpr int kMaxN = 256;                // output rows of a tile, at most
constexpr int kMaxPairN32 = 192;          // of a pair's tile with float32 results, whose sums are in registers
constexpr int kMaxStages = 12;
// Blocks of the reduction that are added up in one accumulator.  The tensor cores cut what they add: a running sum of one sign loses 2^-24
// of itself with every 16 values, 2^-23 at most.  So float32 results are taken out of them every 512 values, bfloat16 results, which are
// rounded to 2^-8, every 16,384 (2^-15 of the sum, 2^-13 at most; left there for 2^20 values: 2^-9, and results are a step off).
constexpr int kPiece = 8, kHalfPiece = 256;
template <bool F32>
constexpr int kPieceOf = F32 ? kPiece : kHalfPiece;
constexpr int kEpiThreads = 256;          // warps 0..7: TMEM lanes 32 (w mod 4) ..; warp 8 loads, warp 9 issues the products
constexpr int kThreads = kEpiThreads + 64;
constexpr int kSmemMost = 227 * 1024, kStaticMost = 22 * 1024;
constexpr long long kWaitLimit = 8000000000ll;   // SM cycles (about 4 s)
constexpr long long kShortLimit = 1 << 20;       // limits below it are a test's
constexpr long long kDrainLimit = 200000000ll;   // (about 0.1 s)

__device__ int32_t g_linear_status;       // 1: a bounded wait ran out

constexpr int kRing = 4;                  // accumulators of a single CTA's long sum, at most

struct LinearCtl {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t done, never;
    uint64_t sums_full[kRing], sums_empty[kRing];
    uint32_t tmem;
    volatile int gave_up;
};

struct PairCtl {
    uint64_t full[kMaxStages], empty[kMaxStages];
    uint64_t sums_full[2], sums_empty[2];
    uint64_t never;
    uint32_t tmem;
    volatile int gave_up;
    alignas(16) float bias[kEpiThreads / 32][kMaxN / 2];      // of the columns that a warp works on
    alignas(128) uint4 turn[kEpiThreads / 32][128];           // 64 bytes of its 32 rows
};

struct LinearParams {
    const float *bias;             // [m]
    const void *residual;          // type of out
    void *out;
    __nv_bfloat16 *preact;
    const int32_t *rows, *count;
    long long ld_res, ld_out, ld_preact, out_rows, wait_limit;
    int m, n, kb;                  // output columns, rows; steps of the reduction: one or two blocks of 64, a stage each
    int m_tiles, tile_n;
    int split;                     // CTAs, or pairs of them, of a cluster that share a tile's reduction
    int bufs;                      // accumulators that a CTA's reduction is cut into
    int piece;                     // single CTAs: steps of an accumulator where there are more pieces than fit, which then take turns; else 0
    int tmem_cols, stages, b_bytes;
    int part_at;                   // place of a CTA's sums in shared memory
    int early;                     // two products in one launch: see TileWalk
    int wide;                      // rows of out, residual, preact and the bias lie on 16-byte boundaries
};

__device__ __forceinline__ uint32_t smem_at(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void bar_init(uint64_t *bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_at(bar)), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_expect(uint64_t *bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_at(bar)), "r"(bytes) : "memory");
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
// Bounded wait: when one gives up, every later wait of the CTA does so at once, the kernel runs to its end with whatever is in its
// buffers, and the status word says that the results are not valid.
template <typename Ctl>
__device__ __noinline__ bool bar_wait_long(uint64_t *bar, uint32_t parity, Ctl *ctl, long long limit) {
    const long long t0 = clock64();
    for (uint32_t spins = 1;; ++spins) {
        if (bar_try(bar, parity)) return true;
        if ((spins & 255) == 0) {
            if (ctl->gave_up) return false;
            if (clock64() - t0 > limit) {
                ctl->gave_up = 1;
                atomicOr(&g_linear_status, 1);
                return false;
            }
        }
    }
}
template <typename Ctl>
__device__ __forceinline__ bool bar_wait(uint64_t *bar, uint32_t parity, Ctl *ctl, long long limit) {
    return bar_try(bar, parity) || bar_wait_long(bar, parity, ctl, limit);
}
// the same for a whole warp
template <typename Ctl>
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Ctl *ctl, long long limit) {
    return __all_sync(0xffffffffu, bar_try(bar, parity)) || __all_sync(0xffffffffu, bar_wait_long(bar, parity, ctl, limit));
}
// for the end of a role, whichever one has given up: what it has started is over before the CTA leaves
template <typename Ctl>
__device__ __forceinline__ void bar_drain(uint64_t *bar, uint32_t parity, Ctl *ctl) {
    const long long t0 = clock64();
    while (!bar_try(bar, parity))
        if (clock64() - t0 > (ctl->gave_up ? kDrainLimit : kWaitLimit)) {
            atomicOr(&g_linear_status, 1);
            return;
        }
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint64_t *bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_at(bar)) : "memory");
}
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap *map, uint64_t *bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(smem_at(bar)), "r"(x), "r"(y)
        : "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t addr, uint32_t rank) {
    uint32_t out;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"(addr), "r"(rank));
    return out;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}

// One lane of the warp, always the same, for the instructions that are issued once; the loops around them are the whole warp's, so that their
// operands stay in uniform registers (with the loops in one lane a block of the reduction took 650 cycles to issue, more than its products).
__device__ __forceinline__ bool elect_one() {
    uint32_t yes;
    asm volatile(
        "{\n"
        ".reg .pred p;\n"
        "elect.sync _|p, 0xffffffff;\n"
        "selp.u32 %0, 1, 0, p;\n"
        "}\n"
        : "=r"(yes));
    return yes != 0;
}

// Operand in shared memory, 128-byte swizzle; low word of its descriptor.  Reduction contiguous: rows of 128 bytes, groups of eight 1,024 bytes
// apart.  Else (MN) a line of 128 bytes holds 64 rows at one k: 8 k's are 1,024 bytes, the next 64 rows 8,192 bytes further.
template <bool MN>
__device__ __forceinline__ uint32_t operand(uint32_t addr) {
    return (addr & 0x3ffffu) >> 4 | (uint32_t)(MN ? 8192 >> 4 : 1) << 16;    // (in a cluster an address has its CTA in the bits above)
}
constexpr uint32_t kOperandHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
// between the k's of successive MMAs (16 of them), in units of 16 bytes
template <bool MN>
constexpr uint32_t kOperandStep = MN ? 2048 >> 4 : 32 >> 4;

// bf16 x bf16 -> fp32
__device__ __forceinline__ uint32_t instruction(int m, int n, bool a_mn, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)a_mn << 15) | ((uint32_t)b_mn << 16) | ((uint32_t)(n >> 3) << 17) |
           ((uint32_t)(m >> 4) << 24);
}
// one block of the reduction, 4 MMAs of 16; PAIR: D (256 x N, 128 rows in each CTA's TMEM) from 128 rows of A and N / 2 of B in each CTA
template <bool PAIR, bool A_MN, bool B_MN>
__device__ __forceinline__ void mma_block(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
#pragma unroll
    for (int i = 0; i < kKb / 16; ++i) {
        const uint32_t a_low = a + i * kOperandStep<A_MN>, b_low = b + i * kOperandStep<B_MN>, more = i ? 1u : accumulate;
        if (PAIR)
            asm volatile(
                "{\n"
                ".reg .pred p;\n"
                ".reg .b64 x, y;\n"
                "setp.ne.b32 p, %4, 0;\n"
                "mov.b64 x, {%1, %5};\n"
                "mov.b64 y, {%2, %5};\n"
                "tcgen05.mma.cta_group::2.kind::f16 [%0], x, y, %3, p;\n"
                "}\n" ::"r"(d),
                "r"(a_low), "r"(b_low), "r"(idesc), "r"(more), "r"(kOperandHigh)
                : "memory");
        else
            asm volatile(
                "{\n"
                ".reg .pred p;\n"
                ".reg .b64 x, y;\n"
                "setp.ne.b32 p, %4, 0;\n"
                "mov.b64 x, {%1, %5};\n"
                "mov.b64 y, {%2, %5};\n"
                "tcgen05.mma.cta_group::1.kind::f16 [%0], x, y, %3, p;\n"
                "}\n" ::"r"(d),
                "r"(a_low), "r"(b_low), "r"(idesc), "r"(more), "r"(kOperandHigh)
                : "memory");
    }
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
// wait for the loads; the registers may only be used behind it
__device__ __forceinline__ void tmem_wait(uint32_t *v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]),
                   "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15])
                 :
                 : "memory");
}
__device__ __forceinline__ void tmem_store(uint32_t addr, const uint32_t *v) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(v[0]), "r"(v[1]), "r"(v[2]),
        "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
        "r"(addr)
        : "memory");
}
// the accumulators take turns
__device__ __forceinline__ void next_buffer(uint32_t &buf, uint32_t &phase, uint32_t bufs = 2) {
    if (++buf == bufs) {
        buf = 0;
        phase ^= 1;
    }
}
// Long sums: the piece at `to` takes up the sum so far, at `from`, which is free then.  Columns from `first` on, 16 at a time.
__device__ __forceinline__ void join_pieces(uint32_t from, uint32_t to, int first, int cols, int step) {
#pragma unroll 1
    for (int c = first; c < cols; c += step) {
        uint32_t v[16], w[16];
        tmem_load(from + c, v);
        tmem_load(to + c, w);
        tmem_wait(v);
        tmem_wait(w);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
        tmem_store(to + c, v);
    }
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
    tc_before();
    __syncwarp();
}
// Exponential and reciprocal of the special-function unit (2^-22 of the result).  At full power the clock falls with every instruction that is
// executed beside the products, so the activation is kept short (8,191 x 4,096 -> 16,384 and back with the library's erfcf: 909 us, so: 799).
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float recip_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Kernels here are launched while the one before them in the stream still runs, and set themselves up meanwhile; nothing that it may write is
// read, and nothing that it may read is written, before this.  The next one may begin at once.
__device__ __forceinline__ void in_turn() {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
}

constexpr float kLog2e = 1.4426950408889634f, kGeluTanh = 0.044715f, kGeluTwice = 1.5957691216057308f;   // 2 sqrt(2 / pi)

// 1 / (1 + 2^-x)
__device__ __forceinline__ float logistic2(float x) { return recip_fast(1.f + exp2_fast(-x)); }

__device__ __forceinline__ uint64_t pair_of(float a, float b) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, float c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(pair_of(c, c)));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
// Phi(z) = erfc(-z / sqrt 2) / 2, from erfc(a) = exp(-a^2) t P(t), t = 1 / (1 + 0.43 a), for a >= 0.  P is the polynomial of seventh degree whose
// largest error relative to erfc is least (8.5e-8, by Remez' exchange; half of it here), so that the left tail is right to a few 2^-24 of
// itself and to what the exponent's rounding does: 1.1 z^2 2^-24.  density: exp(-z^2 / 2).  Two values at a time: the polynomial of one at a time
// makes the slopes' kernel slower, 45.3 instead of 42.9 us for 4,095 x 8,192.
__device__ __forceinline__ void normal_cdf(float z0, float z1, float (&cdf)[2], float (&density)[2]) {
    constexpr float c[8] = {0.12125748710f, 0.12218486825f, 0.10249370120f, 0.12336100105f, -0.042744353075f, 0.19172071880f, -0.15510789720f, 0.03683451189f};
    const uint64_t t = pair_of(recip_fast(fmaf(fabsf(z0), 0.43f * 0.70710678f, 1.f)), recip_fast(fmaf(fabsf(z1), 0.43f * 0.70710678f, 1.f)));
    density[0] = exp2_fast(z0 * z0 * (-0.5f * kLog2e));
    density[1] = exp2_fast(z1 * z1 * (-0.5f * kLog2e));
    uint64_t q = pair_of(c[7], c[7]);
#pragma unroll
    for (int i = 6; i >= 0; --i) q = fma2(t, q, c[i]);
    q = mul2(mul2(q, t), pair_of(density[0], density[1]));
    float q0, q1;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(q0), "=f"(q1) : "l"(q));
    cdf[0] = z0 >= 0.f ? 1.f - q0 : q0;
    cdf[1] = z1 >= 0.f ? 1.f - q1 : q1;
}

template <int ACT, int N>
__device__ __forceinline__ void activate(float (&z)[N]) {
    switch (ACT) {
        case FI_ACT_RELU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] = z[i] < 0.f ? 0.f : z[i];      // (NaN stays)
            break;
        case FI_ACT_GELU:
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                float cdf[2], density[2];
                normal_cdf(z[i], z[i + 1], cdf, density);
                z[i] *= cdf[0];
                z[i + 1] *= cdf[1];
            }
            break;
        case FI_ACT_GELU_TANH:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= logistic2(z[i] * fmaf(kGeluTwice * kGeluTanh * kLog2e, z[i] * z[i], kGeluTwice * kLog2e));
            break;
        case FI_ACT_SILU:
#pragma unroll
            for (int i = 0; i < N; ++i) z[i] *= logistic2(z[i] * kLog2e);
            break;
        default: break;
    }
}

// z within -most .. most (NaN stays): past there every slope has reached 0 or 1, and no product of infinities comes up
__device__ __forceinline__ float within(float z, float most) {
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(z), "f"(most));
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(y), "f"(-most));
    return y;
}

// slopes of the activation, of two values
template <int ACT>
__device__ __forceinline__ float slope(float z) {
    switch (ACT) {
        case FI_ACT_RELU: return z > 0.f ? 1.f : z <= 0.f ? 0.f : z;
        case FI_ACT_GELU_TANH: {
            z = within(z, 20.f);
            const float zz = z * z, s = logistic2(z * fmaf(kGeluTwice * kGeluTanh * kLog2e, zz, kGeluTwice * kLog2e));
            return fmaf(z * fmaf(-s, s, s), fmaf(kGeluTwice * 3.f * kGeluTanh, zz, kGeluTwice), s);
        }
        case FI_ACT_SILU: {
            z = within(z, 100.f);
            const float s = logistic2(z * kLog2e);
            return s * fmaf(z, 1.f - s, 1.f);
        }
        default: return 1.f;
    }
}
template <int ACT>
__device__ __forceinline__ void slopes(float &z0, float &z1) {
    if (ACT == FI_ACT_GELU) {
        z0 = within(z0, 20.f);
        z1 = within(z1, 20.f);
        float cdf[2], density[2];
        normal_cdf(z0, z1, cdf, density);
        z0 = fmaf(z0 * 0.39894228f, density[0], cdf[0]);
        z1 = fmaf(z1 * 0.39894228f, density[1], cdf[1]);
    } else {
        z0 = slope<ACT>(z0);
        z1 = slope<ACT>(z1);
    }
}

__device__ __forceinline__ int actual_rows(const LinearParams &p) {
    if (!p.count) return p.n;
    const int c = *p.count;
    return c < 0 ? 0 : c > p.n ? p.n : c;
}

constexpr int kNoRow = -1, kSkipRow = -2;   // no such row of the product; a row that is in no row of out

// Row of out that row n of the product goes to, or one of these.
__device__ __forceinline__ int row_of(const LinearParams &p, int n, int rows) {
    if (n >= rows) return kNoRow;
    if (!p.rows) return n;
    const int to = p.rows[n];
    return to >= 0 && to < p.out_rows ? to : kSkipRow;
}

// What becomes of N sums, column m and rows n0, n0 + 1 .. of the product; to[i]: their rows of out, negative: none.  (Every choice is
// made once for all of them, the activation when the kernel is compiled: what runs is short, and loads are on the way together.)
template <bool F32, int ACT, int N>
__device__ __forceinline__ void finish(const LinearParams &p, float (&v)[N], float bias, int m, int n0, const int (&to)[N]) {
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    T r[N];
    const bool here = m < p.m;
    if (p.residual) {
        const T *const from = static_cast<const T *>(p.residual) + m;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (here && to[i] >= 0) r[i] = from[to[i] * p.ld_res];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += bias;
    if (p.preact) {
        __nv_bfloat16 *const z = p.preact + (long long)n0 * p.ld_preact + m;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (here && to[i] != kNoRow) z[i * p.ld_preact] = __float2bfloat16_rn(v[i]);
    }
    activate<ACT>(v);
    if (p.residual) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += (float)r[i];
    }
    T *const out = static_cast<T *>(p.out) + m;
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (here && to[i] >= 0) out[to[i] * p.ld_out] = (T)v[i];
}

__device__ __forceinline__ void cluster_store4(uint32_t addr, const uint32_t *v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(map)) : "memory");
}

// Few tiles: a CTA takes 128 output columns and up to 256 output rows; `split` CTAs of a cluster share its reduction, so that the SMs have
// work where the tiles alone are fewer than they are.  Sums of four rows go to CTA (row / 4) mod split, which adds them up in the order of
// the ranks.  Bound by the latency from the start to the last store (one token 2,048 -> 2,560: 5.2 us; its call takes the host 8.2), and by the
// operands' way from memory (48 tokens 4,096 -> 16,384: 28 us for 134 MB of weights, 4.8 TB/s): the loader sets up its barriers and has all
// stages on the way before the CTA has its TMEM.  LONG: more pieces of the reduction than accumulators, which take turns: a
// kernel of its own, as its tests cost the other one up to 2 % (16 tokens 8,192 -> 8,192 in float32 24.5 -> 24.9 us).
template <bool F32, int ACT, bool A_MN, bool B_MN, int DEPTH, bool LONG>
__global__ void __launch_bounds__(kThreads, 1) linear_split_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                   const __grid_constant__ CUtensorMap map_b,
                                                                   const __grid_constant__ LinearParams p) {
    extern __shared__ unsigned char raw_smem[];
    __shared__ LinearCtl ctl_space;
    LinearCtl *const ctl = &ctl_space;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int tile = blockIdx.x / p.split, rank = blockIdx.x - tile * p.split;
    const int m0 = (tile % p.m_tiles) * kM, n0 = (tile / p.m_tiles) * p.tile_n;
    const uint32_t smem = (smem_at(raw_smem) + 1023) & ~1023u;
    const int kb0 = (int)((long long)p.kb * rank / p.split), kb1 = (int)((long long)p.kb * (rank + 1) / p.split);
    const uint32_t block_bytes = kABytes + p.b_bytes, stage_bytes = DEPTH * block_bytes;
    uint32_t stage = 0, phase = 0;                          // of the loader, of the products
    const auto next_stage = [&] {
        if (++stage == (uint32_t)p.stages) {
            stage = 0;
            phase ^= 1;
        }
    };
    const auto load = [&](int kb) {
        if (elect_one()) {
            uint64_t *const bar = &ctl->full[stage];
            bar_expect(bar, stage_bytes);
#pragma unroll
            for (int i = 0; i < DEPTH; ++i) {               // (a second block past the end is zeros)
                const uint32_t a = smem + stage * stage_bytes + i * block_bytes, b = a + kABytes;
                const int k = (kb * DEPTH + i) * kKb;
                if (A_MN) {
                    load_box(a, &map_a, bar, m0, k);
                    load_box(a + 8192, &map_a, bar, m0 + 64, k);
                } else {
                    load_box(a, &map_a, bar, k, m0);
                }
                if (B_MN)
                    for (int c = 0; c < p.tile_n; c += 64) load_box(b + c * 128, &map_b, bar, n0 + c, k);
                else
                    load_box(b, &map_b, bar, k, n0);
            }
        }
        __syncwarp();
        next_stage();
    };
    const int early = min(kb1 - kb0, p.stages);             // blocks that need no free stage
    if (warp == 8) {
        if (elect_one()) {
            prefetch_map(&map_a);
            prefetch_map(&map_b);
            for (int s = 0; s < p.stages; ++s) {
                bar_init(&ctl->full[s], 1);
                bar_init(&ctl->empty[s], 1);
            }
            bar_init(&ctl->done, 1);
            bar_init(&ctl->never, 1);
            ctl->gave_up = 0;
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
        in_turn();
        for (int i = 0; i < early; ++i) load(kb0 + i);
    }
    if (LONG && warp == 9) {
        if (elect_one()) {
            for (int i = 0; i < p.bufs; ++i) {
                bar_init(&ctl->sums_full[i], 1);
                bar_init(&ctl->sums_empty[i], kEpiThreads / 32);
            }
            asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        __syncwarp();
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&ctl->tmem)), "r"(p.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = ctl->tmem;
    if (warp != 8) in_turn();
    const int rows = actual_rows(p);
    const bool apart = p.split > 1 && p.part_at > 0;
    if (apart) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    const int cols = min(p.tile_n, rows - n0);              // rows of the output that there are; no more is done if there is none
    // so that a wait runs out for certain
    if (p.wait_limit < kShortLimit && tid == 0) bar_wait(&ctl->never, 0, ctl, p.wait_limit);
    uint32_t last_buf = 0, last_phase = 0;                  // LONG: the accumulator that holds the sum in the end
    if (warp == 8) {
        int kb = kb0 + early;
        if (cols > 0)
            for (; kb < kb1; ++kb) {
                if (!warp_wait(&ctl->empty[stage], phase ^ 1, ctl, p.wait_limit)) break;
                load(kb);
            }
        for (int back = min(kb - kb0, p.stages); back > 0; --back) {             // (at once where the products have been through)
            if (stage == 0) {
                stage = p.stages;
                phase ^= 1;
            }
            bar_drain(&ctl->full[--stage], phase, ctl);
        }
    } else if (warp == 9) {
        if (cols > 0) {
            const uint32_t idesc = instruction(kM, p.tile_n, A_MN, B_MN);
            const int length = LONG ? p.piece : (kb1 - kb0 + p.bufs - 1) / p.bufs;
            uint32_t buf = 0, buf_phase = 0;
            bool ok = true;
            for (int kb = kb0; kb < kb1 && ok;) {
                if (LONG) {
                    ok = warp_wait(&ctl->sums_empty[buf], buf_phase ^ 1, ctl, p.wait_limit);
                    if (!ok) break;
                    tc_after();
                }
                const uint32_t d = tmem + buf * p.tile_n;
                const int end = min(kb + length, kb1);
                for (uint32_t more = 0; kb < end; ++kb, more = 1) {
                    ok = warp_wait(&ctl->full[stage], phase, ctl, p.wait_limit);
                    if (!ok) break;
                    tc_after();
                    if (elect_one()) {
#pragma unroll
                        for (int i = 0; i < DEPTH; ++i) {
                            const uint32_t at = smem + stage * stage_bytes + i * block_bytes;
                            mma_block<false, A_MN, B_MN>(d, operand<A_MN>(at), operand<B_MN>(at + kABytes), idesc, i ? 1u : more);
                        }
                        tc_commit(&ctl->empty[stage]);
                    }
                    __syncwarp();
                    next_stage();
                }
                if (LONG) {
                    if (elect_one()) tc_commit(&ctl->sums_full[buf]);
                    __syncwarp();
                }
                next_buffer(buf, buf_phase, p.bufs);
            }
            if (elect_one()) tc_commit(&ctl->done);
            __syncwarp();
            bar_drain(&ctl->done, 0, ctl);
        }
    } else if (cols > 0) {
        if (LONG)
            for (int kb = kb0 + p.piece; kb < kb1; kb += p.piece) {
                const uint32_t old = last_buf, at = tmem + ((uint32_t)((warp & 3) * 32) << 16);
                next_buffer(last_buf, last_phase, p.bufs);
                if (!warp_wait(&ctl->sums_full[last_buf], last_phase, ctl, p.wait_limit)) break;
                tc_after();
                join_pieces(at + old * p.tile_n, at + last_buf * p.tile_n, (warp >> 2) * 16, cols, 32);
                if (lane == 0) bar_arrive(&ctl->sums_empty[old]);
            }
        bar_wait(&ctl->done, 0, ctl, p.wait_limit);
        tc_after();
    }
    __syncthreads();                                        // (the loader too has nothing on its way now)
    // Sums of the CTA's reduction: [rank][group of four rows / split][128 columns][4] in the CTA that the group belongs to.  Few rows have a place of
    // their own behind the stages, others that of the stages, which all CTAs of the cluster have to be done with.
    const uint32_t part = smem + p.part_at;
    const int slots = (p.tile_n / 4 + p.split - 1) / p.split, shift = __ffs(p.split) - 1;       // (split is a power of two)
    if (apart) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // (all of them have started, long ago)
    else if (p.split > 1) cluster_sync();
    if (warp < 8 && cols > 0) {
        const int used = (kb1 - kb0 + p.bufs - 1) / p.bufs;                       // blocks of a buffer
        const int bufs = LONG ? 1 : (kb1 - kb0 + used - 1) / used;             // buffers that hold something
        const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + last_buf * p.tile_n;
        const uint32_t to = part + (rank * slots * kM + (warp & 3) * 32 + lane) * 16;
#pragma unroll 1
        for (int c = (warp >> 2) * 16; c < cols; c += 32) {
            uint32_t v[16], w[16];
            tmem_load(at + c, v);
            tmem_wait(v);
#pragma unroll 1
            for (int b = 1; b < bufs; ++b) {
                tmem_load(at + b * p.tile_n + c, w);
                tmem_wait(w);
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) + __uint_as_float(w[i]));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int group = (c >> 2) + i;
                if (group * 4 < cols) cluster_store4(map_to_rank(to + (group >> shift) * (kM * 16), group & (p.split - 1)), v + 4 * i);
            }
        }
        tc_before();
    }
    if (p.split > 1) cluster_sync();
    else __syncthreads();
    if (warp < 8) {
        const int m = m0 + (tid & (kM - 1));
        const float bias = p.bias && m < p.m ? p.bias[m] : 0.f;
#pragma unroll 1
        for (int slot = tid >> 7; (slot * p.split + rank) * 4 < cols; slot += 2) {
            const int c = (slot * p.split + rank) * 4;
            float v[4] = {};
            int to[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = row_of(p, n0 + c + i, rows < n0 + cols ? rows : n0 + cols);
#pragma unroll 1
            for (int s = 0; s < p.split; ++s) {
                float4 x;
                asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];"
                             : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w)
                             : "r"(part + ((s * slots + slot) * kM + (tid & (kM - 1))) * 16)
                             : "memory");
                v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w;
            }
            finish<F32, ACT>(p, v, bias, m, n0 + c, to);
        }
        tc_after();
    }
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols) : "memory");
}

// ---- pairs of CTAs: many tiles ----

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
// lands in this CTA's shared memory, counts its bytes on a barrier of the first CTA
__device__ __forceinline__ void load_box_pair(uint32_t dst, const CUtensorMap *map, uint32_t bar, int x, int y) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(x), "r"(y)
        : "memory");
}
// when the pair's products so far are over: the barrier at this place in both CTAs, `first` and the next of the cluster
__device__ __forceinline__ void tc_commit_pair(uint64_t *bar, uint32_t first) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_at(bar)),
                 "h"((uint16_t)(3u << first))
                 : "memory");
}
__device__ __forceinline__ void bar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}

// tile t of the product: groups of 8 tiles of rows are walked along the columns, so that the tiles that run at one time share their
// operands in L2
__device__ __forceinline__ void tile_place(int t, int row_tiles, int col_tiles, int &row_tile, int &col_tile) {
    constexpr int kGroup = 8;
    const int group = t / (kGroup * col_tiles), first = group * kGroup, width = min(kGroup, row_tiles - first), in = t - first * col_tiles;
    col_tile = in / width;
    row_tile = first + in - col_tile * width;
}

// 64 bytes of each of a warp's 32 rows on their way between registers (a thread has its row's) and memory, through 2 KB of shared memory: a
// warp's access then covers 8 rows by 64 bytes, not 32 rows by 16 (8,192 x 8,192 -> 8,192 added to a float32 stream: 1,133 -> 899 us).
__device__ __forceinline__ uint32_t turn_at(uint32_t base, int row, int piece) { return base + row * 64 + ((piece ^ (row >> 1 & 3)) << 4); }
__device__ __forceinline__ void shared_store4(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint4 shared_load4(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// columns c .. of row `to` (negative: none) of a matrix with `cols` columns: as the warp loads them, and turned to the threads' rows
template <typename T>
__device__ __forceinline__ void rows_load(const T *from, long long ld, int to, int c, int cols, uint32_t *w) {
    constexpr int kPieceCols = 16 / sizeof(T);
    const int lane = threadIdx.x & 31, col = c + (lane & 3) * kPieceCols;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = __shfl_sync(0xffffffffu, to, j * 8 + (lane >> 2));
        const uint4 v = row >= 0 && col < cols ? *reinterpret_cast<const uint4 *>(from + row * ld + col) : make_uint4(0, 0, 0, 0);
        w[4 * j] = v.x; w[4 * j + 1] = v.y; w[4 * j + 2] = v.z; w[4 * j + 3] = v.w;
    }
}
__device__ __forceinline__ void rows_turn(uint32_t base, uint32_t *w) {
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) shared_store4(turn_at(base, j * 8 + (lane >> 2), lane & 3), w[4 * j], w[4 * j + 1], w[4 * j + 2], w[4 * j + 3]);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint4 x = shared_load4(turn_at(base, lane, i));
        w[4 * i] = x.x; w[4 * i + 1] = x.y; w[4 * i + 2] = x.z; w[4 * i + 3] = x.w;
    }
}
template <typename T>
__device__ __forceinline__ void rows_out(T *out, long long ld, int to, int c, int cols, uint32_t base, const uint32_t (&w)[16]) {
    constexpr int kPieceCols = 16 / sizeof(T);
    const int lane = threadIdx.x & 31, col = c + (lane & 3) * kPieceCols;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 4; ++i) shared_store4(turn_at(base, lane, i), w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
    __syncwarp();
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int row = __shfl_sync(0xffffffffu, to, j * 8 + (lane >> 2));
        const uint4 v = shared_load4(turn_at(base, j * 8 + (lane >> 2), lane & 3));
        if (row >= 0 && col < cols) *reinterpret_cast<uint4 *>(out + row * ld + col) = v;
    }
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return reinterpret_cast<const uint32_t &>(h);
}

// Sums of a thread (row n of the product, negative: none; 16 columns from c on, of bfloat16 results 32) on their way out to row `to`.
// `bias`: of these columns, in shared memory; nullptr: none.  add: the residual is still to come.  p.wide: rows of out, residual and
// preact can be read and written 16 bytes at a time (the number of columns is a multiple of 8 anyway).
template <bool F32, int ACT>
__device__ __forceinline__ void finish_row(const LinearParams &p, float (&v)[F32 ? 16 : 32], int c, int n, int to, const float *bias, bool add,
                                           uint32_t base) {
    using T = typename std::conditional<F32, float, __nv_bfloat16>::type;
    constexpr int N = F32 ? 16 : 32;
    uint32_t r[16];
    if (add && p.wide) {
        rows_load(static_cast<const T *>(p.residual), p.ld_res, to, c, p.m, r);
        rows_turn(base, r);
    }
    if (bias) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const float4 b = *reinterpret_cast<const float4 *>(bias + i);
            v[i] += b.x; v[i + 1] += b.y; v[i + 2] += b.z; v[i + 3] += b.w;
        }
    }
    if (p.preact) {
        __nv_bfloat16 *const z = p.preact + (long long)n * p.ld_preact + c;
        uint32_t w[16];
        if (!F32 && p.wide) {
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = pack2(v[F32 ? 0 : 2 * i], v[F32 ? 0 : 2 * i + 1]);
            rows_out(p.preact, p.ld_preact, n, c, p.m, base, w);
        } else if (n >= 0) {
#pragma unroll
            for (int g = 0; g < N; g += 8)
                if (c + g < p.m)
#pragma unroll
                    for (int i = 0; i < 8; ++i) z[g + i] = __float2bfloat16_rn(v[g + i]);
        }
    }
    activate<ACT>(v);
    if (p.wide) {
        if (add) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] += F32 ? __uint_as_float(r[F32 ? i : 0]) : __uint_as_float(i & 1 ? r[F32 ? 0 : i / 2] & 0xffff0000u : r[F32 ? 0 : i / 2] << 16);
        }
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = F32 ? __float_as_uint(v[i]) : pack2(v[F32 ? 0 : 2 * i], v[F32 ? 0 : 2 * i + 1]);
        rows_out(static_cast<T *>(p.out), p.ld_out, to, c, p.m, base, w);
    } else if (to >= 0) {
        const T *const from = static_cast<const T *>(p.residual) + to * p.ld_res + c;
        T *const out = static_cast<T *>(p.out) + to * p.ld_out + c;
#pragma unroll
        for (int g = 0; g < N; g += 8)
            if (c + g < p.m)
#pragma unroll
                for (int i = 0; i < 8; ++i) out[g + i] = (T)(add ? v[g + i] + (float)from[g + i] : v[g + i]);
    }
}

// The tiles of a pair, one after another: every pairs-th one.  Of two products the second follows on the first: the pairs from `late` on,
// which have a tile less of the first, take `early` tiles of the second in its time, then all share the rest.  (Gradients of 4,095 tokens,
// 2,048 -> 8,192: 128 tiles of 128 steps and 256 of 64 on 74 pairs take 448 steps, one after the other in two launches 512.)
template <int JOBS>
struct TileWalk {
    int pair, pairs, tiles[2];
    int late = 0, early = 0, job = 0, k = 0, t = 0;
    __device__ __forceinline__ bool next() {
        if (JOBS == 1 || job == 0) {
            t = pair + k++ * pairs;
            if (t < tiles[0]) return true;
            if (JOBS == 1) return false;
            job = 1;
            k = 0;
        }
        const int lead = pairs - late, mine = pair >= late ? early : 0;
        t = k < mine ? k * lead + pair - late : early * lead + (k - mine) * pairs + pair;
        ++k;
        return t < tiles[1];
    }
};

// One pair of CTAs per two SMs walks over tiles of 256 output rows (128 per CTA) and tile_n output columns; each CTA loads its half of
// both operands.  Two accumulators in TMEM: the sums of one tile (F32: of 512 values of the
// reduction, else a piece of 16,384) go out while the next is formed.
// Here the MMA's rows are rows of the output, so that a thread has neighbouring values of one row: 16 bytes a store, the row looked up once.
// Bound by the tensor cores and, in long runs, by the power that they draw: 4,096^3 takes 94 us, 1,460 TFLOP/s (tensor pipe 91 % active);
// with float32 results, whose sums are added up outside of it, 104 us; 8,191 x 4,096 -> 16,384 651 to 665 us, 1,680 TFLOP/s.
// JOBS = 2: a second product behind the first, whose rows' operand lies the other way round (the two gradients).
// SPLIT = 2: two pairs, a cluster of 4, have a tile together, each half of its reduction; sums of half of the columns go to the other pair, and
// a cluster has no second tile.  (Tiles twice as wide bring half of the rows' operand through L2 for as many SMs.)
template <bool F32, int ACT, bool A_MN, bool B_MN, int DEPTH, int JOBS, int SPLIT>
__device__ __forceinline__ void linear_pair(const CUtensorMap *maps_a, const CUtensorMap *maps_b, const LinearParams *jobs) {
    const LinearParams &p = jobs[0];                        // (tiles and stages are those of both)
    extern __shared__ unsigned char raw_smem[];
    __shared__ PairCtl ctl_space;
    PairCtl *const ctl = &ctl_space;
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const uint32_t cluster = cluster_rank(), rank = cluster & 1, first_cta = cluster & ~1u, part = cluster >> 1;
    const int pair = blockIdx.x / (2 * SPLIT), pairs = gridDim.x / (2 * SPLIT);
    const uint32_t smem = (smem_at(raw_smem) + 1023) & ~1023u, block_bytes = kABytes + p.b_bytes, stage_bytes = DEPTH * block_bytes;
    const int half_n = p.tile_n >> 1;
    const auto step0 = [&](const LinearParams &q) { return SPLIT == 1 ? 0 : (int)(part * (uint32_t)q.kb) / SPLIT; };
    const auto step1 = [&](const LinearParams &q) { return SPLIT == 1 ? q.kb : (int)((part + 1) * (uint32_t)q.kb) / SPLIT; };
    if (tid == 0) {
        for (int s = 0; s < p.stages; ++s) {
            bar_init(&ctl->full[s], 1);
            bar_init(&ctl->empty[s], 1);
        }
        for (int i = 0; i < 2; ++i) {
            bar_init(&ctl->sums_full[i], 1);
            bar_init(&ctl->sums_empty[i], 2 * kEpiThreads / 32);   // the warps of both CTAs
        }
        bar_init(&ctl->never, 1);
        ctl->gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&ctl->tmem)), "r"(p.tmem_cols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    tc_before();
    __syncthreads();
    cluster_sync();                                         // the other CTA's barriers are there before anything signals them
    tc_after();
    const uint32_t tmem = ctl->tmem;
    in_turn();
    const int rows0 = actual_rows(p);
    const auto rows_of = [&](int job) { return JOBS == 2 && job ? jobs[1].n : rows0; };
    const auto row_tiles_of = [&](int job) { return (rows_of(job) + 2 * kM - 1) / (2 * kM); };
    TileWalk<JOBS> walk = {pair, pairs, {row_tiles_of(0) * p.m_tiles, JOBS == 2 ? row_tiles_of(1) * jobs[JOBS - 1].m_tiles : 0}};
    walk.late = walk.tiles[0] % pairs;
    walk.early = p.early;
    if (p.wait_limit < kShortLimit && tid == 0) bar_wait(&ctl->never, 0, ctl, p.wait_limit);
    uint32_t stage = 0, phase = 0;                          // of the loader, of the products
    const auto next_stage = [&] {
        if (++stage == (uint32_t)p.stages) {
            stage = 0;
            phase ^= 1;
        }
    };
    if (warp == 8) {
        int issued = 0;                                     // (up to the number of stages)
        bool ok = true;
        for (TileWalk<JOBS> w = walk; ok && w.next();) {
            const LinearParams &q = jobs[w.job];
            const CUtensorMap *const map_a = maps_a + w.job, *const map_b = maps_b + w.job;
            const bool b_mn = B_MN != (w.job != 0);
            int rt, ct;
            tile_place(w.t, row_tiles_of(w.job), q.m_tiles, rt, ct);
            const int r0 = rt * 2 * kM + (int)rank * kM, c0 = ct * p.tile_n + (int)rank * half_n;
            for (int kb = step0(q); kb < step1(q); ++kb) {
                ok = warp_wait(&ctl->empty[stage], phase ^ 1, ctl, p.wait_limit);
                if (!ok) break;
                if (elect_one()) {
                    if (rank == 0) bar_expect(&ctl->full[stage], 2u * stage_bytes);
                    const uint32_t bar = map_to_rank(smem_at(&ctl->full[stage]), first_cta);
#pragma unroll
                    for (int i = 0; i < DEPTH; ++i) {
                        const uint32_t a = smem + stage * stage_bytes + i * block_bytes, b = a + kABytes;
                        const int k = (kb * DEPTH + i) * kKb;
                        if (b_mn) {
                            load_box_pair(a, map_b, bar, r0, k);
                            load_box_pair(a + 8192, map_b, bar, r0 + 64, k);
                        } else {
                            load_box_pair(a, map_b, bar, k, r0);
                        }
                        if (A_MN)
                            for (int c = 0; c < half_n; c += 64) load_box_pair(b + c * 128, map_a, bar, c0 + c, k);
                        else
                            load_box_pair(b, map_a, bar, k, c0);
                    }
                }
                __syncwarp();
                issued = min(issued + 1, p.stages);
                next_stage();
            }
        }
        // The copies of both CTAs that were started land first, which the first CTA's barriers count.  After a wait that ran out one CTA may have
        // started copies that the other has no part in: 10 ms for those.
        if (rank == 0) {
            for (; issued > 0; --issued) {
                if (stage == 0) {
                    stage = p.stages;
                    phase ^= 1;
                }
                bar_drain(&ctl->full[--stage], phase, ctl);
            }
        }
        if (!ok || ctl->gave_up) {
            const long long t0 = clock64();
            while (clock64() - t0 < kDrainLimit / 10) {}
        }
    } else if (warp == 9) {
        if (rank == 0) {
            uint32_t buf = 0, buf_phase = 0;
            bool ok = true;
            for (TileWalk<JOBS> w = walk; ok && w.next();) {
                const int steps = step1(jobs[w.job]), piece = kPieceOf<F32> / DEPTH;             // steps of an accumulator
                const uint32_t idesc = instruction(2 * kM, p.tile_n, B_MN != (w.job != 0), A_MN);
                for (int kb = step0(jobs[w.job]); kb < steps && ok;) {
                    ok = warp_wait(&ctl->sums_empty[buf], buf_phase ^ 1, ctl, p.wait_limit);
                    if (!ok) break;
                    tc_after();
                    const uint32_t d = tmem + buf * p.tile_n;
                    const int end = min(kb + piece, steps);
                    for (uint32_t more = 0; kb < end; ++kb, more = 1) {
                        ok = warp_wait(&ctl->full[stage], phase, ctl, p.wait_limit);
                        if (!ok) break;
                        tc_after();
                        if (elect_one()) {
#pragma unroll
                            for (int i = 0; i < DEPTH; ++i) {
                                const uint32_t at = smem + stage * stage_bytes + i * block_bytes;
                                if (JOBS == 2 && w.job) mma_block<true, !B_MN, A_MN>(d, operand<!B_MN>(at), operand<A_MN>(at + kABytes), idesc, i ? 1u : more);
                                else mma_block<true, B_MN, A_MN>(d, operand<B_MN>(at), operand<A_MN>(at + kABytes), idesc, i ? 1u : more);
                            }
                            tc_commit_pair(&ctl->empty[stage], first_cta);
                        }
                        __syncwarp();
                        next_stage();
                    }
                    if (ok) {
                        if (elect_one()) tc_commit_pair(&ctl->sums_full[buf], first_cta);
                        __syncwarp();
                        buf ^= 1;
                        if (buf == 0) buf_phase ^= 1;
                    }
                }
            }
            if (!ok) {                                      // no product is on its way when TMEM is freed
                if (elect_one()) tc_commit_pair(&ctl->never, first_cta);
                __syncwarp();
                const long long t0 = clock64();
                while (clock64() - t0 < kDrainLimit / 10) {}
            }
        }
    } else if constexpr (SPLIT == 1) {
        // ---- sums on their way out: warp w reads TMEM lanes 32 (w mod 4) .., and half of the tile's columns ----
        const int first = (warp >> 2) * half_n, my_row = (int)rank * kM + (warp & 3) * 32 + lane;
        const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + first;
        uint32_t buf = 0, buf_phase = 0;
        bool ok = true;
        for (TileWalk<JOBS> w = walk; ok && w.next();) {
            const LinearParams &q = jobs[w.job];
            const int rows = rows_of(w.job);
            int rt, ct;
            tile_place(w.t, row_tiles_of(w.job), q.m_tiles, rt, ct);
            const int row = rt * 2 * kM + my_row, n = row < rows ? row : -1, to = row_of(q, row, rows), c0 = ct * p.tile_n + first;
            const int cols = min(half_n, q.m - c0);
            const float *bias = nullptr;
            if (q.bias) {
                __syncwarp();
                for (int c = lane; c < cols; c += 32) ctl->bias[warp][c] = q.bias[c0 + c];
                __syncwarp();
                bias = ctl->bias[warp];
            }
            const uint32_t turn = smem_at(ctl->turn[warp]);
            const bool add = q.residual != nullptr;
            if constexpr (F32) {
                float sum[kMaxPairN32 / 2] = {};
                for (int kb = 0; kb < q.kb && ok; kb += kPiece / DEPTH) {
                    ok = warp_wait(&ctl->sums_full[buf], buf_phase, ctl, p.wait_limit);
                    tc_after();
                    // (a load from TMEM ahead of the sums)
                    uint32_t v[2][16];
                    tmem_load(at + buf * p.tile_n, v[0]);
#pragma unroll
                    for (int c = 0; c < kMaxPairN32 / 2; c += 16) {
                        uint32_t (&now)[16] = v[c / 16 & 1], (&next)[16] = v[c / 16 + 1 & 1];
                        tmem_wait(now);
                        if (c + 16 < kMaxPairN32 / 2 && c + 16 < half_n) tmem_load(at + buf * p.tile_n + c + 16, next);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c + i] += __uint_as_float(now[i]);
                    }
                    tc_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(map_to_rank(smem_at(&ctl->sums_empty[buf]), first_cta));
                    buf ^= 1;
                    if (buf == 0) buf_phase ^= 1;
                }
#pragma unroll
                for (int c = 0; c < kMaxPairN32 / 2; c += 16)
                    if (c < cols) {
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) v[i] = sum[c + i];
                        finish_row<true, ACT>(q, v, c0 + c, n, to, bias ? bias + c : nullptr, add, turn);
                    }
            } else {
                ok = warp_wait(&ctl->sums_full[buf], buf_phase, ctl, p.wait_limit);
                tc_after();
                for (int kb = kHalfPiece / DEPTH; kb < q.kb && ok; kb += kHalfPiece / DEPTH) {
                    const uint32_t old = buf;
                    next_buffer(buf, buf_phase);
                    ok = warp_wait(&ctl->sums_full[buf], buf_phase, ctl, p.wait_limit);
                    tc_after();
                    join_pieces(at + old * p.tile_n, at + buf * p.tile_n, 0, cols, 16);
                    if (lane == 0) bar_arrive_cluster(map_to_rank(smem_at(&ctl->sums_empty[old]), first_cta));
                }
#pragma unroll 1
                for (int c = 0; c < cols; c += 32) {
                    uint32_t s0[16], s1[16];
                    tmem_load(at + buf * p.tile_n + c, s0);
                    tmem_load(at + buf * p.tile_n + c + 16, s1);
                    tmem_wait(s0);
                    tmem_wait(s1);
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        v[i] = __uint_as_float(s0[i]);
                        v[16 + i] = __uint_as_float(s1[i]);
                    }
                    finish_row<false, ACT>(q, v, c0 + c, n, to, bias ? bias + c : nullptr, add, turn);
                }
                tc_before();
                __syncwarp();
                if (lane == 0) bar_arrive_cluster(map_to_rank(smem_at(&ctl->sums_empty[buf]), first_cta));
                buf ^= 1;
                if (buf == 0) buf_phase ^= 1;
            }
        }
    }
    if constexpr (SPLIT == 2) {
        // As above, but of the columns that a warp has, it sends half to its like in the other pair, to where the stages were, and adds what
        // comes from there to the other half.
        float sum[F32 ? kMaxPairN32 / 2 : 1] = {};
        const int first = (warp >> 2) * half_n, my_row = (int)rank * kM + (warp & 3) * 32 + lane, mine = half_n / 2, keep = (int)part * mine;
        const int send = mine - keep;
        const uint32_t at = tmem + ((uint32_t)((warp & 3) * 32) << 16) + first;
        const bool tile = walk.next();
        uint32_t last_buf = 0;                              // accumulator that holds a bfloat16 result's sum in the end
        if (warp < 8 && tile) {
            if constexpr (F32) {
                uint32_t buf = 0, buf_phase = 0;
                for (int kb = step0(p); kb < step1(p); kb += kPiece / DEPTH) {
                    if (!warp_wait(&ctl->sums_full[buf], buf_phase, ctl, p.wait_limit)) break;
                    tc_after();
                    uint32_t v[2][16];
                    tmem_load(at + buf * p.tile_n, v[0]);
#pragma unroll
                    for (int c = 0; c < kMaxPairN32 / 2; c += 16) {
                        uint32_t (&now)[16] = v[c / 16 & 1], (&next)[16] = v[c / 16 + 1 & 1];
                        tmem_wait(now);
                        if (c + 16 < kMaxPairN32 / 2 && c + 16 < half_n) tmem_load(at + buf * p.tile_n + c + 16, next);
#pragma unroll
                        for (int i = 0; i < 16; ++i) sum[c + i] += __uint_as_float(now[i]);
                    }
                    tc_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive_cluster(map_to_rank(smem_at(&ctl->sums_empty[buf]), first_cta));
                    buf ^= 1;
                    if (buf == 0) buf_phase ^= 1;
                }
            } else {
                bool ok = warp_wait(&ctl->sums_full[0], 0, ctl, p.wait_limit);
                tc_after();
                uint32_t buf_phase = 0;
                for (int kb = step0(p) + kHalfPiece / DEPTH; kb < step1(p) && ok; kb += kHalfPiece / DEPTH) {
                    const uint32_t old = last_buf;
                    next_buffer(last_buf, buf_phase);
                    ok = warp_wait(&ctl->sums_full[last_buf], buf_phase, ctl, p.wait_limit);
                    tc_after();
                    join_pieces(at + old * p.tile_n, at + last_buf * p.tile_n, 0, half_n, 16);
                    if (lane == 0) bar_arrive_cluster(map_to_rank(smem_at(&ctl->sums_empty[old]), first_cta));
                }
            }
        }
        __syncwarp();
        cluster_sync();                                     // no product reads the stages any more, in either pair
        const uint32_t box = smem + (uint32_t)(warp * mine * 32 + lane * 4) * 4;            // [8 warps][mine / 4][32 rows][4]
        if (warp < 8 && tile) {
            const uint32_t there = map_to_rank(box, cluster ^ 2);
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < kMaxPairN32 / 2; c += 16)
                    if (c >= send && c < send + mine)
#pragma unroll
                        for (int i = 0; i < 16; i += 4) cluster_store4(there + (uint32_t)(c + i - send) * 128, reinterpret_cast<const uint32_t *>(sum + c + i));
            } else {
#pragma unroll 1
                for (int c = 0; c < mine; c += 16) {
                    uint32_t v[16];
                    tmem_load(at + last_buf * p.tile_n + send + c, v);
                    tmem_wait(v);
#pragma unroll
                    for (int i = 0; i < 16; i += 4) cluster_store4(there + (uint32_t)(c + i) * 128, v + i);
                }
            }
        }
        __syncwarp();
        cluster_sync();
        if (warp < 8 && tile) {
            int rt, ct;
            tile_place(walk.t, row_tiles_of(0), p.m_tiles, rt, ct);
            const int row = rt * 2 * kM + my_row, n = row < rows0 ? row : -1, to = row_of(p, row, rows0), c0 = ct * p.tile_n + first + keep;
            const int cols = min(mine, p.m - c0);
            if (p.bias) {
                for (int c = lane; c < cols; c += 32) ctl->bias[warp][c] = p.bias[c0 + c];
                __syncwarp();
            }
            const uint32_t turn = smem_at(ctl->turn[warp]);
            const bool add = p.residual != nullptr;
            const auto from_other = [&](int c) {
                const uint4 x = shared_load4(box + (uint32_t)c * 128);
                return make_float4(__uint_as_float(x.x), __uint_as_float(x.y), __uint_as_float(x.z), __uint_as_float(x.w));
            };
            if constexpr (F32) {
#pragma unroll
                for (int c = 0; c < kMaxPairN32 / 2; c += 16)
                    if (c >= keep && c < keep + cols) {
                        float v[16];
#pragma unroll
                        for (int i = 0; i < 16; i += 4) {
                            const float4 x = from_other(c + i - keep);
                            v[i] = sum[c + i] + x.x; v[i + 1] = sum[c + i + 1] + x.y; v[i + 2] = sum[c + i + 2] + x.z; v[i + 3] = sum[c + i + 3] + x.w;
                        }
                        finish_row<true, ACT>(p, v, c0 + c - keep, n, to, p.bias ? ctl->bias[warp] + c - keep : nullptr, add, turn);
                    }
            } else {
#pragma unroll 1
                for (int c = 0; c < cols; c += 32) {
                    uint32_t s0[16], s1[16];
                    tmem_load(at + last_buf * p.tile_n + keep + c, s0);
                    tmem_load(at + last_buf * p.tile_n + keep + c + 16, s1);
                    tmem_wait(s0);
                    tmem_wait(s1);
                    float v[32];
#pragma unroll
                    for (int i = 0; i < 16; i += 4) {
                        const float4 x = from_other(c + i), y = from_other(c + 16 + i);
                        v[i] = __uint_as_float(s0[i]) + x.x; v[i + 1] = __uint_as_float(s0[i + 1]) + x.y;
                        v[i + 2] = __uint_as_float(s0[i + 2]) + x.z; v[i + 3] = __uint_as_float(s0[i + 3]) + x.w;
                        v[16 + i] = __uint_as_float(s1[i]) + y.x; v[17 + i] = __uint_as_float(s1[i + 1]) + y.y;
                        v[18 + i] = __uint_as_float(s1[i + 2]) + y.z; v[19 + i] = __uint_as_float(s1[i + 3]) + y.w;
                    }
                    finish_row<false, ACT>(p, v, c0 + c, n, to, p.bias ? ctl->bias[warp] + c : nullptr, add, turn);
                }
            }
        }
    }
    __syncwarp();
    tc_before();
    __syncthreads();
    cluster_sync();                                         // neither leaves before the other's products and signals are over
    if (warp == 0) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(p.tmem_cols) : "memory");
    }
}

template <bool F32, int ACT, bool A_MN, bool B_MN, int DEPTH, int SPLIT>
__global__ void __launch_bounds__(kThreads, 1) linear_pair_kernel(const __grid_constant__ CUtensorMap map_a,
                                                                  const __grid_constant__ CUtensorMap map_b,
                                                                  const __grid_constant__ LinearParams p) {
    linear_pair<F32, ACT, A_MN, B_MN, DEPTH, 1, SPLIT>(&map_a, &map_b, &p);
}

// Both gradients, the one with the longer reduction first (ROWS_MN: that of the weights).
struct LinearTwo {
    CUtensorMap a[2], b[2];
    LinearParams p[2];
};
template <bool ROWS_MN, int DEPTH>
__global__ void __launch_bounds__(kThreads, 1) linear_two_kernel(const __grid_constant__ LinearTwo two) {
    linear_pair<false, FI_ACT_NONE, true, ROWS_MN, DEPTH, 2, 1>(two.a, two.b, two.p);
}

// dz = dy act'(preact), and dbias, the sums of its columns (of dy itself without an activation: nothing else is stored then).  A CTA takes 64
// (where there are few, 16) columns, eight per thread, and its share of the rows, four of them on their way per thread; the CTAs of a cluster have the same
// columns, whose sums the first one adds up in the order of their ranks.  Bound by the traffic.
// dz is rounded to bfloat16 (2^-8 of it), the type of the tensor cores' other operand; its sums are not.  DY32: dy is float32.
constexpr int kSlopeThreads = 256;

template <int ACT, int kSlopeCols, bool DY32>
__global__ void __launch_bounds__(kSlopeThreads, 4) linear_slope_kernel(const void *dy, long long ld_dy, const __nv_bfloat16 *z, long long ld_z,
                                                                     __nv_bfloat16 *dz, float *dbias, long long rows, int cols) {
    constexpr int kSlopeRows = kSlopeThreads * 8 / kSlopeCols, kSlopeAhead = DY32 ? 2 : 4;      // (64 registers a thread)
    __shared__ float s[kSlopeRows][kSlopeCols + 1], mine[kSlopeCols];
    const int part = threadIdx.x & (kSlopeCols / 8 - 1), group = threadIdx.x / (kSlopeCols / 8);
    const int c = blockIdx.x * kSlopeCols + part * 8;
    float sum[8] = {};
    in_turn();
    if (c < cols)
        for (long long r0 = (long long)blockIdx.y * kSlopeRows * kSlopeAhead + group; r0 < rows; r0 += (long long)gridDim.y * kSlopeRows * kSlopeAhead) {
            uint4 a[kSlopeAhead][DY32 ? 2 : 1], b[kSlopeAhead];
#pragma unroll
            for (int u = 0; u < kSlopeAhead; ++u) {
                const long long r = r0 + u * kSlopeRows;
                a[u][0] = a[u][DY32 ? 1 : 0] = b[u] = make_uint4(0, 0, 0, 0);
                if (r < rows) {
                    const uint4 *const from = reinterpret_cast<const uint4 *>(static_cast<const char *>(dy) + (r * ld_dy + c) * (DY32 ? 4 : 2));
                    a[u][0] = __ldcs(from);
                    if (DY32) a[u][DY32 ? 1 : 0] = __ldcs(from + 1);
                    if (ACT != FI_ACT_NONE) b[u] = __ldcs(reinterpret_cast<const uint4 *>(z + r * ld_z + c));
                }
            }
#pragma unroll
            for (int u = 0; u < kSlopeAhead; ++u) {
                const long long r = r0 + u * kSlopeRows;
                const uint4 &more = a[u][DY32 ? 1 : 0];
                const uint32_t aw[8] = {a[u][0].x, a[u][0].y, a[u][0].z, a[u][0].w, more.x, more.y, more.z, more.w}, bw[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
                uint32_t o[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float lo = __uint_as_float(DY32 ? aw[2 * i] : aw[i] << 16), hi = __uint_as_float(DY32 ? aw[2 * i + 1] : aw[i] & 0xffff0000u);
                    float lo_slope = __uint_as_float(bw[i] << 16), hi_slope = __uint_as_float(bw[i] & 0xffff0000u);
                    slopes<ACT>(lo_slope, hi_slope);
                    lo *= lo_slope;
                    hi *= hi_slope;
                    sum[2 * i] += lo;
                    sum[2 * i + 1] += hi;
                    o[i] = pack2(lo, hi);
                }
                if (dz && r < rows) *reinterpret_cast<uint4 *>(dz + r * cols + c) = make_uint4(o[0], o[1], o[2], o[3]);
            }
        }
    if (!dbias) return;
#pragma unroll
    for (int i = 0; i < 8; ++i) s[group][part * 8 + i] = sum[i];
    __syncthreads();
    if (threadIdx.x < kSlopeCols) {
        float total = 0.f;
#pragma unroll 8
        for (int g = 0; g < kSlopeRows; ++g) total += s[g][threadIdx.x];
        mine[threadIdx.x] = total;
    }
    cluster_sync();
    if (blockIdx.y == 0 && threadIdx.x < kSlopeCols && blockIdx.x * kSlopeCols + threadIdx.x < (unsigned)cols) {
        float total = 0.f;
        for (unsigned i = 0; i < gridDim.y; ++i) {
            float v;
            asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(map_to_rank(smem_at(mine + threadIdx.x), i)) : "memory");
            total += v;
        }
        dbias[blockIdx.x * kSlopeCols + threadIdx.x] = total;
    }
    cluster_sync();                                         // the first CTA has read the others' sums
}

// ------------------------------------------------------------------------------------------------------------- host

using LinearKernel = void (*)(CUtensorMap, CUtensorMap, LinearParams);

// see in_turn
template <typename... Params, typename... Args>
fi_status_t launch_early(const char *name, void (*kernel)(Params...), dim3 grid, int threads, int smem, dim3 cluster, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cluster.x;
    attr[0].val.clusterDim.y = cluster.y;
    attr[0].val.clusterDim.z = cluster.z;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = (size_t)smem;
    cfg.stream = stream;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
    if (e != cudaSuccess) return cuda_fail(e, name);
    count_launch();
    return check_launch(name);
}

// forward products in all their forms; gradients have no activation and bfloat16 results.  PAIRS: that have a tile together, 0: single CTAs,
// -1: single CTAs with long sums
template <int PAIRS, int DEPTH, bool F32, int ACT, bool A_MN, bool B_MN>
constexpr LinearKernel linear_kernel_of() {
    if constexpr (PAIRS <= 0) return &linear_split_kernel<F32, ACT, A_MN, B_MN, DEPTH, PAIRS < 0>;
    else return &linear_pair_kernel<F32, ACT, A_MN, B_MN, DEPTH, PAIRS>;
}

template <int PAIRS, int DEPTH, bool F32>
LinearKernel forward_kernel(int act) {
    switch (act) {
        case FI_ACT_RELU: return linear_kernel_of<PAIRS, DEPTH, F32, FI_ACT_RELU, false, false>();
        case FI_ACT_GELU: return linear_kernel_of<PAIRS, DEPTH, F32, FI_ACT_GELU, false, false>();
        case FI_ACT_GELU_TANH: return linear_kernel_of<PAIRS, DEPTH, F32, FI_ACT_GELU_TANH, false, false>();
        case FI_ACT_SILU: return linear_kernel_of<PAIRS, DEPTH, F32, FI_ACT_SILU, false, false>();
        default: return linear_kernel_of<PAIRS, DEPTH, F32, FI_ACT_NONE, false, false>();
    }
}
template <int PAIRS, int DEPTH>
LinearKernel linear_kernel(bool f32, int act, bool a_mn, bool b_mn) {
    if (a_mn) return b_mn ? linear_kernel_of<PAIRS, DEPTH, false, FI_ACT_NONE, true, true>() : linear_kernel_of<PAIRS, DEPTH, false, FI_ACT_NONE, true, false>();
    return f32 ? forward_kernel<PAIRS, DEPTH, true>(act) : forward_kernel<PAIRS, DEPTH, false>(act);
}
LinearKernel linear_kernel(int pairs, int depth, bool f32, int act, bool a_mn, bool b_mn) {
    if (pairs == 2) return depth == 2 ? linear_kernel<2, 2>(f32, act, a_mn, b_mn) : linear_kernel<2, 1>(f32, act, a_mn, b_mn);
    if (pairs == 1) return depth == 2 ? linear_kernel<1, 2>(f32, act, a_mn, b_mn) : linear_kernel<1, 1>(f32, act, a_mn, b_mn);
    if (pairs == 0) return depth == 2 ? linear_kernel<0, 2>(f32, act, a_mn, b_mn) : linear_kernel<0, 1>(f32, act, a_mn, b_mn);
    return depth == 2 ? linear_kernel<-1, 2>(f32, act, a_mn, b_mn) : linear_kernel<-1, 1>(f32, act, a_mn, b_mn);
}

using TwoKernel = void (*)(LinearTwo);
TwoKernel two_kernel(bool rows_mn, int depth) {
    if (rows_mn) return depth == 2 ? linear_two_kernel<true, 2> : linear_two_kernel<true, 1>;
    return depth == 2 ? linear_two_kernel<false, 2> : linear_two_kernel<false, 1>;
}

struct DeviceFacts {
    int clusters[4];                                        // of 1, 2, 4, 8 CTAs that run at one time
};
std::atomic<unsigned long long> g_facts[kMaxDevices];       // 16 bits each, published in one piece; 0: not known yet

// Facts of the current device; its kernels are set up at the first call
fi_status_t device_facts(DeviceFacts &f, const char *name) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, name);
    if (dev < 0 || dev >= kMaxDevices) {
        set_error("%s: device ordinal %d", name, dev);
        return FI_ERR_UNSUPPORTED;
    }
    if (const unsigned long long known = g_facts[dev].load(std::memory_order_acquire)) {
        for (int i = 0; i < 4; ++i) f.clusters[i] = (int)(known >> (16 * i) & 0xffff);
        return FI_OK;
    }
    int n = 0;
    e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
    for (int form = 0; form < 12; ++form) {                 // of a product: type and activation, or one of two gradients
        const bool back = form >= 10, f32 = !back && form >= 5;
        for (int i = 0; i < 8 && e == cudaSuccess; ++i)
            e = cudaFuncSetAttribute(reinterpret_cast<const void *>(linear_kernel((i >> 1) - 1, 1 + (i & 1), f32, form % 5, back, form == 11)),
                                     cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemMost - kStaticMost);
    }
    for (int i = 0; i < 4 && e == cudaSuccess; ++i)
        e = cudaFuncSetAttribute(reinterpret_cast<const void *>(two_kernel(i & 1, 1 + (i >> 1))), cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kSmemMost - kStaticMost);
    f.clusters[0] = n;
    for (int i = 1; i < 4 && e == cudaSuccess; ++i) {
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << i;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1u << i);
        cfg.blockDim = dim3(kThreads);
        cfg.dynamicSmemBytes = kSmemMost - kStaticMost;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&f.clusters[i], linear_kernel(i == 1, 1, false, FI_ACT_NONE, false, false), &cfg);
        if (e == cudaSuccess && f.clusters[i] < 1) e = cudaErrorInvalidConfiguration;
    }
    if (e != cudaSuccess) return cuda_fail(e, name);
    unsigned long long known = 0;
    for (int i = 0; i < 4; ++i) known |= (unsigned long long)f.clusters[i] << (16 * i);
    g_facts[dev].store(known, std::memory_order_release);   // (threads that come here together find the same)
    return FI_OK;
}

// one operand: `rows` lines of `dim` contiguous values
struct Matrix {
    const void *base;
    long long rows, dim, ld;
};

fi_status_t operand_map(CUtensorMap *map, const Matrix &x, int box_rows, const char *name) {
    static std::atomic<void *> entry{nullptr};
    void *fn = entry.load(std::memory_order_acquire);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess) {
            set_error("%s: cuTensorMapEncodeTiled is not available from this driver", name);
            return FI_ERR_UNSUPPORTED;
        }
        entry.store(fn, std::memory_order_release);
    }
    const cuuint64_t size[2] = {(cuuint64_t)x.dim, (cuuint64_t)x.rows}, stride[1] = {(cuuint64_t)(x.rows > 1 ? x.ld : (x.dim + 7) / 8 * 8) * 2};
    const cuuint32_t box[2] = {kKb, (cuuint32_t)box_rows}, step[2] = {1, 1};
    const CUresult r = reinterpret_cast<decltype(&cuTensorMapEncodeTiled)>(fn)(
        map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void *>(x.base), size, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
        CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) {
        set_error("%s: cuTensorMapEncodeTiled failed with code %d (%lld x %lld values, %lld apart)", name, (int)r, x.rows, x.dim, x.ld);
        return FI_ERR_CUDA;
    }
    return FI_OK;
}

// Which kernel, and its tiles: the one with the least estimated cycles.  The tensor cores take 16 x 256 x 256 products of a pair in 128 cycles (a
// CTA's 16 x 128 x 256 in as many), an SM gets 80 bytes a cycle from L2 where pairs ask for them and 55 where single CTAs do, all together
// 8,600, and the device 5,000 from memory and what L2 still has; a tile's way out is hidden behind the next one of a pair, but for a fifth
// of it.  These figures and the ways out are fitted to the times of 212 products in all their forms (1 to 8,192 tokens, 80 to 8,192 values,
// both types): what is taken is 0.9 % slower than the best form of each in the mean, 16 % at most.  (Both sides, us: 777 x 512 -> 2,048:
// pairs of 128 columns 6.3, CTAs with 96 tokens 8.8; 32 x 4,096 -> 4,096: clusters of 4 9.5, single CTAs 11.3; 4,000 x 768 <- 768: pairs
// 9.3, CTAs 14.2; 200 x 8,192 -> 2,048 in float32: clusters of 4 18.4, pairs 25.3; two pairs a tile against the best of the others:
// 256 x 4,096 -> 4,096 in float32 16.4 and 17.9, 1,000 x 8,192 -> 1,024 19.1 and 21.8, 256 x 14,336 -> 4,096 31.5 and 35.5.)
struct LinearPlan {
    bool pair;
    int tile_n, split;
    double cycles;
};

double most(double a, double b) { return a > b ? a : b; }
long long up(long long a, long long b) { return (a + b - 1) / b; }
// the same of whole numbers below 2^53, without the long division of whole numbers (a plan has some hundred of them)
double times(double a, double b) {
    const double q = a / b;
    const long long i = (long long)q;
    return (double)(i + ((double)i * b < a));
}

// what a product of m columns, n rows and kb blocks has to move, in cycles: from memory, and from L2 in tiles
double memory_cycles(double m, double n, double kb, int size) { return ((m + n) * kb * (kKb * 2) + m * n * size) / 5000.; }
double tile_traffic(double m, double n, double kb, double m_tiles, double n_tiles) { return (m_tiles * n + n_tiles * m) * kb * (kKb * 2) / 8600.; }

struct PairCost {
    double tiles, each, least, end;                         // a tile's cycles; what the traffic takes at least; the last way out
};
PairCost pair_cost(long long m, long long n, long long kb, int tile, bool f32, int size) {
    const double m_tiles = times((double)m, tile), n_tiles = (double)up(n, 2 * kM), end = 2500 + (f32 ? 20. : 12.) * tile;
    const double each = most(kb * most(2. * tile, (128 + tile / 2) * 128 / 80.), 0.8 * end);
    return {m_tiles * n_tiles, each, most(memory_cycles((double)m, (double)n, (double)kb, size), tile_traffic((double)m, (double)n, (double)kb, m_tiles, n_tiles)), end};
}

LinearPlan plan_product(long long m, long long n, long long kb, bool a_mn, bool f32, int size, const int *clusters) {
    LinearPlan best = {false, 16, 1, 1e30};
    for (int tile = 64; tile <= kMaxN; tile += 64) {          // (a warp takes 32 columns of a half at a time)
        if ((a_mn && tile % 128) || (f32 && tile > kMaxPairN32)) continue;
        const PairCost c = pair_cost(m, n, kb, tile, f32, size);
        const double cycles = most(times(c.tiles, clusters[1]) * c.each, c.least) + c.end;
        if (cycles < best.cycles) best = {true, tile, 1, cycles};
        // two pairs a tile; what a warp has of the columns is halved, 16 (in bfloat16 32) of them go out together
        if (kb < 16 || tile % (f32 ? 64 : 128)) continue;
        const double split = most(times(c.tiles, clusters[2]) * (0.5 * c.each + c.end), c.least) + c.end + 3000;
        if (split < best.cycles) best = {true, tile, 2, split};
    }
    const double memory = memory_cycles((double)m, (double)n, (double)kb, size), weights = (double)m * kb * (kKb * 2), m_tiles = (double)up(m, kM);
    for (int tile = 16; tile <= kMaxN; tile += 16) {
        if (tile > 16 && tile - 16 >= n) break;
        const double n_tiles = times((double)n, tile), block = most(2. * tile, (128 + tile) * 128 / 55.);
        // columns' operand (weights) that L2 does not hold is read again for every tile of rows
        const double again = weights > 64e6 ? (n_tiles - 1) * weights / 3400. : 0;
        const double least = most(memory + again, tile_traffic((double)m, (double)n, (double)kb, m_tiles, n_tiles));
        for (int i = 0; i < 4 && 1 << i <= kb; ++i) {
            const long long blocks = (kb + (1 << i) - 1) >> i;
            if (f32 && (blocks + kPiece - 1) / kPiece * tile > 512 && tile > 16) continue;   // pieces of 512 values have an accumulator each
            const double rounds = times(m_tiles * n_tiles, clusters[i]), end = i ? 2800 + 40. * tile : 6000 + 20. * tile;
            const double cycles = most(rounds * ((double)blocks * block + end) - end, least) + end;
            if (cycles < best.cycles) best = {false, tile, 1 << i, cycles};
        }
    }
    return best;
}

// two blocks a stage where the products of one are over before the next is issued (430 cycles: 16 x 256 x 128 take 64)
int stage_blocks(const LinearPlan &plan, long long kb) { return plan.tile_n <= 128 && kb > 1 ? 2 : 1; }

// Both gradients (m columns each) as two launches, or in one by pairs with tiles of one size, which share the SMs without a gap between them.
// (777 tokens, 1,000 -> 1,400: 13.1 us together, one after the other 20.1 as pairs and 22.)
void plan_two(long long m, long long n0, long long kb0, long long n1, long long kb1, const int *clusters, LinearPlan &x, LinearPlan &y) {
    x = plan_product(m, n0, kb0, true, false, 2, clusters);
    y = plan_product(m, n1, kb1, true, false, 2, clusters);
    double least = x.cycles + y.cycles;
    for (int tile = 128; tile <= kMaxN; tile += 128) {
        const PairCost a = pair_cost(m, n0, kb0, tile, false, 2), b = pair_cost(m, n1, kb1, tile, false, 2);
        const double work = most((a.tiles * a.each + b.tiles * b.each) / clusters[1], most(a.each, b.each)), cycles = most(work, a.least + b.least) + a.end;
        const LinearPlan plan = {true, tile, 1, cycles};
        if (cycles < least && stage_blocks(plan, kb0) == stage_blocks(plan, kb1)) {
            least = cycles;
            x = y = plan;
        }
    }
}

// A product that is ready to be launched
struct Product {
    CUtensorMap map_a, map_b;
    LinearParams p;
    LinearPlan plan;
    long long tiles;
    int depth, smem;
};

// D[n][m] = sum over k of A(m, k) B(n, k); x.p holds what becomes of the sums
fi_status_t plan_launch(Product &x, const LinearPlan &plan, const Matrix &a, bool a_mn, const Matrix &b, bool b_mn, long long m, long long n, long long k,
                        bool f32, const char *name) {
    LinearParams &p = x.p;
    p.m = (int)m;
    p.n = (int)n;
    p.kb = (int)up(k, kKb);
    const int depth = stage_blocks(plan, p.kb), blocks = p.kb;
    p.kb = (p.kb + depth - 1) / depth;
    p.tile_n = plan.tile_n;
    p.split = plan.split;
    while (p.split > p.kb) p.split /= 2;
    // tiles: of a pair 256 output rows and tile_n columns, of a CTA 128 columns and tile_n rows; the operand of the tile_n ones is the second
    const bool second_mn = plan.pair ? a_mn : b_mn;
    const int mine = plan.pair ? p.tile_n / 2 : p.tile_n;                                   // of them that a CTA loads
    p.m_tiles = (int)(plan.pair ? (m + p.tile_n - 1) / p.tile_n : (m + kM - 1) / kM);
    const long long n_tiles = plan.pair ? (n + 2 * kM - 1) / (2 * kM) : (n + p.tile_n - 1) / p.tile_n, tiles = p.m_tiles * n_tiles;
    p.bufs = 2;
    p.piece = 0;
    if (!plan.pair) {
        const int room = 512 / p.tile_n, pieces = f32 ? ((blocks + p.split - 1) / p.split + depth + kPiece - 1) / kPiece
                                                      : (int)up(up(p.kb, p.split), kHalfPiece / depth);
        // (in float32 a few blocks more a piece where their number is at the limit)
        if (pieces > room + (f32 ? 1 : 0)) {
            p.piece = (f32 ? kPiece : kHalfPiece) / depth;
            p.bufs = room < kRing ? room : kRing;
        } else {
            p.bufs = pieces < room ? pieces : room;
        }
    }
    p.tmem_cols = 32;
    while (p.tmem_cols < p.bufs * p.tile_n) p.tmem_cols *= 2;
    p.b_bytes = second_mn ? (mine + 63) / 64 * 8192 : mine * kKb * 2;
    const int stage = depth * (kABytes + p.b_bytes), room = kSmemMost - kStaticMost - 1024 /* alignment */;
    const int part = plan.pair ? 0 : p.split * ((p.tile_n / 4 + p.split - 1) / p.split) * kM * 16;
    const bool apart = !plan.pair && p.split > 1 && p.tile_n <= 64;
    p.stages = (room - (apart ? part : 0)) / stage;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    p.part_at = apart ? p.stages * stage : 0;
    int smem = p.stages * stage + (apart ? part : 0);
    if (smem < part) smem = part;
    smem += 1024;
    if (tiles * p.split * 2 > 1073741823ll) {
        set_error("%s: too many tiles", name);
        return FI_ERR_INVALID_ARG;
    }
    fi_status_t st = operand_map(&x.map_a, a, a_mn ? kKb : plan.pair ? mine : kM, name);
    if (st == FI_OK) st = operand_map(&x.map_b, b, b_mn ? kKb : plan.pair ? kM : mine, name);
    x.plan = plan;
    x.tiles = tiles;
    x.depth = depth;
    x.smem = smem;
    return st;
}

fi_status_t launch_planned(const Product &x, bool a_mn, bool b_mn, bool f32, int act, const DeviceFacts &facts, cudaStream_t stream, const char *name) {
    const int pairs = x.plan.pair ? x.p.split : x.p.piece ? -1 : 0, cluster = pairs > 0 ? 2 * pairs : x.p.split;
    const long long ctas = pairs == 1 ? 2 * (x.tiles < facts.clusters[1] ? x.tiles : facts.clusters[1]) : x.tiles * cluster;
    return launch_early(name, linear_kernel(pairs, x.depth, f32, act, a_mn, b_mn), dim3((unsigned)ctas), kThreads, x.smem, dim3(cluster), stream, x.map_a,
                        x.map_b, x.p);
}

fi_status_t launch_product(const Matrix &a, bool a_mn, const Matrix &b, bool b_mn, long long m, long long n, long long k, bool f32, int act,
                           const LinearParams &what, const DeviceFacts &facts, cudaStream_t stream, const char *name) {
    Product x;
    x.p = what;
    const LinearPlan plan = plan_product(m, n, up(k, kKb), a_mn, f32, f32 ? 4 : 2, facts.clusters);
    const fi_status_t st = plan_launch(x, plan, a, a_mn, b, b_mn, m, n, k, f32, name);
    return st == FI_OK ? launch_planned(x, a_mn, b_mn, f32, act, facts, stream, name) : st;
}

// Two products of pairs in one launch, the one with the longer reduction first; their tiles and stages are the same.
fi_status_t launch_two(const Product &x, const Product &y, bool rows_mn, const DeviceFacts &facts, cudaStream_t stream, const char *name) {
    LinearTwo two;
    two.a[0] = x.map_a;
    two.a[1] = y.map_a;
    two.b[0] = x.map_b;
    two.b[1] = y.map_b;
    two.p[0] = x.p;
    two.p[1] = y.p;
    two.p[0].early = (x.p.kb + y.p.kb / 2) / y.p.kb;
    const long long tiles = x.tiles + y.tiles;
    return launch_early(name, two_kernel(rows_mn, x.depth), dim3((unsigned)(2 * (tiles < facts.clusters[1] ? tiles : facts.clusters[1]))), kThreads, x.smem,
                        dim3(2), stream, two);
}

constexpr long long kMostRows = 1 << 30;                    // (rows are indexed with int32, tiles may overshoot)

long long wait_limit_of(long long given) { return given > 0 && given < kWaitLimit ? given : kWaitLimit; }

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

fi_status_t check_sizes(long long tokens, int in_dim, int out_dim, int act, const char *name) {
    if (tokens < 0 || tokens > kMostRows || in_dim < 8 || in_dim % 8 || in_dim > kMostRows || out_dim < 8 || out_dim % 8 || out_dim > kMostRows) {
        set_error("%s: in_dim and out_dim must be multiples of 8, and they and tokens at most 2^30 (got %lld tokens, %d -> %d)", name, tokens, in_dim,
                  out_dim);
        return FI_ERR_INVALID_ARG;
    }
    if (act < FI_ACT_NONE || act > FI_ACT_SILU) {
        set_error("%s: unknown activation %d", name, act);
        return FI_ERR_INVALID_ARG;
    }
    return FI_OK;
}

// rows of `dim` values that TMA reads: on 16-byte boundaries, strides below 2^39
bool tma_rows(const void *p, long long rows, long long dim, long long ld) {
    return aligned16(p) && (rows <= 1 || (ld % 8 == 0 && ld >= dim && ld < (1ll << 38)));
}

// CTAs of a cluster, which share the rows of `width` columns: up to eight, as many as run at one time (4,095 x 8,192 behind silu: 41 us,
// 4.9 TB/s; 46 with 1,024 CTAs, 592 of which run together)
int slope_parts(long long tokens, int out_dim, int width, int sms) {
    const long long columns = (out_dim + width - 1) / width;
    int parts = 1;
    while (parts < 8 && tokens > (long long)parts * (kSlopeThreads * 8 / width) && columns * parts * 2 <= 4ll * sms) parts *= 2;
    return parts;
}

template <int WIDTH, bool DY32>
auto slope_kernel(int act) {
    return act == FI_ACT_RELU        ? linear_slope_kernel<FI_ACT_RELU, WIDTH, DY32>
           : act == FI_ACT_GELU      ? linear_slope_kernel<FI_ACT_GELU, WIDTH, DY32>
           : act == FI_ACT_GELU_TANH ? linear_slope_kernel<FI_ACT_GELU_TANH, WIDTH, DY32>
           : act == FI_ACT_SILU      ? linear_slope_kernel<FI_ACT_SILU, WIDTH, DY32>
                                     : linear_slope_kernel<FI_ACT_NONE, WIDTH, DY32>;
}
template <int WIDTH>
auto slope_kernel(int act, bool dy32) {
    return dy32 ? slope_kernel<WIDTH, true>(act) : slope_kernel<WIDTH, false>(act);
}

}  // namespace
}  // namespace fi

using namespace fi;

extern "C" {

fi_status_t fi_linear(const fi_linear_t *a, void *cuda_stream) {
    const char *const name = "fi_linear";
    if (!a) {
        set_error("%s: null argument", name);
        return FI_ERR_INVALID_ARG;
    }
    fi_status_t st = check_sizes(a->tokens, a->in_dim, a->out_dim, a->activation, name);
    if (st != FI_OK) return st;
    if (a->out_dtype != FI_F32 && a->out_dtype != FI_BF16) {
        set_error("%s: out_dtype must be FI_F32 or FI_BF16", name);
        return FI_ERR_INVALID_ARG;
    }
    const bool nowhere = a->rows && a->out_rows == 0;       // (preact is written all the same)
    if (a->tokens == 0 || (nowhere && !a->preact)) return FI_OK;
    if (!a->x || !a->weight || (!a->out && !nowhere)) {
        set_error("%s: null pointer", name);
        return FI_ERR_INVALID_ARG;
    }
    const long long out_rows = a->rows ? a->out_rows : a->tokens;
    const int size = a->out_dtype == FI_F32 ? 4 : 2;
    if (!tma_rows(a->x, a->tokens, a->in_dim, a->x_stride) || !tma_rows(a->weight, a->out_dim, a->in_dim, a->weight_stride)) {
        set_error("%s: rows of x and weight must start on 16-byte boundaries and not overlap", name);
        return FI_ERR_INVALID_ARG;
    }
    if (out_rows < 0 || (out_rows > 1 && (a->out_stride < a->out_dim || (a->residual && a->residual_stride < a->out_dim))) ||
        (a->preact && a->tokens > 1 && a->preact_stride < a->out_dim) || (reinterpret_cast<uintptr_t>(a->out) & (size - 1)) ||
        (reinterpret_cast<uintptr_t>(a->residual) & (size - 1)) || (reinterpret_cast<uintptr_t>(a->preact) & 1) ||
        (reinterpret_cast<uintptr_t>(a->bias) & 3) || a->wait_limit < 0) {
        set_error("%s: rows of out, residual and preact must not overlap; pointers must be aligned to their types", name);
        return FI_ERR_INVALID_ARG;
    }
    DeviceFacts facts;
    st = device_facts(facts, name);
    if (st != FI_OK) return st;
    LinearParams p = {};
    p.bias = a->bias;
    p.residual = a->residual;
    p.out = a->out;
    p.preact = static_cast<__nv_bfloat16 *>(a->preact);
    p.rows = a->rows;
    p.count = a->tokens_dev;
    p.ld_res = a->residual_stride;
    p.ld_out = a->out_stride;
    p.ld_preact = a->preact_stride;
    p.out_rows = out_rows;
    p.wait_limit = wait_limit_of(a->wait_limit);
    const auto wide = [&](const void *at, int64_t ld, long long rows_of, int bytes) { return aligned16(at) && (rows_of <= 1 || ld * bytes % 16 == 0); };
    p.wide = wide(a->out, a->out_stride, out_rows, size) && wide(a->residual, a->residual_stride, out_rows, size) &&
             wide(a->preact, a->preact_stride, a->tokens, 2) && aligned16(a->bias);
    const Matrix w = {a->weight, a->out_dim, a->in_dim, a->weight_stride}, x = {a->x, a->tokens, a->in_dim, a->x_stride};
    return launch_product(w, false, x, false, a->out_dim, a->tokens, a->in_dim, a->out_dtype == FI_F32, a->activation, p, facts,
                          static_cast<cudaStream_t>(cuda_stream), name);
}

int64_t fi_linear_backward_workspace(int64_t tokens, int32_t out_dim, int32_t activation) {
    if (tokens < 0 || tokens > kMostRows || out_dim < 8) return 0;
    return activation != FI_ACT_NONE ? (tokens * out_dim * 2 + 255) / 256 * 256 : 0;
}

fi_status_t fi_linear_backward(const fi_linear_backward_t *a, void *cuda_stream) {
    const char *const name = "fi_linear_backward";
    if (!a) {
        set_error("%s: null argument", name);
        return FI_ERR_INVALID_ARG;
    }
    fi_status_t st = check_sizes(a->tokens, a->in_dim, a->out_dim, a->activation, name);
    if (st != FI_OK) return st;
    const bool slopes = a->activation != FI_ACT_NONE, dy32 = a->dy_f32 != 0, apart = slopes || dy32;      // apart: dz is not dy
    if ((a->tokens > 0 && (!a->dy || (slopes && !a->preact) || (a->dx && !a->weight) || (a->dweight && !a->x))) ||
        (apart && (a->dx || a->dweight) && a->tokens > 0 && !a->workspace)) {
        set_error("%s: null pointer", name);
        return FI_ERR_INVALID_ARG;
    }
    const bool dy_rows = dy32 ? aligned16(a->dy) && (a->tokens <= 1 || (a->dy_stride % 4 == 0 && a->dy_stride >= a->out_dim))
                              : tma_rows(a->dy, a->tokens, a->out_dim, a->dy_stride);
    if (!dy_rows || (slopes && !tma_rows(a->preact, a->tokens, a->out_dim, a->preact_stride)) ||
        (a->dx && !tma_rows(a->weight, a->out_dim, a->in_dim, a->weight_stride)) ||
        (a->dweight && !tma_rows(a->x, a->tokens, a->in_dim, a->x_stride)) || !aligned16(a->workspace)) {
        set_error("%s: rows of x, weight, dy and preact must start on 16-byte boundaries and not overlap", name);
        return FI_ERR_INVALID_ARG;
    }
    if ((a->dx && a->tokens > 1 && a->dx_stride < a->in_dim) || (a->dweight && a->dweight_stride < a->in_dim) ||
        (reinterpret_cast<uintptr_t>(a->dx) & 1) || (reinterpret_cast<uintptr_t>(a->dweight) & 1) || (reinterpret_cast<uintptr_t>(a->dbias) & 3) ||
        a->wait_limit < 0) {
        set_error("%s: rows of dx and dweight must not overlap; pointers must be aligned to their types", name);
        return FI_ERR_INVALID_ARG;
    }
    DeviceFacts facts;
    st = device_facts(facts, name);
    if (st != FI_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    if (a->tokens == 0) {                                   // sums over nothing
        cudaError_t e = cudaSuccess;
        if (a->dweight) e = cudaMemset2DAsync(a->dweight, (size_t)a->dweight_stride * 2, 0, (size_t)a->in_dim * 2, (size_t)a->out_dim, stream);
        if (e == cudaSuccess && a->dbias) e = cudaMemsetAsync(a->dbias, 0, (size_t)a->out_dim * 4, stream);
        return e == cudaSuccess ? FI_OK : cuda_fail(e, name);
    }
    __nv_bfloat16 *const dz = apart && (a->dx || a->dweight) ? static_cast<__nv_bfloat16 *>(a->workspace) : nullptr;
    if (dz || a->dbias) {
        const int width = a->out_dim <= 64 * 16 && a->tokens >= 1024 ? 16 : 64, parts = slope_parts(a->tokens, a->out_dim, width, facts.clusters[0]);
        st = launch_early(name, width == 16 ? slope_kernel<16>(a->activation, dy32) : slope_kernel<64>(a->activation, dy32),
                          dim3((a->out_dim + width - 1) / width, parts), kSlopeThreads, 0, dim3(1, parts), stream, a->dy, (long long)a->dy_stride, static_cast<const __nv_bfloat16 *>(a->preact), (long long)a->preact_stride, dz, a->dbias,
                          (long long)a->tokens, (int)a->out_dim);
        if (st != FI_OK) return st;
    }
    const Matrix g = apart ? Matrix{dz, a->tokens, a->out_dim, a->out_dim} : Matrix{a->dy, a->tokens, a->out_dim, a->dy_stride};
    const Matrix w = {a->weight, a->out_dim, a->in_dim, a->weight_stride}, x = {a->x, a->tokens, a->in_dim, a->x_stride};
    LinearParams dx = {}, dw = {};
    dx.wait_limit = dw.wait_limit = wait_limit_of(a->wait_limit);
    dx.out = a->dx;
    dx.wide = aligned16(a->dx) && (a->tokens <= 1 || a->dx_stride % 8 == 0);
    dx.ld_out = a->dx_stride;
    dx.out_rows = a->tokens;
    dw.out = a->dweight;
    dw.wide = aligned16(a->dweight) && a->dweight_stride % 8 == 0;
    dw.ld_out = a->dweight_stride;
    dw.out_rows = a->out_dim;
    if (a->dx && a->dweight) {
        Product px, pw;
        px.p = dx;
        pw.p = dw;
        LinearPlan plan_x, plan_w;
        plan_two(a->in_dim, a->tokens, up(a->out_dim, kKb), a->out_dim, up(a->tokens, kKb), facts.clusters, plan_x, plan_w);
        st = plan_launch(px, plan_x, w, true, g, false, a->in_dim, a->tokens, a->out_dim, false, name);
        if (st == FI_OK) st = plan_launch(pw, plan_w, x, true, g, true, a->in_dim, a->out_dim, a->tokens, false, name);
        if (st != FI_OK) return st;
        if (plan_x.pair && plan_w.pair && plan_x.split == 1 && plan_w.split == 1 && plan_x.tile_n == plan_w.tile_n && px.depth == pw.depth)
            return px.p.kb >= pw.p.kb ? launch_two(px, pw, false, facts, stream, name) : launch_two(pw, px, true, facts, stream, name);
        st = launch_planned(px, true, false, false, FI_ACT_NONE, facts, stream, name);
        return st == FI_OK ? launch_planned(pw, true, true, false, FI_ACT_NONE, facts, stream, name) : st;
    }
    if (a->dx) st = launch_product(w, true, g, false, a->in_dim, a->tokens, a->out_dim, false, FI_ACT_NONE, dx, facts, stream, name);
    if (st == FI_OK && a->dweight)
        st = launch_product(x, true, g, true, a->in_dim, a->out_dim, a->tokens, false, FI_ACT_NONE, dw, facts, stream, name);
    return st;
}

fi_status_t fi_linear_poll_status(void) {
    int32_t word = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e == cudaSuccess) e = cudaMemcpyFromSymbol(&word, g_linear_status, sizeof word);
    if (e == cudaSuccess && word) {
        const int32_t zero = 0;
        e = cudaMemcpyToSymbol(g_linear_status, &zero, sizeof zero);
    }
    if (e != cudaSuccess) return cuda_fail(e, "fi_linear_poll_status");
    if (word) {
        set_error("fi_linear, fi_linear_backward: a wait inside a kernel ran out; its results are not valid");
        return FI_ERR_TIMEOUT;
    }
    return FI_OK;
}

}  // extern "C"

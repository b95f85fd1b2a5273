// Pages that requests share: forking a request, giving pages back by their owners, bringing used pages together, and copying what
// pages hold.
//
// Only full pages are shared, and only by requests with the same beginning: a page that is still written to has one owner, so neither
// the page tables' step nor the store has to look at owners.  shared[page] counts the owners beyond the first.
#include "fi_pages.cuh"

namespace fi {
namespace {

// see launch_early
__device__ __forceinline__ void in_turn() {
    cudaGridDependencySynchronize();
    cudaTriggerProgrammaticLaunchCompletion();
}

// last i in [0, n) with first[i] <= x, for non-decreasing first[] with first[0] <= x
__device__ __forceinline__ int find_last64(const long long *first, int n, long long x) {
    int lo = 0, hi = n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (first[mid] <= x) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Every CTA forms the sums over all requests for itself (wanted tails, then full pages), the entries of the full pages are dealt out to
// the grid, and the first CTA gives the tails their pages.  Lengths and the free count are committed by the last CTA to finish, so
// they may be updated in place; counts of owners are added up by atomics on whole numbers.
__global__ void __launch_bounds__(kPageThreads) pages_fork_kernel(const fi_pages_fork_t a, int page_shift, int max_blocks, uint32_t *ticket) {
    extern __shared__ long long s_cu[];                       // first full page of each request, all laid end to end
    int *const s_src = reinterpret_cast<int *>(s_cu + a.batch_max), *const s_dst = s_src + a.batch_max;
    __shared__ int s_taken;
    in_turn();
    if (threadIdx.x == 0) s_taken = 0;
    LensCopy copy;
    copy.get(a.lens, a.lens_out, a.rows);
    const int n = actual_count(a.batch_count, a.batch_max);
    const int free_count = min(max(*a.free_count, 0), a.num_pages);
    const int items = (a.batch_max + blockDim.x - 1) / blockDim.x, i0 = threadIdx.x * items;
    const int place = (1 << page_shift) - 1;
    int length[kPageItems], flags[kPageItems];                // flags: 1 possible, 2 needs a page for its tail, 4 granted
    long long need = 0;
#pragma unroll
    for (int e = 0; e < kPageItems; ++e) {
        const int i = i0 + e;
        flags[e] = length[e] = 0;
        if (e < items && i < n) {
            const int src = a.src_rows[i], dst = a.dst_rows[i];
            if (src >= 0 && src < a.rows && dst >= 0 && dst < a.rows && src != dst && a.lens[dst] == 0) {
                length[e] = a.lens[src];
                if (length[e] >= 0 && ((long long)length[e] + place) >> page_shift <= max_blocks) flags[e] = length[e] & place ? 3 : 1;
            }
            s_src[i] = src;
            s_dst[i] = dst;
            need += flags[e] >> 1;
        }
    }
    long long wanted;
    long long before = block_exclusive(need, &wanted);
    long long full = 0;
    int taken = 0;
#pragma unroll
    for (int e = 0; e < kPageItems; ++e) {
        const int i = i0 + e;
        if (e >= items || i >= a.batch_max) continue;
        int page = -1, tail = -1;
        if (i < n) {
            if ((flags[e] & 1) && (!(flags[e] & 2) || before < free_count)) {
                flags[e] |= 4;
                full += length[e] >> page_shift;
            }
            if (flags[e] & 2) {
                if (flags[e] & 4) {
                    page = a.free_pages[free_count - 1 - (int)before];
                    ++taken;
                }
                ++before;
            }
        }
        if (blockIdx.x == 0) {
            if (page >= 0) {
                tail = a.block_table[(long long)s_src[i] * a.table_ld + (length[e] >> page_shift)];
                a.block_table[(long long)s_dst[i] * a.table_ld + (length[e] >> page_shift)] = page;
            }
            a.granted[i] = flags[e] & 4 ? 1 : 0;
            a.copies[3 * (long long)i] = tail;
            a.copies[3 * (long long)i + 1] = page;
            a.copies[3 * (long long)i + 2] = page >= 0 ? length[e] & place : 0;
        }
    }
    long long pages;
    long long cu = block_exclusive(full, &pages);
#pragma unroll
    for (int e = 0; e < kPageItems; ++e) {
        const int i = i0 + e;
        if (e < items && i < n) {
            s_cu[i] = cu;
            if (flags[e] & 4) cu += length[e] >> page_shift;
        }
    }
    if (taken > 0) atomicAdd(&s_taken, taken);
    copy.put(a.lens, a.lens_out);
    __syncthreads();
    for (long long p = (long long)blockIdx.x * blockDim.x + threadIdx.x; p < pages; p += (long long)gridDim.x * blockDim.x) {
        const int i = find_last64(s_cu, n, p);                // (requests without full pages share their first with the next one)
        const long long j = p - s_cu[i];
        const int page = a.block_table[(long long)s_src[i] * a.table_ld + j];
        a.block_table[(long long)s_dst[i] * a.table_ld + j] = page;
        if (page >= 0 && page < a.num_pages) atomicAdd(a.shared + page, 1);
    }
    if (!last_cta(ticket)) return;
#pragma unroll
    for (int e = 0; e < kPageItems; ++e)
        if (e < items && i0 + e < n && (flags[e] & 4)) a.lens_out[s_dst[i0 + e]] = length[e];
    if (threadIdx.x == 0) *a.free_count_out = free_count - s_taken;
}

// Every listed page loses an owner; one that had no other goes below 0 and is counted in its segment of 256 pages.  The last CTA then
// takes the segments in order (a warp each), which puts the free pages in order of their numbers whatever the order of the atomics.  Bound by
// the chain of its steps, most of it two sums over a CTA and the way to the last one: 12 us for 93 requests of up to 128 pages.
__global__ void __launch_bounds__(kPageThreads) pages_free_kernel(const fi_pages_free_t a, int page_shift, int max_blocks, uint32_t *ticket,
                                                                  int32_t *segments) {
    extern __shared__ long long s_cu[];
    int *const s_row = reinterpret_cast<int *>(s_cu + a.batch_max);
    __shared__ int s_base[kPageSegments];
    in_turn();
    LensCopy copy;
    copy.get(a.lens, a.lens_out, a.rows);
    const int n = actual_count(a.batch_count, a.batch_max);
    const int free_count = min(max(*a.free_count, 0), a.num_pages);
    const int items = (a.batch_max + blockDim.x - 1) / blockDim.x, i0 = threadIdx.x * items;
    int used[kPageItems];
    long long sum = 0;
#pragma unroll
    for (int e = 0; e < kPageItems; ++e) {
        const int i = i0 + e;
        used[e] = 0;
        if (e < items && i < n) {
            const int row = a.row_idx[i];
            const bool ok = row >= 0 && row < a.rows;
            if (ok) used[e] = (int)min(((long long)max(a.lens[row], 0) + (1ll << page_shift) - 1) >> page_shift, (long long)max_blocks);
            s_row[i] = ok ? row : -1;
            sum += used[e];
        }
    }
    long long pages;
    long long cu = block_exclusive(sum, &pages);
#pragma unroll
    for (int e = 0; e < kPageItems; ++e)
        if (e < items && i0 + e < n) {
            s_cu[i0 + e] = cu;
            cu += used[e];
        }
    copy.put(a.lens, a.lens_out);
    __syncthreads();
    for (long long p = (long long)blockIdx.x * blockDim.x + threadIdx.x; p < pages; p += (long long)gridDim.x * blockDim.x) {
        const int i = find_last64(s_cu, n, p);
        const int page = a.block_table[(long long)s_row[i] * a.table_ld + (p - s_cu[i])];
        if (page >= 0 && page < a.num_pages && atomicSub(a.shared + page, 1) == 0) atomicAdd(segments + (page >> kSegmentShift), 1);
    }
    if (!last_cta(ticket)) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int count = (a.num_pages + (1 << kSegmentShift) - 1) >> kSegmentShift;
    // each thread four neighbouring segments at a time
    long long total = 0;
    for (int s0 = 0; s0 < count; s0 += 4 * blockDim.x) {
        int here[4];
        long long mine = 0, all;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int s = s0 + 4 * threadIdx.x + e;
            here[e] = s < count ? __ldcg(segments + s) : 0;
            mine += here[e];
        }
        long long at = total + block_exclusive(mine, &all);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int s = s0 + 4 * threadIdx.x + e;
            if (s < count) {
                s_base[s] = here[e] ? (int)at : -1;
                if (here[e]) segments[s] = 0;
                at += here[e];
            }
        }
        total += all;
    }
    __syncthreads();
    for (int s = warp; s < count; s += warps) {
        long long at = s_base[s];
        if (at < 0) continue;
        int v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int page = (s << kSegmentShift) + e * 32 + lane;
            v[e] = page < a.num_pages ? __ldcg(a.shared + page) : 0;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int page = (s << kSegmentShift) + e * 32 + lane;
            const unsigned gone = __ballot_sync(0xffffffffu, v[e] < 0);
            if (v[e] < 0) {
                const long long to = free_count + at + __popc(gone & ((1u << lane) - 1));
                if (to < a.num_pages) a.free_pages[to] = page;           // (more pages than there are: a stack that was not one)
                a.shared[page] = 0;
            }
            at += __popc(gone);
        }
    }
    for (int i = threadIdx.x; i < n; i += blockDim.x)
        if (s_row[i] >= 0) a.lens_out[s_row[i]] = 0;
    if (threadIdx.x == 0) *a.free_count_out = (int)min(free_count + total, (long long)a.num_pages);
}

// Workspace of a compaction, in words: [0] used pages, from [32] on the new name of each page at or above that number, -1 where it keeps it.
constexpr int kNamesAt = 32;
constexpr int kCompactMost = 64, kCompactPages = 2048;     // CTAs of a compaction, and pages for each of them (beyond 131,072 pages: more)

// Used pages at or above the number of used pages, in order, get the free places below it, in order.  Every CTA has a bit for each page in
// its shared memory and counts all of them for itself, so that nothing is waited for between CTAs; each then takes its share of the moves.
// Bound by the chain of loads, two sums over the CTA and stores: 9.5 us for 5,224 pages (a cluster that shared bits in global memory between
// six barriers: 15.9).  The free stack is read here by all, and rewritten by the kernel behind this one.
__global__ void __launch_bounds__(kPageThreads) pages_compact_kernel(const fi_pages_compact_t a, int page_size, int share) {
    extern __shared__ uint32_t s_free[];                     // a bit for each free page; then the pages to fill and to move of this CTA's share
    in_turn();
    const int words = (a.num_pages + 31) / 32, tid = threadIdx.x;
    int32_t *const s_hole = reinterpret_cast<int32_t *>(s_free + words), *const s_high = s_hole + share;
    int32_t *const name = static_cast<int32_t *>(a.workspace) + kNamesAt;
    const int free_count = min(max(*a.free_count, 0), a.num_pages);
    for (int w = tid; w < words; w += kPageThreads) s_free[w] = 0;
    __syncthreads();
    for (int i0 = tid; i0 < a.num_pages; i0 += 4 * kPageThreads) {
        int page[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) page[e] = i0 + e * kPageThreads < a.num_pages ? a.free_pages[i0 + e * kPageThreads] : -1;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (i0 + e * kPageThreads < free_count && page[e] >= 0 && page[e] < a.num_pages) atomicOr(s_free + (page[e] >> 5), 1u << (page[e] & 31));
    }
    __syncthreads();
    // each thread a run of words
    const int run = (words + kPageThreads - 1) / kPageThreads, first = min(tid * run, words), last = min(first + run, words);
    long long mine = 0, all;
    for (int w = first; w < last; ++w) mine += __popc(s_free[w]);
    block_exclusive(mine, &all);
    const int used = a.num_pages - (int)all;
    // bits of word w that are below `used`, and that are pages
    const auto low = [&](int w) { return w * 32 + 32 <= used ? 0xffffffffu : w * 32 >= used ? 0u : (1u << (used & 31)) - 1; };
    const auto valid = [&](int w) { return w * 32 + 32 <= a.num_pages ? 0xffffffffu : (1u << (a.num_pages & 31)) - 1; };
    // places to fill in the low, pages to move in the high half
    mine = 0;
    for (int w = first; w < last; ++w)
        mine += (long long)__popc(s_free[w] & low(w)) | (long long)__popc(~s_free[w] & ~low(w) & valid(w)) << 32;
    const long long at = block_exclusive(mine, &all);
    int hole = (int)(at & 0xffffffffll), high = (int)(at >> 32);
    const int moves = min((int)(all & 0xffffffffll), (int)(all >> 32)), k0 = blockIdx.x * share, k1 = min(k0 + share, moves);
    for (int w = first; w < last; ++w) {
        const uint32_t f = s_free[w];
        for (uint32_t m = f & low(w); m; m &= m - 1, ++hole)
            if (hole >= k0 && hole < k1) s_hole[hole - k0] = w * 32 + __ffs(m) - 1;
        for (uint32_t m = ~f & ~low(w) & valid(w); m; m &= m - 1, ++high)
            if (high >= k0 && high < k1) s_high[high - k0] = w * 32 + __ffs(m) - 1;
            else if (high >= moves && blockIdx.x == 0) name[w * 32 + __ffs(m) - 1] = -1;       // (a stack that was not one)
        if (w % gridDim.x == blockIdx.x)
            for (uint32_t m = f & ~low(w); m; m &= m - 1) name[w * 32 + __ffs(m) - 1] = -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
        *static_cast<int32_t *>(a.workspace) = used;
        *a.moves = moves;
    }
    __syncthreads();
    for (int k = k0 + tid; k < k1; k += kPageThreads) {
        const int src = s_high[k - k0], dst = s_hole[k - k0];
        name[src] = dst;
        a.shared[dst] = a.shared[src];
        a.shared[src] = 0;
        a.copies[3ll * k] = src;
        a.copies[3ll * k + 1] = dst;
        a.copies[3ll * k + 2] = page_size;
    }
    for (long long k = moves + (long long)blockIdx.x * kPageThreads + tid; k < a.max_copies; k += (long long)gridDim.x * kPageThreads) {
        a.copies[3 * k] = a.copies[3 * k + 1] = -1;
        a.copies[3 * k + 2] = 0;
    }
}

// The new names of the pages that moved, in the rows' entries; and the free stack, lowest number on top.
__global__ void __launch_bounds__(256) pages_rename_kernel(const fi_pages_compact_t a, int page_shift, int max_blocks) {
    in_turn();
    const int used = *static_cast<const int32_t *>(a.workspace), free_count = min(max(*a.free_count, 0), a.num_pages);
    const int32_t *const name = static_cast<const int32_t *>(a.workspace) + kNamesAt;
    for (int row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const int blocks = (int)min(((long long)max(a.lens[row], 0) + (1ll << page_shift) - 1) >> page_shift, (long long)max_blocks);
        int32_t *const entries = a.block_table + (long long)row * a.table_ld;
        for (int j = threadIdx.x; j < blocks; j += 256) {
            const int page = entries[j], to = page >= used && page < a.num_pages ? name[page] : -1;
            if (to >= 0) entries[j] = to;
        }
    }
    for (int i = blockIdx.x * 256 + threadIdx.x; i < free_count; i += gridDim.x * 256) a.free_pages[i] = a.num_pages - 1 - i;
}

struct CopyPools {
    unsigned char *codes[2];
    uint32_t *meta[2];
    long long ps, hs, ts, mps, mhs, mts;
    int heads, page_size, num_pages, pieces;   // pieces of 16 bytes of a vector's codes
    int32_t *status;
};

// A warp per page and head: codes of keys and values in pieces of 16 bytes, 2 + 2 on the way per lane, and their pairs beside them.  Bound
// by the traffic, twice what the tokens take, and by two round trips (1,300 pages of 16 tokens and 8 heads of 128: 9.7 us, 22 MB; with 4 + 4
// pieces, of which such a page has 2 + 2, in 80 registers 13.1).
__global__ void __launch_bounds__(256, 4) kv_copy_pages_kernel(const CopyPools p, const int32_t *copies, const int32_t *count_dev, int most) {
    in_turn();
    const int n = actual_count(count_dev, most), lane = threadIdx.x & 31;
    const long long units = (long long)n * p.heads, step = (long long)gridDim.x * 8;
    for (long long u = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); u < units; u += step) {
        const long long i = u / p.heads;
        const int head = (int)(u - i * p.heads);
        const int src = copies[3 * i], dst = copies[3 * i + 1], tokens = min(copies[3 * i + 2], p.page_size);
        if (src < 0 || tokens <= 0) continue;
        if (src >= p.num_pages || dst < 0 || dst >= p.num_pages) {
            if (lane == 0) atomicOr(p.status, 2);
            continue;
        }
        const long long from = src * p.ps + head * p.hs, to = dst * p.ps + head * p.hs;
        const long long mfrom = src * p.mps + head * p.mhs, mto = dst * p.mps + head * p.mhs;
        const int pieces = tokens * p.pieces;
        uint32_t m[2];
        const bool first = lane < tokens;
#pragma unroll
        for (int kind = 0; kind < 2; ++kind)
            if (first) m[kind] = p.meta[kind][mfrom + lane * p.mts];
        for (int q0 = lane; q0 < pieces; q0 += 64) {
            uint4 v[2][2];
            long long at[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int q = q0 + 32 * e, token = q / p.pieces;
                at[e] = token * p.ts + (q - token * p.pieces) * 16ll;
                if (q < pieces) {
                    v[0][e] = *reinterpret_cast<const uint4 *>(p.codes[0] + from + at[e]);
                    v[1][e] = *reinterpret_cast<const uint4 *>(p.codes[1] + from + at[e]);
                }
            }
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (q0 + 32 * e < pieces) {
                    *reinterpret_cast<uint4 *>(p.codes[0] + to + at[e]) = v[0][e];
                    *reinterpret_cast<uint4 *>(p.codes[1] + to + at[e]) = v[1][e];
                }
        }
#pragma unroll
        for (int kind = 0; kind < 2; ++kind) {
            if (first) p.meta[kind][mto + lane * p.mts] = m[kind];
            for (int t = lane + 32; t < tokens; t += 32) p.meta[kind][mto + t * p.mts] = p.meta[kind][mfrom + t * p.mts];
        }
    }
}

// A launch that may begin while the kernel before it in the stream still runs (a small kernel's launch takes as long as the kernel): every
// kernel here waits for that one before it reads or writes anything, and lets the next one begin at once.
template <typename... Params, typename... Args>
cudaError_t launch_early(void (*kernel)(Params...), int grid, int threads, size_t smem, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)grid);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cfg.attrs = &early;
    cfg.numAttrs = 1;
    count_launch();
    return cudaLaunchKernelEx(&cfg, kernel, Params(args)...);
}

int shift_of(int page_size) {
    int s = 0;
    while (1 << s < page_size) ++s;
    return s;
}

}  // namespace

cudaError_t prepare_pages_share() {
    cudaError_t e = cudaFuncSetAttribute(pages_fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPageMaxBatch * 16);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(pages_free_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPageMaxBatch * 12);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(pages_compact_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 200 * 1024);
    return e;
}

}  // namespace fi

using namespace fi;

extern "C" {

fi_status_t fi_pages_fork(fi_pages_t *p, const fi_pages_fork_t *a, void *cuda_stream) {
    if (!p || !a) {
        set_error("fi_pages_fork: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (a->batch_max < 0 || a->batch_max > p->cfg.max_batch || a->rows < 0 || a->num_pages < 0 || a->table_ld < p->cfg.max_blocks) {
        set_error("fi_pages_fork: batch %d outside 0..%d, a negative size, or table_ld below max_blocks", a->batch_max, p->cfg.max_batch);
        return FI_ERR_INVALID_ARG;
    }
    if ((a->rows > 0 && (!a->lens || !a->lens_out || !a->block_table)) || (a->num_pages > 0 && (!a->free_pages || !a->shared)) || !a->free_count ||
        !a->free_count_out || (a->batch_max > 0 && (!a->src_rows || !a->dst_rows || !a->granted || !a->copies))) {
        set_error("fi_pages_fork: null pointer (only batch_count may be)");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(p->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_pages_fork");
    // an upper bound of the pages, a thread each where the sums over the requests are cheap (64 forks of 48 pages: 8.2 us,
    // in one CTA 14.5)
    const int threads = a->batch_max <= 256 ? 256 : kPageThreads;
    long long grid = (long long)a->batch_max * p->cfg.max_blocks / (a->batch_max <= 256 ? 512 : 4096);
    grid = grid < 1 ? 1 : grid > p->sm_count ? p->sm_count : grid;
    const cudaError_t e = launch_early(pages_fork_kernel, (int)grid, threads, (size_t)a->batch_max * 16, static_cast<cudaStream_t>(cuda_stream), *a,
                                       shift_of(p->cfg.page_size), p->cfg.max_blocks, p->ticket);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_pages_fork");
}

fi_status_t fi_pages_free(fi_pages_t *p, const fi_pages_free_t *a, void *cuda_stream) {
    if (!p || !a) {
        set_error("fi_pages_free: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (a->batch_max < 0 || a->batch_max > p->cfg.max_batch || a->rows < 0 || a->num_pages < 0 || a->num_pages > kPageSegments << kSegmentShift ||
        a->table_ld < p->cfg.max_blocks) {
        set_error("fi_pages_free: batch %d outside 0..%d, a negative size, more than %d pages, or table_ld below max_blocks", a->batch_max,
                  p->cfg.max_batch, kPageSegments << kSegmentShift);
        return FI_ERR_INVALID_ARG;
    }
    if ((a->rows > 0 && (!a->lens || !a->lens_out || !a->block_table)) || (a->num_pages > 0 && (!a->free_pages || !a->shared)) || !a->free_count ||
        !a->free_count_out || (a->batch_max > 0 && !a->row_idx)) {
        set_error("fi_pages_free: null pointer (only batch_count may be)");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(p->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_pages_free");
    long long grid = (long long)a->batch_max * p->cfg.max_blocks / 2048;
    grid = grid < 1 ? 1 : grid > p->sm_count ? p->sm_count : grid;
    const cudaError_t e = launch_early(pages_free_kernel, (int)grid, kPageThreads, (size_t)a->batch_max * 12, static_cast<cudaStream_t>(cuda_stream), *a,
                                       shift_of(p->cfg.page_size), p->cfg.max_blocks, p->ticket, p->segments);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_pages_free");
}

int64_t fi_pages_compact_workspace(int32_t num_pages) {
    if (num_pages < 0) return 0;
    return 4 * (kNamesAt + (int64_t)num_pages);
}

fi_status_t fi_pages_compact(fi_pages_t *p, const fi_pages_compact_t *a, void *cuda_stream) {
    if (!p || !a) {
        set_error("fi_pages_compact: null argument");
        return FI_ERR_INVALID_ARG;
    }
    if (a->rows < 0 || a->num_pages < 0 || a->num_pages > kPageSegments << kSegmentShift || a->max_copies < a->num_pages / 2 ||
        a->table_ld < p->cfg.max_blocks) {
        set_error("fi_pages_compact: a negative size, more than %d pages, room for fewer copies than half of them, or table_ld below max_blocks",
                  kPageSegments << kSegmentShift);
        return FI_ERR_INVALID_ARG;
    }
    if ((a->rows > 0 && (!a->lens || !a->block_table)) || (a->num_pages > 0 && (!a->free_pages || !a->shared)) || !a->free_count || !a->moves ||
        !a->workspace || (a->max_copies > 0 && !a->copies) || (reinterpret_cast<uintptr_t>(a->workspace) & 3)) {
        set_error("fi_pages_compact: null pointer, or a workspace that is not on a 4-byte boundary");
        return FI_ERR_INVALID_ARG;
    }
    DeviceGuard guard(p->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_pages_compact");
    cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    int ctas = (a->num_pages + kCompactPages - 1) / kCompactPages;
    ctas = ctas < 1 ? 1 : ctas > kCompactMost ? kCompactMost : ctas;
    const int share = (a->num_pages / 2 + ctas - 1) / ctas;
    cudaError_t e = launch_early(pages_compact_kernel, ctas, kPageThreads, ((size_t)(a->num_pages + 31) / 32 + 2 * (size_t)share) * 4, stream, *a,
                                 p->cfg.page_size, share);
    if (e == cudaSuccess)
        e = launch_early(pages_rename_kernel, a->rows < 1 ? 1 : a->rows < 8 * p->sm_count ? a->rows : 8 * p->sm_count, 256, 0, stream, *a,
                         shift_of(p->cfg.page_size), p->cfg.max_blocks);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_pages_compact");
}

fi_status_t fi_kv_copy_pages(fi_kv_t *kv, const int32_t *copies, int32_t max_copies, const int32_t *count, void *cuda_stream) {
    if (!kv || max_copies < 0 || (max_copies > 0 && !copies)) {
        set_error("fi_kv_copy_pages: null argument or a negative size");
        return FI_ERR_INVALID_ARG;
    }
    if (max_copies == 0) return FI_OK;
    DeviceGuard guard(kv->cfg.device);
    if (!guard.ok) return cuda_fail(cudaErrorInvalidDevice, "fi_kv_copy_pages");
    const fi_kv_config_t &c = kv->cfg;
    const CopyPools p = {{static_cast<unsigned char *>(c.k_codes), static_cast<unsigned char *>(c.v_codes)},
                         {static_cast<uint32_t *>(c.k_meta), static_cast<uint32_t *>(c.v_meta)},
                         c.page_stride, c.head_stride, c.token_stride, c.meta_page_stride, c.meta_head_stride, c.meta_token_stride,
                         c.kv_heads, c.page_size, c.num_pages, c.head_dim / 32, kv->status_dev};
    const long long units = ((long long)max_copies * c.kv_heads + 7) / 8, most = 4ll * kv->sm_count;
    const cudaError_t e = launch_early(kv_copy_pages_kernel, (int)(units < most ? units : most), 256, 0, static_cast<cudaStream_t>(cuda_stream), p, copies,
                                       count, max_copies);
    return e == cudaSuccess ? FI_OK : cuda_fail(e, "fi_kv_copy_pages");
}

}  // extern "C"

// Page tables of the caches: fork (continue, share, copy, free), grow, compact.
//
// Each call is a plan and, where pages have to be copied, the copies.  The plan is integer work on a few thousand words
// and all of it is latency: one cluster of eight blocks runs it in a handful of phases with the cluster's barrier between
// them (one block alone took as many round trips to memory per phase as it has entries per thread).  Nothing depends on
// the order in which atomics arrive: they only add to counters and take minima, and free pages are found by rank - every
// warp counts those of its slice of the pool, the counts are summed over the warps before it, and a second look at the
// slice names the page of each rank.
//
// The copies (a job is a source page, a target page and a number of tokens) are bound by HBM: a warp copies the codes of
// one (job, kv head, K or V), eight 16-byte words per lane in flight.
#include <cooperative_groups.h>

#include "slim_common.cuh"
#include "slim_tmap.cuh"

namespace slim {

namespace cg = cooperative_groups;

constexpr int kPgCluster = 8;
constexpr int kPgThreads = 512;
constexpr int kPgWarps = kPgCluster * kPgThreads / 32;
constexpr int kPgMaxLayers = 64;   // of one launch (they are passed by value)

constexpr int kAll = kPgCluster * kPgThreads;

// Workspace, in ints: how many jobs there are; the warps' totals; then by page: counters, job sources, job targets; then
// by row: the first child, the rank of the first page that a row needs, and by job the tokens to copy.
struct PagesWork {
    int *n_jobs, *totals, *count, *source, *target, *first, *rank, *part;
};
constexpr int kPgHead = 4 + 3 * kPgWarps;
static PagesWork pages_work(void *workspace, int num_pages, int rows)
{
    int *w = static_cast<int *>(workspace);
    PagesWork p;
    p.n_jobs = w;
    p.totals = w + 4;
    p.count = w + kPgHead;
    p.source = p.count + num_pages;
    p.target = p.source + num_pages;
    p.first = p.target + num_pages;
    p.rank = p.first + rows;
    p.part = p.rank + rows;
    return p;
}
size_t pages_workspace_bytes(int num_pages, int rows)
{
    return ((size_t)kPgHead + 3 * (size_t)num_pages + 3 * (size_t)rows) * sizeof(int);
}

struct PagesParams {
    slim_pages_t from, to;
    PagesWork w;
    const int32_t *parent, *kv_len;
    int32_t *len_out, *result;
    int room;
};

// What the cluster's threads have written becomes visible to all of them.  Words that another block has written are read
// with pg_ld, past the L1.
__device__ __forceinline__ void pg_sync() { cg::this_cluster().sync(); }
__device__ __forceinline__ int pg_ld(const int *ptr) { return __ldcg(ptr); }

// The warp's contiguous slice of n things, in whole groups of 32.
__device__ __forceinline__ void pg_slice(int n, int warp, int &lo, int &hi)
{
    const long long per = ((long long)n + kPgWarps * 32 - 1) / (kPgWarps * 32) * 32;
    lo = (int)min((long long)n, per * warp);
    hi = (int)min((long long)n, per * (warp + 1));
}
// Sum of the totals of the warps before this one, and of all.
__device__ __forceinline__ int pg_before(const int *totals, int warp, int lane, int &all)
{
    int mine = 0, sum = 0;
    for (int i = lane; i < kPgWarps; i += 32) {
        const int v = pg_ld(totals + i);
        sum += v;
        if (i < warp) mine += v;
    }
    all = __reduce_add_sync(0xffffffffu, sum);
    return __reduce_add_sync(0xffffffffu, mine);
}
// How many i of the warp's slice of n satisfy `is`.
template <class Is>
__device__ __forceinline__ int pg_count(int n, int warp, int lane, Is is)
{
    int lo, hi, sum = 0;
    pg_slice(n, warp, lo, hi);
    for (int i = lo + lane; i - lane < hi; i += 32) sum += __popc(__ballot_sync(0xffffffffu, i < hi && is(i)));
    return sum;
}
// Calls found(i, rank) for every i of the slice that satisfies `is`; ranks go on from `base`.
template <class Is, class Found>
__device__ __forceinline__ void pg_rank(int n, int warp, int lane, int base, Is is, Found found)
{
    int lo, hi;
    pg_slice(n, warp, lo, hi);
    for (int i = lo + lane; i - lane < hi; i += 32) {
        const bool yes = i < hi && is(i);
        const unsigned all = __ballot_sync(0xffffffffu, yes);
        if (yes) found(i, base + __popc(all & ((1u << lane) - 1u)));
        base += __popc(all);
    }
}

__device__ __forceinline__ int pg_held(const slim_pages_t &p, int row) { return min(max(__ldg(p.held + row), 0), p.stride); }

// What row i of the new table takes over from its parent: all pages held as the heir, else the full ones; a row that is
// no heir and whose parent's last page is filled in part gets a copy of it.
struct PgRow {
    int parent, shared, part;   // part: tokens of the page to copy (0: none)
    bool heir;
};
__device__ __forceinline__ PgRow pg_row(const PagesParams &p, int i)
{
    PgRow r;
    r.parent = __ldg(p.parent + i);
    r.shared = r.part = 0;
    r.heir = false;
    if (r.parent < 0 || r.parent >= p.from.rows) {
        r.parent = -1;
        return r;
    }
    const int held = pg_held(p.from, r.parent), len = max(__ldg(p.kv_len + r.parent), 0), whole = len / kPageTokens;
    r.heir = pg_ld(p.w.first + r.parent) == i;
    r.shared = r.heir ? held : min(whole, held);
    r.part = (!r.heir && whole < held) ? len % kPageTokens : 0;
    return r;
}

__global__ void __cluster_dims__(kPgCluster, 1, 1) __launch_bounds__(kPgThreads)
slim_pages_fork_kernel(const PagesParams p)
{
    const int lane = threadIdx.x & 31, warp = blockIdx.x * (kPgThreads / 32) + (threadIdx.x >> 5);
    const int thread = blockIdx.x * kPgThreads + threadIdx.x, n_pages = p.from.num_pages;
    int *count = p.w.count;
    pdl_launch_dependents();   // the copies queued behind this launch wait for its end
    pdl_wait();
    for (int i = thread; i < n_pages; i += kAll) count[i] = p.from.refs[i];
    for (int i = thread; i < p.from.rows; i += kAll) p.w.first[i] = 0x7FFFFFFF;
    pg_sync();
    // ---- the old rows let go of their pages; the first child of every row
    for (int b = warp; b < p.from.rows; b += kPgWarps) {
        const int held = pg_held(p.from, b);
        for (int j = lane; j < held; j += 32) {
            const int page = __ldg(p.from.table + (size_t)b * p.from.stride + j);
            if (page >= 0 && page < n_pages) atomicSub(count + page, 1);
        }
    }
    for (int i = thread; i < p.to.rows; i += kAll) {
        const int parent = __ldg(p.parent + i);
        if (parent >= 0 && parent < p.from.rows) atomicMin(p.w.first + parent, i);
    }
    pg_sync();
    // ---- the new rows take theirs
    for (int i = warp; i < p.to.rows; i += kPgWarps) {
        const PgRow r = pg_row(p, i);
        for (int j = lane; j < r.shared; j += 32) {
            const int page = __ldg(p.from.table + (size_t)r.parent * p.from.stride + j);
            if (page >= 0 && page < n_pages) atomicAdd(count + page, 1);
        }
    }
    auto copies = [&](int i) { return pg_row(p, i).part > 0; };
    auto is_free = [&](int page) { return pg_ld(count + page) == 0; };
    {
        const int n = pg_count(p.to.rows, warp, lane, copies);
        if (lane == 0) p.w.totals[warp] = n;
    }
    pg_sync();
    {
        const int n = pg_count(n_pages, warp, lane, is_free);
        if (lane == 0) p.w.totals[kPgWarps + warp] = n;
    }
    pg_sync();
    int need, free_pages;
    const int row_base = pg_before(p.w.totals, warp, lane, need), page_base = pg_before(p.w.totals + kPgWarps, warp, lane, free_pages);
    if (thread == 0) {
        p.result[0] = max(0, need - free_pages);
        p.result[1] = max(0, free_pages - need);
        *p.w.n_jobs = (need <= free_pages) ? need : 0;
    }
    if (need > free_pages) return;   // (every thread of the cluster)
    pg_rank(n_pages, warp, lane, page_base, is_free, [&](int page, int rank) {
        if (rank < need) p.w.target[rank] = page;
    });
    pg_rank(p.to.rows, warp, lane, row_base, copies, [&](int i, int rank) { p.w.rank[i] = rank; });
    pg_sync();
    // ---- rows, jobs and counters
    for (int i = warp; i < p.to.rows; i += kPgWarps) {
        const PgRow r = pg_row(p, i);
        const int32_t *old = p.from.table + (size_t)max(r.parent, 0) * p.from.stride;
        int32_t *row = p.to.table + (size_t)i * p.to.stride;
        int fresh = -1;
        if (r.part > 0) {
            const int rank = pg_ld(p.w.rank + i);
            fresh = pg_ld(p.w.target + rank);
            if (lane == 0) {
                const int page = __ldg(old + r.shared);
                const bool real = page >= 0 && page < n_pages;
                p.w.source[rank] = real ? page : fresh;
                p.w.part[rank] = real ? r.part : 0;
            }
        }
        for (int j = lane; j < p.to.stride; j += 32) row[j] = (j < r.shared) ? __ldg(old + j) : (j == r.shared ? fresh : -1);
        if (lane == 0) {
            p.to.held[i] = r.shared + (r.part > 0 ? 1 : 0);
            p.len_out[i] = (r.parent < 0) ? -1 : __ldg(p.kv_len + r.parent);
        }
    }
    // (a fresh page's counter is 0 in `count` and 1 in the result)
    pg_rank(n_pages, warp, lane, page_base, is_free, [&](int page, int rank) { p.to.refs[page] = (rank < need) ? 1 : 0; });
    for (int i = thread; i < n_pages; i += kAll) {
        const int v = pg_ld(count + i);
        if (v != 0) p.to.refs[i] = v;
    }
}

// Pages that row i lacks for its tokens.
__device__ __forceinline__ int pg_lacks(const PagesParams &p, int i)
{
    const int len = __ldg(p.kv_len + i);
    if (len < 0) return 0;
    const long long want = ((long long)len + p.room + kPageTokens - 1) / kPageTokens;
    return max(0, (int)min(want, (long long)p.from.stride) - min(max(p.from.held[i], 0), p.from.stride));
}

__global__ void __cluster_dims__(kPgCluster, 1, 1) __launch_bounds__(kPgThreads)
slim_pages_grow_kernel(const PagesParams p)
{
    const int lane = threadIdx.x & 31, warp = blockIdx.x * (kPgThreads / 32) + (threadIdx.x >> 5);
    const int n_pages = p.from.num_pages;
    pdl_launch_dependents();
    pdl_wait();
    auto is_free = [&](int page) { return pg_ld(p.from.refs + page) == 0; };
    int lo, hi, lacking = 0;
    pg_slice(p.from.rows, warp, lo, hi);
    // (bounded so that no sum passes 32 bits: more than the largest pool has, and the call ends below)
    constexpr int kMost = (1 << 24) - 1;
    for (int i = lo + lane; i < hi; i += 32) lacking = min(lacking + min(pg_lacks(p, i), kMost), kMost);
    lacking = __reduce_add_sync(0xffffffffu, lacking);
    const int n_free = pg_count(n_pages, warp, lane, is_free);
    if (lane == 0) {
        p.w.totals[warp] = min(lacking, kMost);
        p.w.totals[kPgWarps + warp] = n_free;
    }
    pg_sync();
    int need, free_pages;
    const int row_base = pg_before(p.w.totals, warp, lane, need), page_base = pg_before(p.w.totals + kPgWarps, warp, lane, free_pages);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        p.result[0] = max(0, need - free_pages);
        p.result[1] = max(0, free_pages - need);
    }
    if (need > free_pages || need == 0) return;   // (every thread of the cluster)
    pg_rank(n_pages, warp, lane, page_base, is_free, [&](int page, int rank) {
        if (rank < need) p.w.target[rank] = page;
    });
    pg_sync();   // (the counters of the pages taken change from here on)
    int base = row_base;
    for (int i0 = lo; i0 < hi; i0 += 32) {
        const int i = i0 + lane, n = (i < hi) ? pg_lacks(p, i) : 0;
        int upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const int held = (i < hi) ? min(max(p.from.held[i], 0), p.from.stride) : 0;
        for (int r = 0; r < min(32, hi - i0); ++r) {
            const int n_r = __shfl_sync(0xffffffffu, n, r), at = base + __shfl_sync(0xffffffffu, upto, r) - n_r, held_r = __shfl_sync(0xffffffffu, held, r);
            for (int j = lane; j < n_r; j += 32) {
                const int page = pg_ld(p.w.target + at + j);
                p.from.table[(size_t)(i0 + r) * p.from.stride + held_r + j] = page;
                p.from.refs[page] = 1;
            }
        }
        if (n > 0) p.from.held[i] = held + n;
        base += __shfl_sync(0xffffffffu, upto, 31);
    }
}

__global__ void __cluster_dims__(kPgCluster, 1, 1) __launch_bounds__(kPgThreads)
slim_pages_compact_kernel(const PagesParams p)
{
    const int lane = threadIdx.x & 31, warp = blockIdx.x * (kPgThreads / 32) + (threadIdx.x >> 5);
    const int thread = blockIdx.x * kPgThreads + threadIdx.x, n_pages = p.from.num_pages;
    int *count = p.w.count;
    pdl_launch_dependents();
    pdl_wait();
    for (int i = thread; i < n_pages; i += kAll) count[i] = p.from.refs[i];   // (`to` may be `from`)
    pg_sync();
    auto is_used = [&](int page) { return pg_ld(count + page) != 0; };
    const int mine = pg_count(n_pages, warp, lane, is_used);
    if (lane == 0) p.w.totals[warp] = mine;
    pg_sync();
    int n_used;
    const int before = pg_before(p.w.totals, warp, lane, n_used);
    (void)before;
    auto moves = [&](int page) { return page >= n_used && is_used(page); };
    auto hole = [&](int page) { return page < n_used && !is_used(page); };
    const int n_moves = pg_count(n_pages, warp, lane, moves), n_holes = pg_count(n_pages, warp, lane, hole);
    if (lane == 0) {
        p.w.totals[kPgWarps + warp] = n_moves;
        p.w.totals[2 * kPgWarps + warp] = n_holes;
    }
    pg_sync();
    int all, all_holes;   // (as many holes as movers)
    const int base = pg_before(p.w.totals + kPgWarps, warp, lane, all), hole_base = pg_before(p.w.totals + 2 * kPgWarps, warp, lane, all_holes);
    if (thread == 0) {
        p.result[0] = n_used;
        p.result[1] = all;
        *p.w.n_jobs = all;
    }
    pg_rank(n_pages, warp, lane, hole_base, hole, [&](int page, int rank) { p.w.target[rank] = page; });
    pg_sync();
    // ---- a mover's page takes its counter along and leaves its new id in `count` (as a negative number)
    pg_rank(n_pages, warp, lane, base, moves, [&](int page, int rank) {
        const int to = pg_ld(p.w.target + rank);
        p.w.source[rank] = page;
        p.to.refs[to] = pg_ld(count + page);
        p.to.refs[page] = 0;
        count[page] = -1 - to;
    });
    pg_sync();
    for (int i = thread; i < n_pages; i += kAll) {
        const int v = pg_ld(count + i);
        if (i < n_used && v != 0) p.to.refs[i] = v;
        if (i >= n_used && v == 0) p.to.refs[i] = 0;
    }
    for (int b = warp; b < p.from.rows; b += kPgWarps) {
        const int held = min(max(p.from.held[b], 0), p.from.stride);
        for (int j = lane; j < p.from.stride; j += 32) {
            int page = -1;
            if (j < held) {
                page = p.from.table[(size_t)b * p.from.stride + j];
                if (page >= n_used && page < n_pages) {
                    const int v = pg_ld(count + page);
                    if (v < 0) page = -1 - v;
                }
            }
            p.to.table[(size_t)b * p.to.stride + j] = page;
        }
        if (lane == 0) p.to.held[b] = held;
    }
}

// ---------------------------------------------------------------- copies
struct PageLayersArg {
    slim_layer_t at[kPgMaxLayers];
};
constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 8;

// `bytes` (a multiple of 4) from one 16-byte aligned place to another by a warp.
__device__ __forceinline__ void pg_copy(unsigned char *dst, const unsigned char *src, int bytes, int lane)
{
    const uint4 *s = reinterpret_cast<const uint4 *>(src);
    uint4 *d = reinterpret_cast<uint4 *>(dst);
    const int words = bytes / 16;
    int i = lane;
    for (; i + 32 * (kCopyUnroll - 1) < words; i += 32 * kCopyUnroll) {
        uint4 v[kCopyUnroll];
#pragma unroll
        for (int k = 0; k < kCopyUnroll; ++k) v[k] = __ldcs(s + i + 32 * k);
#pragma unroll
        for (int k = 0; k < kCopyUnroll; ++k) __stcs(d + i + 32 * k, v[k]);
    }
    for (; i < words; i += 32) d[i] = __ldcs(s + i);
    for (int k = words * 4 + lane; k < bytes / 4; k += 32) reinterpret_cast<uint32_t *>(dst)[k] = reinterpret_cast<const uint32_t *>(src)[k];
}

// blockIdx.y: the layer.  An item is one (job, kv head, K or V): the codes of its tokens and their scales.
__global__ void __launch_bounds__(kCopyThreads)
slim_pages_copy_kernel(const __grid_constant__ PageLayersArg layers, const PagesWork w, const int whole)
{
    const int lane = threadIdx.x & 31;
    const slim_layer_t &layer = layers.at[blockIdx.y];
    pdl_wait();
    const int blocks = 2 * layer.num_kv_heads;
    const long long items = (long long)pg_ld(w.n_jobs) * blocks;
    for (long long it = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); it < items; it += (long long)gridDim.x * (kCopyThreads / 32)) {
        const int job = (int)(it / blocks), part = (int)(it - (long long)job * blocks);
        const int tokens = whole ? kPageTokens : pg_ld(w.part + job);
        const size_t from = (size_t)pg_ld(w.source + job) * blocks + part, to = (size_t)pg_ld(w.target + job) * blocks + part;
        const size_t code_block = (size_t)kPageTokens * layer.row_bytes, scale_block = (size_t)kPageTokens * 4;
        unsigned char *codes = static_cast<unsigned char *>(layer.codes), *scales = static_cast<unsigned char *>(layer.scales);
        pg_copy(codes + to * code_block, codes + from * code_block, tokens * layer.row_bytes, lane);
        pg_copy(scales + to * scale_block, scales + from * scale_block, tokens * 4, lane);
    }
}

// ---------------------------------------------------------------- host side
static int launch_copies(const PagesWork &w, const slim_layer_t *layers, int n_layers, long long most_jobs, bool whole, cudaStream_t stream)
{
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc != SLIM_OK) return rc;
    for (int l0 = 0; l0 < n_layers; l0 += kPgMaxLayers) {
        const int n = n_layers - l0 < kPgMaxLayers ? n_layers - l0 : kPgMaxLayers;
        PageLayersArg arg;
        long long items = 1;
        for (int i = 0; i < kPgMaxLayers; ++i) {
            arg.at[i] = layers[l0 + (i < n ? i : 0)];
            const long long here = most_jobs * 2 * arg.at[i].num_kv_heads;
            items = here > items ? here : items;
        }
        long long blocks = (items + kCopyThreads / 32 - 1) / (kCopyThreads / 32);
        const long long most = (8LL * sms + n - 1) / n;   // eight blocks of 256 threads per SM
        if (blocks > most) blocks = most;
        SLIM_CUDA_TRY(launch_pdl(slim_pages_copy_kernel, dim3((unsigned)blocks, (unsigned)n), dim3(kCopyThreads), 0, stream, arg, w, whole ? 1 : 0));
    }
    return SLIM_OK;
}

int launch_pages_fork(const slim_pages_t *from, const slim_pages_t *to, const int32_t *parent, const int32_t *kv_len, int32_t *len_out,
                      const slim_layer_t *layers, int n_layers, int32_t *result, void *workspace, cudaStream_t stream)
{
    PagesParams p;
    p.from = *from;
    p.to = *to;
    p.w = pages_work(workspace, from->num_pages, from->rows > to->rows ? from->rows : to->rows);
    p.parent = parent;
    p.kv_len = kv_len;
    p.len_out = len_out;
    p.result = result;
    p.room = 0;
    SLIM_CUDA_TRY(launch_pdl(slim_pages_fork_kernel, dim3(kPgCluster), dim3(kPgThreads), 0, stream, p));
    return launch_copies(p.w, layers, n_layers, to->rows, false, stream);
}

int launch_pages_grow(const slim_pages_t *pages, const int32_t *kv_len, int room, int32_t *result, void *workspace, cudaStream_t stream)
{
    PagesParams p;
    p.from = p.to = *pages;
    p.w = pages_work(workspace, pages->num_pages, pages->rows);
    p.parent = nullptr;
    p.kv_len = kv_len;
    p.len_out = nullptr;
    p.result = result;
    p.room = room;
    SLIM_CUDA_TRY(launch_pdl(slim_pages_grow_kernel, dim3(kPgCluster), dim3(kPgThreads), 0, stream, p));
    return SLIM_OK;
}

int launch_pages_compact(const slim_pages_t *from, const slim_pages_t *to, const slim_layer_t *layers, int n_layers, int32_t *result,
                         void *workspace, cudaStream_t stream)
{
    PagesParams p;
    p.from = *from;
    p.to = *to;
    p.w = pages_work(workspace, from->num_pages, from->rows);
    p.parent = p.kv_len = nullptr;
    p.len_out = nullptr;
    p.result = result;
    p.room = 0;
    SLIM_CUDA_TRY(launch_pdl(slim_pages_compact_kernel, dim3(kPgCluster), dim3(kPgThreads), 0, stream, p));
    return launch_copies(p.w, layers, n_layers, from->num_pages, true, stream);
}

}  // namespace slim

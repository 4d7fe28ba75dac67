// Page tables of the caches: fork (continue, share, copy, free), grow, compact.
//
// Each call is a plan and, where pages have to be copied, the copies.  The plan is integer work on a few thousand words
// and all of it is latency, so one block runs it, with the page counters and what it notes per row in shared memory where
// they fit (below 50,000 words: phases then cost a barrier each.  A cluster of eight blocks with its counters in global memory,
// a cluster barrier and a trip to the L2 per phase took 10.9 us where this form takes 5.0 us on 16 rows of 59 pages in all).
// It walks all rows x stride entries of a table, held or not, which only wide tables feel: 256 rows of 64 pages, 4 held each, fork 12
// and compact 11 us; of 1024 pages, 10 held, 108 and 85; 900 held (230,000 pages, counted in global memory) 351 and 300, grow 72.
// Nothing depends on the order in which atomics arrive: they only add to counters and take minima, and free pages are found
// by rank - every warp counts those of its slice of the pool, the counts of the warps before it are summed, and a second
// look at the slice names the page of each rank.
//
// The copies (a job is a source page, a target page and a number of tokens) are bound by HBM: a warp copies the codes of
// one (job, kv head, K or V), eight 16-byte words per lane in flight.  About 500 pages in eight INT8 layers, 2.1 GB read and written:
// 354 us (366 with the two plans), 6.0 TB/s, 92 % of the copy rate.  Four or sixteen words per lane: 351 and 347 there, but about 250
// pages copied in part after a fork of 256 rows take 85 and 156 us in all in place of 83.
#include "slim_common.cuh"
#include "slim_tmap.cuh"

namespace slim {

constexpr int kPgThreads = 1024;
constexpr int kPgWarps = kPgThreads / 32;
constexpr int kPgMaxLayers = 64;           // of one launch (they are passed by value)
constexpr int kPgSharedInts = 50000;       // counters and rows' notes that go into shared memory (a fork of 16 rows, 59 pages: 4.9 us,
                                           // in global memory 7.4; of 256 rows, 1020 pages: 9.6 and 13.9)

// Workspace, in ints: how many jobs there are; by page: job sources and targets, counters; by row: tokens of the job, the
// row's notes.  The copies read the jobs (and callers a compaction's, from SLIM_PAGES_MOVED_OFFSET on); counters and notes are
// used only where shared memory does not hold them.
struct PagesWork {
    int *n_jobs, *source, *target, *part, *notes;
};
constexpr int kPgHead = SLIM_PAGES_MOVED_OFFSET / (int)sizeof(int);
constexpr int kPgNotes = 4;   // notes per row
static PagesWork pages_work(void *workspace, int num_pages, int rows)
{
    PagesWork p;
    p.n_jobs = static_cast<int *>(workspace);
    p.source = p.n_jobs + kPgHead;
    p.target = p.source + num_pages;
    p.part = p.target + num_pages;
    p.notes = p.part + rows;
    return p;
}
size_t pages_workspace_bytes(int num_pages, int rows)
{
    return (kPgHead + 3 * (size_t)num_pages + (1 + kPgNotes) * (size_t)rows) * sizeof(int);
}

struct PagesParams {
    slim_pages_t from, to;
    PagesWork w;
    const int32_t *parent, *kv_len;
    int32_t *len_out, *result;
    int room, rows;   // rows: the larger of the two tables'
};

// The block's arrays: counters by page, then four notes by row.  Where they lie in global memory the atomics on them bypass
// the L1, and so do these loads.
template <bool kShared>
struct PgArrays {
    int *count, *a, *b, *c, *d;
    __device__ __forceinline__ PgArrays(const PagesParams &p, int *smem)
    {
        count = kShared ? smem : p.w.notes;
        a = count + p.from.num_pages;
        b = a + p.rows, c = b + p.rows, d = c + p.rows;
    }
    __device__ __forceinline__ static int ld(const int *ptr) { return kShared ? *ptr : __ldcg(ptr); }
};

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
    const int v = totals[lane];
    all = __reduce_add_sync(0xffffffffu, v);
    return __reduce_add_sync(0xffffffffu, lane < warp ? v : 0);
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
// Calls body(row, j) for every entry of a table, several of a thread's entries in flight.
template <class Body>
__device__ __forceinline__ void pg_entries(int rows, int stride, Body body)
{
    const long long n = (long long)rows * stride;
    if (n <= 0x7FFFFFFF - 4 * kPgThreads) {
#pragma unroll 4
        for (int i = threadIdx.x; i < (int)n; i += kPgThreads) body((int)((unsigned)i / (unsigned)stride), (int)((unsigned)i % (unsigned)stride));
    } else {
        for (long long i = threadIdx.x; i < n; i += kPgThreads) body((int)(i / stride), (int)(i % stride));
    }
}
__device__ __forceinline__ int pg_held(const slim_pages_t &p, int row) { return min(max(p.held[row], 0), p.stride); }

template <bool kShared>
__global__ void __launch_bounds__(kPgThreads, 1)
slim_pages_fork_kernel(const PagesParams p)
{
    extern __shared__ int smem_ints[];
    __shared__ int totals[2][kPgWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_pages = p.from.num_pages, n_in = p.from.rows, n_out = p.to.rows;
    const PgArrays<kShared> ar(p, smem_ints);
    auto ld = [](const int *ptr) { return PgArrays<kShared>::ld(ptr); };
    int *count = ar.count, *first = ar.a, *kids = ar.b;      // by old row: its first child, how many it has
    pdl_launch_dependents();   // the copies queued behind this launch wait for its end
    pdl_wait();
    for (int i = tid; i < n_pages; i += kPgThreads) count[i] = p.from.refs[i];
    for (int b = tid; b < n_in; b += kPgThreads) first[b] = 0x7FFFFFFF, kids[b] = 0;
    __syncthreads();
    for (int i = tid; i < n_out; i += kPgThreads) {
        const int parent = __ldg(p.parent + i);
        if (parent >= 0 && parent < n_in) {
            atomicMin(first + parent, i);
            atomicAdd(kids + parent, 1);
        }
    }
    __syncthreads();
    // ---- a full page is held by all children from now on, the pages behind those by the first child
    pg_entries(n_in, p.from.stride, [&](int b, int j) {
        const int n = ld(kids + b);
        if (n == 1 || j >= pg_held(p.from, b)) return;
        const int change = (n == 0) ? -1 : (j < max(__ldg(p.kv_len + b), 0) / kPageTokens ? n - 1 : 0);
        if (change == 0) return;
        const int page = __ldg(p.from.table + (size_t)b * p.from.stride + j);
        if (page >= 0 && page < n_pages) atomicAdd(count + page, change);
    });
    // ---- what a new row takes over: all pages held as its parent's first child, else the full ones and a copy of the tokens
    //      behind them
    int *shared = ar.c, *rank = ar.d;   // by new row: pages taken over; tokens to copy, later the copy's rank
    for (int i = tid; i < n_out; i += kPgThreads) {
        const int parent = __ldg(p.parent + i);
        int take = 0, part = 0;
        if (parent >= 0 && parent < n_in) {
            const int held = pg_held(p.from, parent), len = max(__ldg(p.kv_len + parent), 0), whole = len / kPageTokens;
            const bool heir = ld(first + parent) == i;
            take = heir ? held : min(whole, held);
            part = (!heir && whole < held) ? len % kPageTokens : 0;
        }
        shared[i] = take, rank[i] = part;
    }
    __syncthreads();
    auto copies = [&](int i) { return ld(rank + i) > 0; };
    auto is_free = [&](int page) { return ld(count + page) == 0; };
    {
        const int a = pg_count(n_out, warp, lane, copies), b = pg_count(n_pages, warp, lane, is_free);
        if (lane == 0) totals[0][warp] = a, totals[1][warp] = b;
    }
    __syncthreads();
    int need, free_pages;
    const int row_base = pg_before(totals[0], warp, lane, need), page_base = pg_before(totals[1], warp, lane, free_pages);
    if (tid == 0) {
        p.result[0] = max(0, need - free_pages);
        p.result[1] = max(0, free_pages - need);
        *p.w.n_jobs = (need <= free_pages) ? need : 0;
    }
    if (need > free_pages) return;   // (every thread)
    // ---- free pages by rank, jobs by rank; a page taken has one holder
    pg_rank(n_pages, warp, lane, page_base, is_free, [&](int page, int r) {
        if (r < need) p.w.target[r] = page;
        p.to.refs[page] = (r < need) ? 1 : 0;
    });
    pg_rank(n_out, warp, lane, row_base, copies, [&](int i, int r) {
        const int page = __ldg(p.from.table + (size_t)__ldg(p.parent + i) * p.from.stride + ld(shared + i));
        const bool real = page >= 0 && page < n_pages;
        p.w.source[r] = real ? page : 0;
        p.w.part[r] = real ? ld(rank + i) : 0;
        rank[i] = -1 - r;
    });
    for (int i = tid; i < n_pages; i += kPgThreads) {
        const int v = ld(count + i);
        if (v != 0) p.to.refs[i] = v;
    }
    __syncthreads();
    pg_entries(n_out, p.to.stride, [&](int i, int j) {
        const int take = ld(shared + i), r = ld(rank + i);
        int page = -1;
        if (j < take) page = __ldg(p.from.table + (size_t)__ldg(p.parent + i) * p.from.stride + j);
        else if (j == take && r < 0) page = __ldcg(p.w.target - 1 - r);
        p.to.table[(size_t)i * p.to.stride + j] = page;
    });
    for (int i = tid; i < n_out; i += kPgThreads) {
        const int parent = __ldg(p.parent + i);
        p.to.held[i] = ld(shared + i) + (ld(rank + i) < 0 ? 1 : 0);
        p.len_out[i] = (parent >= 0 && parent < n_in) ? __ldg(p.kv_len + parent) : -1;
    }
}

template <bool kShared>
__global__ void __launch_bounds__(kPgThreads, 1)
slim_pages_grow_kernel(const PagesParams p)
{
    extern __shared__ int smem_ints[];
    __shared__ int totals[2][kPgWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_pages = p.from.num_pages, n = p.from.rows, stride = p.from.stride;
    const PgArrays<kShared> ar(p, smem_ints);
    auto ld = [](const int *ptr) { return PgArrays<kShared>::ld(ptr); };
    int *count = ar.count, *lacks = ar.a, *base = ar.b, *held = ar.c;   // by row: pages that it lacks, the rank of the first of them
    pdl_launch_dependents();
    pdl_wait();
    for (int i = tid; i < n_pages; i += kPgThreads) count[i] = p.from.refs[i];
    for (int i = tid; i < n; i += kPgThreads) {
        const int len = __ldg(p.kv_len + i), has = pg_held(p.from, i);
        const long long want = ((long long)max(len, 0) + p.room + kPageTokens - 1) / kPageTokens;
        lacks[i] = (len < 0) ? 0 : max(0, (int)min(want, (long long)stride) - has);
        held[i] = has;
    }
    __syncthreads();
    auto is_free = [&](int page) { return ld(count + page) == 0; };
    int lo, hi, mine = 0;
    pg_slice(n, warp, lo, hi);
    // (bounded so that no sum passes 32 bits: more than the largest pool has, and the call ends below)
    constexpr int kMost = (1 << 24) - 1;
    for (int i = lo + lane; i < hi; i += 32) mine = min(mine + min(ld(lacks + i), kMost), kMost);
    mine = min(__reduce_add_sync(0xffffffffu, mine), kMost);
    const int n_free = pg_count(n_pages, warp, lane, is_free);
    if (lane == 0) totals[0][warp] = mine, totals[1][warp] = n_free;
    __syncthreads();
    int need, free_pages;
    int at = pg_before(totals[0], warp, lane, need);
    const int page_base = pg_before(totals[1], warp, lane, free_pages);
    if (tid == 0) {
        p.result[0] = max(0, need - free_pages);
        p.result[1] = max(0, free_pages - need);
    }
    if (need > free_pages || need == 0) return;   // (every thread)
    pg_rank(n_pages, warp, lane, page_base, is_free, [&](int page, int r) {
        if (r < need) p.w.target[r] = page, p.from.refs[page] = 1;
    });
    for (int i0 = lo; i0 < hi; i0 += 32) {
        const int v = (i0 + lane < hi) ? ld(lacks + i0 + lane) : 0;
        int upto = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += x;
        }
        if (i0 + lane < hi) base[i0 + lane] = at + upto - v;
        at += __shfl_sync(0xffffffffu, upto, 31);
    }
    __syncthreads();
    // (a row lacks few pages as a rule: a warp takes a row at a time, several in flight)
#pragma unroll 4
    for (int i = warp; i < n; i += kPgWarps) {
        const int v = ld(lacks + i), b = ld(base + i), has = ld(held + i);
        for (int j = lane; j < v; j += 32) p.from.table[(size_t)i * stride + has + j] = __ldcg(p.w.target + b + j);
        if (lane == 0 && v > 0) p.from.held[i] = has + v;
    }
}

template <bool kShared>
__global__ void __launch_bounds__(kPgThreads, 1)
slim_pages_compact_kernel(const PagesParams p)
{
    extern __shared__ int smem_ints[];
    __shared__ int totals[3][kPgWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n_pages = p.from.num_pages, n = p.from.rows, stride = p.from.stride;
    const PgArrays<kShared> ar(p, smem_ints);
    auto ld = [](const int *ptr) { return PgArrays<kShared>::ld(ptr); };
    int *count = ar.count, *held = ar.a;
    pdl_launch_dependents();
    pdl_wait();
    for (int i = tid; i < n_pages; i += kPgThreads) count[i] = p.from.refs[i];   // (`to` may be `from`)
    for (int b = tid; b < n; b += kPgThreads) held[b] = pg_held(p.from, b);
    __syncthreads();
    auto is_used = [&](int page) { return ld(count + page) != 0; };
    {
        const int a = pg_count(n_pages, warp, lane, is_used);
        if (lane == 0) totals[0][warp] = a;
    }
    __syncthreads();
    int n_used;
    (void)pg_before(totals[0], warp, lane, n_used);
    auto moves = [&](int page) { return page >= n_used && is_used(page); };
    auto hole = [&](int page) { return page < n_used && !is_used(page); };
    {
        const int a = pg_count(n_pages, warp, lane, moves), b = pg_count(n_pages, warp, lane, hole);
        if (lane == 0) totals[1][warp] = a, totals[2][warp] = b;
    }
    __syncthreads();
    int all, all_holes;   // (as many holes as movers)
    const int base = pg_before(totals[1], warp, lane, all), hole_base = pg_before(totals[2], warp, lane, all_holes);
    if (tid == 0) {
        p.result[0] = n_used;
        p.result[1] = all;
        *p.w.n_jobs = all;
    }
    pg_rank(n_pages, warp, lane, hole_base, hole, [&](int page, int r) { p.w.target[r] = page; });
    __syncthreads();
    // ---- a mover's page takes its counter along and leaves its new id in `count` (as a negative number)
    pg_rank(n_pages, warp, lane, base, moves, [&](int page, int r) {
        const int to = __ldcg(p.w.target + r);
        p.w.source[r] = page;
        p.to.refs[to] = ld(count + page);
        p.to.refs[page] = 0;
        count[page] = -1 - to;
    });
    __syncthreads();
    for (int i = tid; i < n_pages; i += kPgThreads) {
        const int v = ld(count + i);
        if (i < n_used && v != 0) p.to.refs[i] = v;
        if (i >= n_used && v == 0) p.to.refs[i] = 0;
    }
    pg_entries(n, stride, [&](int b, int j) {
        int page = -1;
        if (j < ld(held + b)) {
            page = p.from.table[(size_t)b * stride + j];
            if (page >= n_used && page < n_pages) {
                const int v = ld(count + page);
                if (v < 0) page = -1 - v;
            }
        }
        p.to.table[(size_t)b * stride + j] = page;
    });
    for (int b = tid; b < n; b += kPgThreads) p.to.held[b] = ld(held + b);
}

// ---------------------------------------------------------------- copies
struct PageLayersArg {
    slim_layer_t at[kPgMaxLayers];
};
constexpr int kCopyThreads = 256;
constexpr int kCopyUnroll = 8;

// blockIdx.y: the layer.  An item is one (job, kv head, K or V): the codes of its tokens and their scales.  A lane takes four
// tokens' scales (its 16 bytes are on their way with the first codes).
__global__ void __launch_bounds__(kCopyThreads)
slim_pages_copy_kernel(const __grid_constant__ PageLayersArg layers, const PagesWork w, const int whole)
{
    const int lane = threadIdx.x & 31;
    const slim_layer_t &layer = layers.at[blockIdx.y];
    pdl_wait();
    const int blocks = 2 * layer.num_kv_heads;
    const long long items = (long long)__ldcg(w.n_jobs) * blocks;
    for (long long it = (long long)blockIdx.x * (kCopyThreads / 32) + (threadIdx.x >> 5); it < items; it += (long long)gridDim.x * (kCopyThreads / 32)) {
        const int job = (int)(it / blocks), part = (int)(it - (long long)job * blocks);
        const int tokens = whole ? kPageTokens : __ldcg(w.part + job);
        const size_t from = (size_t)__ldcg(w.source + job) * blocks + part, to = (size_t)__ldcg(w.target + job) * blocks + part;
        const int code_words = kPageTokens * layer.row_bytes / 16, words = tokens * layer.row_bytes / 16;
        const uint4 *src = static_cast<const uint4 *>(layer.codes) + from * code_words;
        uint4 *dst = static_cast<uint4 *>(layer.codes) + to * code_words;
        const uint4 *scale_src = static_cast<const uint4 *>(layer.scales) + from * (kPageTokens / 4) + lane;
        uint4 *scale_dst = static_cast<uint4 *>(layer.scales) + to * (kPageTokens / 4) + lane;
        const bool scales = 4 * lane < tokens;
        uint4 sc = make_uint4(0, 0, 0, 0);
        if (scales) sc = __ldcs(scale_src);
        int i = lane;
        for (; i + 32 * (kCopyUnroll - 1) < words; i += 32 * kCopyUnroll) {
            uint4 v[kCopyUnroll];
#pragma unroll
            for (int k = 0; k < kCopyUnroll; ++k) v[k] = __ldcs(src + i + 32 * k);
#pragma unroll
            for (int k = 0; k < kCopyUnroll; ++k) __stcs(dst + i + 32 * k, v[k]);
        }
        for (; i < words; i += 32) __stcs(dst + i, __ldcs(src + i));
        if (4 * lane + 4 <= tokens) {
            __stcs(scale_dst, sc);
        } else if (scales) {   // (the tokens behind the last one keep theirs)
            const uint32_t v[3] = {sc.x, sc.y, sc.z};
            for (int k = 0; k < tokens - 4 * lane; ++k) reinterpret_cast<uint32_t *>(scale_dst)[k] = v[k];
        }
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

// One block; its arrays in shared memory where they fit.
static int launch_plan(void (*in_shared)(PagesParams), void (*in_global)(PagesParams), const PagesParams &p, cudaStream_t stream)
{
    const long long ints = (long long)p.from.num_pages + (long long)kPgNotes * p.rows;
    const bool fits = ints <= kPgSharedInts;
    if (fits) {
        const int rc = allow_dynamic_smem(reinterpret_cast<const void *>(in_shared), kPgSharedInts * (int)sizeof(int));
        if (rc != SLIM_OK) return rc;
    }
    SLIM_CUDA_TRY(launch_pdl(fits ? in_shared : in_global, dim3(1), dim3(kPgThreads), fits ? (size_t)ints * sizeof(int) : 0, stream, p));
    return SLIM_OK;
}
static PagesParams pages_params(const slim_pages_t *from, const slim_pages_t *to, const int32_t *kv_len, int32_t *result, void *workspace)
{
    PagesParams p;
    p.from = *from;
    p.to = *to;
    p.rows = from->rows > to->rows ? from->rows : to->rows;
    p.w = pages_work(workspace, from->num_pages, p.rows);
    p.parent = nullptr;
    p.kv_len = kv_len;
    p.len_out = nullptr;
    p.result = result;
    p.room = 0;
    return p;
}

int launch_pages_fork(const slim_pages_t *from, const slim_pages_t *to, const int32_t *parent, const int32_t *kv_len, int32_t *len_out,
                      const slim_layer_t *layers, int n_layers, int32_t *result, void *workspace, cudaStream_t stream)
{
    PagesParams p = pages_params(from, to, kv_len, result, workspace);
    p.parent = parent;
    p.len_out = len_out;
    const int rc = launch_plan(slim_pages_fork_kernel<true>, slim_pages_fork_kernel<false>, p, stream);
    return rc != SLIM_OK ? rc : launch_copies(p.w, layers, n_layers, to->rows, false, stream);
}

int launch_pages_grow(const slim_pages_t *pages, const int32_t *kv_len, int room, int32_t *result, void *workspace, cudaStream_t stream)
{
    PagesParams p = pages_params(pages, pages, kv_len, result, workspace);
    p.room = room;
    return launch_plan(slim_pages_grow_kernel<true>, slim_pages_grow_kernel<false>, p, stream);
}

int launch_pages_compact(const slim_pages_t *from, const slim_pages_t *to, const slim_layer_t *layers, int n_layers, int32_t *result,
                         void *workspace, cudaStream_t stream)
{
    const PagesParams p = pages_params(from, to, nullptr, result, workspace);
    const int rc = launch_plan(slim_pages_compact_kernel<true>, slim_pages_compact_kernel<false>, p, stream);
    return rc != SLIM_OK ? rc : launch_copies(p.w, layers, n_layers, from->num_pages, true, stream);
}

}  // namespace slim

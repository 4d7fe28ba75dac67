// Eviction from the INT8 cache by accumulated attention weight: every (sequence, kv head) keeps `budget` of its tokens.
//
//   protected(j) = pos_j < n_sink  or  pos_j >= seen - n_recent
//   kept         = the budget first slots in the order (protected first, larger weight first, lower slot first)
//
// Softmax attention does not depend on the order of the keys, so the kept tokens are not shifted together: those in
// the slots below the budget stay where they are, and the others fill, in ascending order, the slots that became free
// there.  Sources (slots >= budget) and destinations (slots < budget) never overlap, so the rows move in any order and
// at most min(budget, length - budget) of them move at all; a cache cut back every step moves one row per head instead
// of rewriting all of it.  What is lost is that a slot tells the position, so positions are kept beside the weights.
//
// Selection: a weight is mapped to an unsigned integer of the same order (a protected token to the largest one).  The
// budget-th largest key is found from one histogram of 2048 equal steps between the smallest and the largest key
// (integers of floats are spread like their logarithms; the smallest key, which the tokens without any weight share, is
// counted apart): the tokens of the step that holds it are listed, and a comparison of each with all gives its rank; a
// step with too many of them gets a histogram of its own.  A thread owns consecutive slots, so the freed and the moving
// slots are ranked by one prefix sum of bit counts; weights and positions are read once, in whole lines, and handed to
// the slots' owners through shared memory.  A row of up to 8192 tokens is one block's, a longer one a cluster's
// of up to eight blocks, which read one another's histograms and lists through distributed shared memory;
// beyond 131072 tokens one block walks the row again for each of four histograms of digits (rows of 131072 tokens cut to
// 16384: 324 us that way, 33 us by the cluster).
// Measured (512 rows of 2049 tokens with their one move / 256 of up to 4096, selection alone / 2 of 32768 with their moves):
// 10.6 / 15 / 19.8 us; forms before it, selection alone: four histograms of the keys' digits 34 / 36 / 29 us (weights share their leading bits, the additions to one counter
// queue up), a search with three bounds a step 18 / 23 / 27 us.
// Nothing depends on the order of atomic additions (counts, and a list that is only ranked), so equal inputs give equal
// results.
// Few moving rows are copied by the block that chose them, many by a second kernel over all the SMs, which keeps enough
// bytes on their way (256 rows of up to 4096 tokens cut to 1024: 15 us of selection and 15 us of moves, 81 MB, 84 % of
// the copy rate; 49 us when the selecting blocks move as many).
#include <cooperative_groups.h>

#include "slim_common.cuh"
#include "slim_tmap.cuh"

namespace slim {

namespace cg = cooperative_groups;

constexpr int kEvBlockMoves = 64;         // moves that the selecting block makes itself; moves of one block of the move kernel
constexpr int kEvItems = 8;               // slots per thread of the 1024-thread blocks
constexpr int kEvBlockTokens = 1024 * kEvItems;
constexpr int kEvMaxCluster = 8;
constexpr int kEvBins = 2048;
constexpr int kEvList = 128;              // keys of one step of the histogram that are ranked by comparing all with all

struct EvictParams {
    int8_t *codes;
    float *scales;
    const int32_t *block_table;
    const float *w_in;
    float *w_out;
    const int32_t *pos_in;
    int32_t *pos_out;
    const int32_t *kv_len, *placed, *seen;
    int32_t *moves;        // [rows][3][cap]: freed slots, the cache rows of the freed slots, the cache rows of the moving slots
    int32_t *n_moves;      // [rows]
    int stride, max_kv, budget, n_sink, n_recent, cap;
    int Hkv, max_pages_per_seq, num_pages;
};

// Weight -> unsigned key of the same order: NaN counts as minus infinity, -0 as 0.  Below 0xFFFFFFFF.
__device__ __forceinline__ uint32_t ev_key(float w)
{
    if (w != w) w = -INFINITY;
    const uint32_t u = __float_as_uint(w + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// What a block needs of its (sequence, kv head).
struct EvRow {
    int len, placed, seen;
    const float *w_in;
    float *w_out;
    const int32_t *pos_in;
    int32_t *pos_out;
    const int32_t *pages;
    __device__ __forceinline__ EvRow(const EvictParams &p, int b, int row)
    {
        len = min(min(max(__ldg(p.kv_len + b), 0), p.max_kv), p.max_pages_per_seq * kPageTokens);
        placed = (p.placed != nullptr) ? min(max(__ldg(p.placed + b), 0), len) : 0;
        seen = (p.seen != nullptr) ? __ldg(p.seen + b) : len;
        const size_t at = (size_t)row * p.stride;
        w_in = p.w_in + at;
        w_out = p.w_out + at;
        pos_in = p.pos_in + at;
        pos_out = p.pos_out + at;
        pages = p.block_table + (size_t)b * p.max_pages_per_seq;
    }
    __device__ __forceinline__ int position(int s) const { return (s < placed) ? pos_in[s] : seen - len + s; }
    __device__ __forceinline__ uint32_t key(const EvictParams &p, int s) const { return key_of(p, position(s), w_in[s]); }
    __device__ __forceinline__ uint32_t key_of(const EvictParams &p, int pos, float w) const
    {
        return (pos < p.n_sink || pos >= seen - p.n_recent) ? 0xFFFFFFFFu : ev_key(w);
    }
    __device__ __forceinline__ void keep(int to, int from) const
    {
        const float w = w_in[from];
        const int pos = position(from);
        w_out[to] = w;
        pos_out[to] = pos;
    }
    // The cache row (128 codes, one scale) of the K vector in a slot, -1 without a page; its V vector lies 128 rows behind.
    __device__ __forceinline__ int cache_row(const EvictParams &p, int head, int s) const
    {
        const int page = __ldg(pages + (s >> 7));
        return (page >= 0 && page < p.num_pages) ? (page * p.Hkv + head) * 2 * kPageTokens + (s & (kPageTokens - 1)) : -1;
    }
};

// One token's K row and V row and their scales, by sixteen lanes.
struct EvMove {
    uint4 piece;
    float scale;
    int to;        // cache row of the lane's vector, -1: nothing
};
__device__ __forceinline__ EvMove ev_fetch(const EvictParams &p, int from, int to, int l16)
{
    EvMove m;
    m.piece = make_uint4(0, 0, 0, 0);
    m.scale = 0.f;
    m.to = -1;
    if (from >= 0 && to >= 0) {
        const int v = (l16 >> 3) * kPageTokens;
        m.to = to + v;
        m.piece = *reinterpret_cast<const uint4 *>(p.codes + (size_t)(from + v) * kHeadDim + 16 * (l16 & 7));
        if ((l16 & 7) == 0) m.scale = p.scales[from + v];
    }
    return m;
}
__device__ __forceinline__ void ev_store(const EvictParams &p, const EvMove &m, int l16)
{
    if (m.to < 0) return;
    *reinterpret_cast<uint4 *>(p.codes + (size_t)m.to * kHeadDim + 16 * (l16 & 7)) = m.piece;
    if ((l16 & 7) == 0) p.scales[m.to] = m.scale;
}

// The digit (256 bins, counts of the keys that match the digits before it) in which the need-th largest key lies, by one
// warp; need becomes its rank inside the bin, count the bin's keys.
__device__ __forceinline__ uint32_t ev_digit(const uint32_t *hist, int lane, int &need, int &count)
{
    // lane l holds bins 255 - 8 l down to 248 - 8 l
    const uint4 a = *reinterpret_cast<const uint4 *>(hist + 252 - 8 * lane), b = *reinterpret_cast<const uint4 *>(hist + 248 - 8 * lane);
    const int c[8] = {(int)a.w, (int)a.z, (int)a.y, (int)a.x, (int)b.w, (int)b.z, (int)b.y, (int)b.x};
    int sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum += c[i];
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += v;
    }
    int before = incl - sum, bin = 0, rank = 0, n = 0;
    const bool mine = before < need && need <= incl;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (mine && before < need && need <= before + c[i]) bin = 255 - 8 * lane - i, rank = need - before, n = c[i];
        before += c[i];
    }
    const int src = __ffs(__ballot_sync(0xffffffffu, mine)) - 1;
    need = __shfl_sync(0xffffffffu, rank, src);
    count = __shfl_sync(0xffffffffu, n, src);
    return (uint32_t)__shfl_sync(0xffffffffu, bin, src);
}

// Shared memory of a selecting block.  Slot s of the block lies at index s + 4 (s / kPer) of w and pos, so that threads
// reading their kPer consecutive slots 16 bytes at a time fall into different banks.
template <int kThreads, int kPer, bool kCluster>
struct EvSmem {
    static constexpr int kSlots = kThreads * kPer;
    static constexpr int kPadded = kSlots + (kPer > 4 ? kThreads * 4 : 0);
    float w[kPadded];
    int pos[kPadded];
    union {
        struct {
            uint32_t hist[kEvBins];
            uint32_t total[kCluster ? kEvBins : 4];   // the row's histogram, then the row's listed keys
        };
        uint16_t slots[kSlots];               // later: the block's freed slots, then its moving ones
    };
    uint32_t list[kEvList];
    int n_list;
    uint16_t kept[kThreads];                  // bit i: the thread's slot i is kept
    int first_free, end_free, first_move, end_move;   // their ranks in the row
    uint2 extremes[32];
    int sums[32];
    int found[4];                             // bin, tokens above it, tokens in it;  or last key, greater, equal ones
    // what the other blocks of the row read
    uint2 block_extremes;
    int block_safe, block_equal, block_sum;
    __device__ static __forceinline__ int at(int s) { return kPer > 4 ? s + 4 * (s / kPer) : s; }
};

// Thread t of the row's block c owns the slots (c * kThreads + t) * kPer and the kPer - 1 behind it.
// (64 registers: four blocks of 256 threads per SM hold a batch of 512 rows at once)
template <int kThreads, int kPer, bool kCluster, bool kMove>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads)
slim_evict_select_kernel(const EvictParams p)
{
    using S = EvSmem<kThreads, kPer, kCluster>;
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(16) unsigned char ev_smem[];
    S &sm = *reinterpret_cast<S *>(ev_smem);
    __shared__ int list[kMove ? 3 * kEvBlockMoves : 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int n_blocks = kCluster ? (int)cg::this_cluster().num_blocks() : 1;
    const int rank = kCluster ? (int)cg::this_cluster().block_rank() : 0;
    const int b = blockIdx.y, head = (int)blockIdx.x / n_blocks;
    const int row = b * p.Hkv + head;
    const int base = rank * S::kSlots;          // the block's first slot
    // (barrier of the row's blocks; it also makes their shared memory visible to one another)
    auto sync_row = [&] {
        if constexpr (kCluster) cg::this_cluster().sync();
        else __syncthreads();
    };
    auto of_block = [&](auto *local, int c) {
        if constexpr (kCluster) return cg::this_cluster().map_shared_rank(local, c);
        else return local;
    };
    pdl_launch_dependents();
    pdl_wait();
    // weights and positions are requested before the row's length is known (a row has room for max_kv of each)
    float w_raw[kPer];
    int pos_raw[kPer];
    {
        const float *w_in = p.w_in + (size_t)row * p.stride + base;
        const int32_t *pos_in = p.pos_in + (size_t)row * p.stride + base;
#pragma unroll
        for (int i = 0; i < kPer; ++i) w_raw[i] = (base + tid + i * kThreads < p.max_kv) ? w_in[tid + i * kThreads] : 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) pos_raw[i] = (p.placed != nullptr && base + tid + i * kThreads < p.max_kv) ? pos_in[tid + i * kThreads] : 0;
    }
    for (int i = tid; i < kEvBins; i += kThreads) sm.hist[i] = 0;
    if (tid == 0) sm.n_list = 0;
    const EvRow r(p, b, row);
    const bool cut = r.len > p.budget;          // (the same for all of the row)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = base + tid + i * kThreads;
        if (base + i * kThreads >= r.len) break;   // (the same for the block: short rows leave the rest of it out)
        const int pos = (s < r.placed) ? pos_raw[i] : r.seen - r.len + s;
        if (!cut) {
            // nothing leaves: weights and positions as they are
            if (s < r.len) r.w_out[s] = w_raw[i], r.pos_out[s] = pos;
        } else {
            sm.w[S::at(tid + i * kThreads)] = w_raw[i];
            sm.pos[S::at(tid + i * kThreads)] = pos;
        }
    }
    if (!cut) {
        if (tid == 0 && rank == 0 && !kMove) p.n_moves[row] = 0;
        return;
    }
    __syncthreads();
    const int s0 = base + tid * kPer;           // the thread's first slot
    const bool any = s0 < r.len;                // the thread has slots of the row
    uint32_t key[kPer];                         // 0 behind the row's end (no token's key is 0)
    uint32_t lo = 0xFFFFFFFFu, hi = 0;          // smallest and largest key of the tokens that are not protected
    int safe = 0;                               // protected tokens
#pragma unroll
    for (int i = 0; i < kPer; ++i) key[i] = 0u;
    if (any) {
#pragma unroll
        for (int i4 = 0; i4 < kPer; i4 += 4) {
            const float4 w4 = *reinterpret_cast<const float4 *>(&sm.w[S::at(tid * kPer) + i4]);
            const int4 p4 = *reinterpret_cast<const int4 *>(&sm.pos[S::at(tid * kPer) + i4]);
            const float w[4] = {w4.x, w4.y, w4.z, w4.w};
            const int pos[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t k = (s0 + i4 + i < r.len) ? r.key_of(p, pos[i], w[i]) : 0u;
                key[i4 + i] = k;
                if (k == 0xFFFFFFFFu) ++safe;
                else if (k != 0u) lo = min(lo, k), hi = max(hi, k);
                }
    }
    }
    lo = __reduce_min_sync(0xffffffffu, lo);
    hi = __reduce_max_sync(0xffffffffu, hi);
    safe = __reduce_add_sync(0xffffffffu, safe);
    if (lane == 0) sm.extremes[warp] = make_uint2(lo, hi), sm.sums[warp] = safe;
    __syncthreads();
    {
        const uint2 e = (lane < kWarps) ? sm.extremes[lane] : make_uint2(0xFFFFFFFFu, 0u);
        lo = __reduce_min_sync(0xffffffffu, e.x);
        hi = __reduce_max_sync(0xffffffffu, e.y);
        safe = __reduce_add_sync(0xffffffffu, lane < kWarps ? sm.sums[lane] : 0);
        if constexpr (kCluster) {
            if (tid == 0) sm.block_extremes = make_uint2(lo, hi), sm.block_safe = safe;
            sync_row();
            const uint2 x = (lane < n_blocks) ? *of_block(&sm.block_extremes, lane) : make_uint2(0xFFFFFFFFu, 0u);
            const int n = (lane < n_blocks) ? *of_block(&sm.block_safe, lane) : 0;
            lo = __reduce_min_sync(0xffffffffu, x.x);
            hi = __reduce_max_sync(0xffffffffu, x.y);
            safe = __reduce_add_sync(0xffffffffu, n);
        }
    }

    // ---- the last key that is kept: of the `count` slots that hold `last`, the first `need` are kept, and every slot above
    uint32_t last = 0xFFFFFFFFu;
    int need = p.budget, count = safe;
    if (safe < p.budget) {
        need = p.budget - safe;
        int left = r.len - safe;                // tokens of [lo, hi]; need of them are kept
        for (;;) {
            // the tokens above lo, by equal steps of (lo, hi]
            const uint32_t width = hi - lo;     // 0: all of them are at lo
            const int shift = (width > kEvBins) ? 32 - __clz((int)((width - 1) >> 11)) : 0;
            if (any) {
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (key[i] > lo && key[i] <= hi) atomicAdd(&sm.hist[(key[i] - lo - 1) >> shift], 1u);
            }
            sync_row();
            const uint32_t *hist = sm.hist;
            if constexpr (kCluster) {
                for (int i = tid; i < kEvBins; i += kThreads) {
                    uint32_t n = 0;
#pragma unroll
                    for (int c = 0; c < kEvMaxCluster; ++c) n += (c < n_blocks) ? of_block(&sm.hist[0], c)[i] : 0u;   // (all on their way at once)
                    sm.total[i] = n;
                }
                hist = sm.total;
                __syncthreads();
            }
            // the bins from the largest down, kBinsPer of them per thread of the first warps
            constexpr int kBinsPer = 8, kBinWarps = kEvBins / kBinsPer / 32;
            if (warp < kBinWarps) {
                uint32_t c[kBinsPer];
                int sum = 0;
#pragma unroll
                for (int i = 0; i < kBinsPer; i += 4) {
                    const uint4 v = *reinterpret_cast<const uint4 *>(hist + kEvBins - 4 - kBinsPer * tid - i);
                    c[i] = v.w, c[i + 1] = v.z, c[i + 2] = v.y, c[i + 3] = v.x;
                    sum += (int)(v.x + v.y + v.z + v.w);
                }
                int incl = sum;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const int v = __shfl_up_sync(0xffffffffu, incl, o);
                    if (lane >= o) incl += v;
                }
                if (lane == 31) sm.sums[warp] = incl;
                asm volatile("bar.sync 1, %0;\n" ::"r"(kBinWarps * 32) : "memory");
                const int total = (lane < kBinWarps) ? sm.sums[lane] : 0;
                int before = __reduce_add_sync(0xffffffffu, lane < warp ? total : 0) + incl - sum;
                const int above_lo = __reduce_add_sync(0xffffffffu, total);
                if (tid == 0 && above_lo < need) sm.found[0] = -1, sm.found[1] = above_lo;   // the last kept key is lo
#pragma unroll
                for (int i = 0; i < kBinsPer; ++i) {
                    if (before < need && need <= before + (int)c[i]) sm.found[0] = kEvBins - 1 - kBinsPer * tid - i, sm.found[1] = before, sm.found[2] = (int)c[i];
                    before += (int)c[i];
                }
            }
            __syncthreads();
            const int bin = sm.found[0], above = sm.found[1], inside = sm.found[2];
            if (bin < 0) {
                last = lo, need -= above, count = left - above;
                break;
            }
            // the bin's keys
            const uint32_t first_key = lo + 1 + ((uint32_t)bin << shift), last_key = min(hi, first_key + ((1u << shift) - 1));
            need -= above;
            if (need == inside || shift == 0) {
                // all of the bin, or a single key
                last = first_key, count = inside;
                break;
            }
            if (inside <= kEvList) {
                // listed per block, then (in a cluster) all the blocks' lists in every block
                if (any) {
#pragma unroll
                    for (int i = 0; i < kPer; ++i)
                        if (key[i] >= first_key && key[i] <= last_key) sm.list[atomicAdd(&sm.n_list, 1)] = key[i];
                }
                sync_row();
                const uint32_t *all = sm.list;
                if constexpr (kCluster) {
                    static_assert(!kCluster || kThreads == kEvMaxCluster * kEvList, "a thread per listed key");
                    const int c = tid / kEvList, i = tid % kEvList;
                    int first = 0, n = 0;
#pragma unroll
                    for (int u = 0; u < kEvMaxCluster; ++u) {
                        const int m = (u < n_blocks) ? *of_block(&sm.n_list, u) : 0;
                        first += (u < c) ? m : 0;
                        n = (u == c) ? m : n;
                    }
                    if (i < n) sm.total[first + i] = of_block(&sm.list[0], c)[i];
                    all = sm.total;
                    __syncthreads();
                }
                for (int i = tid; i < inside; i += kThreads) {
                    const uint32_t k = all[i];
                    int greater = 0, equal = 0;
                    for (int j = 0; j < inside; ++j) greater += all[j] > k ? 1 : 0, equal += all[j] == k ? 1 : 0;
                    if (greater < need && need <= greater + equal) sm.found[0] = (int)k, sm.found[1] = greater, sm.found[2] = equal;   // (the same from equal keys)
                }
                __syncthreads();
                last = (uint32_t)sm.found[0], need -= sm.found[1], count = sm.found[2];
                break;
            }
            // a histogram of the bin alone: its keys are (first_key - 1, last_key], none of them at the new lo
            lo = first_key - 1, hi = last_key, left = inside;
            sync_row();                          // every block has read the histogram
            for (int i = tid; i < kEvBins; i += kThreads) sm.hist[i] = 0;
            __syncthreads();
        }
    }

    unsigned keep = 0;   // bit i: slot s0 + i is kept
    if (any) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) keep |= (key[i] != 0u && key[i] >= last) ? 1u << i : 0u;
    }
    // Exclusive prefix, over the row's threads, of a value per thread.
    auto row_prefix = [&](int v, int *block_value) {
        int incl = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        __syncthreads();                        // sums may still be read from before
        if (lane == 31) sm.sums[warp] = incl;
        __syncthreads();
        const int mine = (lane < kWarps) ? sm.sums[lane] : 0;
        int before = (int)__reduce_add_sync(0xffffffffu, lane < warp ? mine : 0) + incl - v;
        if constexpr (kCluster) {
            const int all = (int)__reduce_add_sync(0xffffffffu, mine);
            if (tid == 0) *block_value = all;
            sync_row();
            const int other = (lane < rank) ? *of_block(block_value, lane) : 0;
            before += (int)__reduce_add_sync(0xffffffffu, other);
        }
        return before;
    };
    if (need != count) {
        // some of the slots that hold the last key leave: those behind the first `need`
        unsigned equal = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) equal |= (key[i] == last) ? 1u << i : 0u;
        int at = row_prefix(__popc(equal), &sm.block_equal);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if ((equal >> i) & 1u) {
                if (at >= need) keep &= ~(1u << i);
                ++at;
            }
        }
    }
    const int low_n = min(max(p.budget - s0, 0), kPer);                          // the thread's slots below the budget
    const unsigned low = (low_n == 32) ? 0xFFFFFFFFu : (1u << low_n) - 1u;
    unsigned fr = ~keep & low, mv = keep & ~low;
    // both counts in one prefix: as many slots are freed as move, fewer than 65536
    const unsigned both = (unsigned)row_prefix((int)((unsigned)__popc(fr) << 16 | (unsigned)__popc(mv)), &sm.block_sum);
    int free_at = (int)(both >> 16), move_at = (int)(both & 0xFFFFu);
    const int move0 = move_at;
    // the block's freed and moving slots, each in order (their ranks in the row are consecutive), into shared memory, from
    // there in whole lines to the row's lists
    if (tid == 0) sm.first_free = free_at, sm.first_move = move_at;
    if (tid == kThreads - 1) sm.end_free = free_at + __popc(fr), sm.end_move = move_at + __popc(mv);
    sm.kept[tid] = (uint16_t)keep;
    __syncthreads();
    const int free0 = sm.first_free, n_free = sm.end_free - free0, n_move = sm.end_move - sm.first_move;
    {
        uint16_t *at = sm.slots + (free_at - free0);
        for (unsigned m = fr; m; m &= m - 1) *at++ = (uint16_t)(tid * kPer + __ffs(m) - 1);
        at = sm.slots + n_free + (move_at - sm.first_move);
        for (unsigned m = mv; m; m &= m - 1) *at++ = (uint16_t)(tid * kPer + __ffs(m) - 1);
    }
    __syncthreads();
    const int cap = kMove ? kEvBlockMoves : p.cap;
    int32_t *freed = kMove ? list : p.moves + (size_t)row * 3 * cap, *freed_row = freed + cap, *moving_row = freed_row + cap;
    for (int i = tid; i < n_free + n_move; i += kThreads) {
        const int s = base + sm.slots[i];
        const int cache_row = r.cache_row(p, head, s);
        if (i < n_free) freed[free0 + i] = s, freed_row[free0 + i] = cache_row;
        else moving_row[sm.first_move + i - n_free] = cache_row;
    }
    if (!kMove && rank == n_blocks - 1 && tid == 0) p.n_moves[row] = sm.end_move;   // the row's last slots' end: all of its moves
    sync_row();                                  // the list of freed slots is complete (and no block's shared memory is reached from another any more)
    // ---- the moving slots' weights and positions to the freed slots
    {
        int to[kPer];
        if (mv != 0u) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int at = move0 + __popc(mv & ((1u << i) - 1u));
                to[i] = !((mv >> i) & 1u) ? -1 : kMove ? freed[at] : __ldcg(freed + at);
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                if (to[i] >= 0) {
                    r.w_out[to[i]] = sm.w[S::at(tid * kPer) + i];
                    r.pos_out[to[i]] = sm.pos[S::at(tid * kPer) + i];
                }
            }
        }
    }
    if (kMove) {
        const int n = sm.end_move;
        for (int i = tid >> 4; i < n; i += kThreads / 16) ev_store(p, ev_fetch(p, moving_row[i], freed_row[i], tid & 15), tid & 15);
    }
    // ---- the others stay where they are (whole lines)
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int s = tid + i * kThreads;
        if (base + i * kThreads >= p.budget) break;
        if (base + s < p.budget && ((sm.kept[s / kPer] >> (s % kPer)) & 1u)) {
            r.w_out[base + s] = sm.w[S::at(s)];
            r.pos_out[base + s] = sm.pos[S::at(s)];
        }
    }
}

// Rows of any length: one block, the keys formed anew from weights and positions for every digit and every walk.
__global__ void __launch_bounds__(1024)
slim_evict_select_long_kernel(const EvictParams p)
{
    constexpr int kThreads = 1024, kWarps = 32;
    __shared__ __align__(16) uint32_t hist[4][256];
    __shared__ int warp_n[32], all_moves;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.y, head = blockIdx.x, row = b * p.Hkv + head;
    pdl_launch_dependents();
    (&hist[0][0])[tid] = 0;
    pdl_wait();
    const EvRow r(p, b, row);
    const int len = r.len;
    if (len <= p.budget) {
        for (int s = tid; s < len; s += kThreads) r.keep(s, s);
        if (tid == 0) p.n_moves[row] = 0;
        return;
    }
    __syncthreads();
    uint32_t prefix = 0;
    int need = p.budget, count = 0;
    for (int pass = 0; pass < 4; ++pass) {
        const int shift = 24 - 8 * pass;
        for (int s = tid; s < len; s += kThreads) {
            const uint32_t k = r.key(p, s);
            if (pass == 0 || (k >> (shift + 8)) == (prefix >> (shift + 8))) {
                // one addition per bin and warp
                const uint32_t bin = (k >> shift) & 255u;
                const unsigned peers = __match_any_sync(__activemask(), bin);
                if (lane == __ffs(peers) - 1) atomicAdd(&hist[pass][bin], (uint32_t)__popc(peers));
            }
        }
        __syncthreads();
        prefix |= ev_digit(hist[pass], lane, need, count) << shift;
    }
    auto block_prefix = [&](int n) {
        __syncthreads();
        if (lane == 0) warp_n[warp] = n;
        __syncthreads();
        return __reduce_add_sync(0xffffffffu, lane < warp ? warp_n[lane] : 0);
    };
    const int run = ((len + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int s0 = min(warp * run, len), s1 = min(s0 + run, len);
    const unsigned lower = (1u << lane) - 1u;
    int equal = 0;
    for (int s = s0; s < s1; s += 32) equal += __popc(__ballot_sync(0xffffffffu, s + lane < s1 && r.key(p, s + lane) == prefix));
    const int equal0 = block_prefix(equal);
    // walks the warp's slots in order; visit(slot, kept) sees 32 of them at a time
    auto walk = [&](auto visit) {
        int at = equal0;
        for (int s = s0; s < s1; s += 32) {
            const bool in = s + lane < s1;
            const uint32_t k = in ? r.key(p, s + lane) : 0u;
            const unsigned eq = __ballot_sync(0xffffffffu, in && k == prefix);
            visit(s + lane, in, in && (k > prefix || (k == prefix && at + __popc(eq & lower) < need)));
            at += __popc(eq);
        }
    };
    int free_n = 0, move_n = 0;
    walk([&](int s, bool in, bool kept) {
        free_n += __popc(__ballot_sync(0xffffffffu, in && s < p.budget && !kept));
        move_n += __popc(__ballot_sync(0xffffffffu, s >= p.budget && kept));
    });
    int free_at = block_prefix(free_n), move_at = block_prefix(move_n);
    int32_t *freed = p.moves + (size_t)row * 3 * p.cap, *freed_row = freed + p.cap, *moving_row = freed_row + p.cap;
    // the lists, and the slots that stay: what is written here in place of an input is what stands there, so the walk's keys hold
    walk([&](int s, bool in, bool kept) {
        const unsigned fr = __ballot_sync(0xffffffffu, in && s < p.budget && !kept), mv = __ballot_sync(0xffffffffu, s >= p.budget && kept);
        if (in && s < p.budget && !kept) {
            const int at = free_at + __popc(fr & lower);
            freed[at] = s;
            freed_row[at] = r.cache_row(p, head, s);
        }
        if (s >= p.budget && kept) moving_row[move_at + __popc(mv & lower)] = s;   // (the slot, until the lists are complete)
        if (s < p.budget && kept) r.keep(s, s);
        free_at += __popc(fr);
        move_at += __popc(mv);
    });
    if (warp == kWarps - 1 && lane == 0) all_moves = p.n_moves[row] = move_at;
    __syncthreads();   // every key has been read: from here on freed slots are overwritten where the outputs are the inputs
    for (int i = tid, n = all_moves; i < n; i += kThreads) {
        const int s = __ldcg(moving_row + i);
        r.keep(__ldcg(freed + i), s);
        moving_row[i] = r.cache_row(p, head, s);
    }
}

// The rows of every (sequence, kv head): sixteen lanes per row, four rows in flight.
__global__ void __launch_bounds__(256)
slim_evict_move_kernel(const EvictParams p)
{
    const int row = (int)blockIdx.z * p.Hkv + (int)blockIdx.y;
    const int l16 = threadIdx.x & 15, first = (int)blockIdx.x * kEvBlockMoves + (threadIdx.x >> 4);
    const int32_t *freed_row = p.moves + (size_t)row * 3 * p.cap + p.cap, *moving_row = freed_row + p.cap;
    pdl_wait();
    // the lists are read before it is known how many of their entries count
    int from[kEvBlockMoves / 16], to[kEvBlockMoves / 16];
#pragma unroll
    for (int u = 0; u < kEvBlockMoves / 16; ++u) {
        const int i = min(first + 16 * u, p.cap - 1);
        from[u] = __ldcg(moving_row + i);
        to[u] = __ldcg(freed_row + i);
    }
    const int n = __ldcg(p.n_moves + row);
    EvMove m[kEvBlockMoves / 16];
#pragma unroll
    for (int u = 0; u < kEvBlockMoves / 16; ++u) m[u] = ev_fetch(p, (first + 16 * u < n) ? from[u] : -1, to[u], l16);
#pragma unroll
    for (int u = 0; u < kEvBlockMoves / 16; ++u) ev_store(p, m[u], l16);
}

// ---------------------------------------------------------------- host side
static int evict_cap(int max_kv, int budget) { return max_kv > budget ? (budget < max_kv - budget ? budget : max_kv - budget) : 0; }

size_t evict_workspace_bytes(int B, int Hkv, int max_kv, int budget)
{
    return (size_t)B * Hkv * (1 + 3 * (size_t)evict_cap(max_kv, budget)) * sizeof(int32_t);
}

template <int kThreads, int kPer, bool kCluster, bool kMove>
static int launch_select(const EvictParams &p, int B, int cluster, cudaStream_t stream)
{
    constexpr int bytes = (int)sizeof(EvSmem<kThreads, kPer, kCluster>);
    const int rc = allow_dynamic_smem(reinterpret_cast<const void *>(slim_evict_select_kernel<kThreads, kPer, kCluster, kMove>), bytes);
    if (rc != SLIM_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.Hkv * cluster), (unsigned)B);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = bytes;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = kCluster ? 2 : 1;
    SLIM_CUDA_TRY(cudaLaunchKernelEx(&cfg, slim_evict_select_kernel<kThreads, kPer, kCluster, kMove>, p));
    return SLIM_OK;
}

// The smallest block (or cluster) that holds the longest row's keys.
template <bool kMove>
static int launch_select_any(const EvictParams &p, int B, cudaStream_t stream)
{
    if (p.max_kv <= 256 * 4) return launch_select<256, 4, false, kMove>(p, B, 1, stream);
    if (p.max_kv <= 256 * 8) return launch_select<256, 8, false, kMove>(p, B, 1, stream);
    if (p.max_kv <= 256 * 16) return launch_select<256, 16, false, kMove>(p, B, 1, stream);
    if (p.max_kv <= kEvBlockTokens) return launch_select<1024, kEvItems, false, kMove>(p, B, 1, stream);
    if constexpr (!kMove) {
        if (p.max_kv <= 2 * kEvBlockTokens) return launch_select<1024, kEvItems, true, false>(p, B, 2, stream);
        if (p.max_kv <= 4 * kEvBlockTokens) return launch_select<1024, kEvItems, true, false>(p, B, 4, stream);
        if (p.max_kv <= kEvMaxCluster * kEvBlockTokens) return launch_select<1024, kEvItems, true, false>(p, B, kEvMaxCluster, stream);
        // (the counts of freed and moving slots share 32 bits)
        if (p.max_kv <= 2 * kEvMaxCluster * kEvBlockTokens && p.cap < 65536) return launch_select<1024, 2 * kEvItems, true, false>(p, B, kEvMaxCluster, stream);
    }
    SLIM_CUDA_TRY(launch_pdl(slim_evict_select_long_kernel, dim3((unsigned)p.Hkv, (unsigned)B), dim3(1024), 0, stream, p));
    return SLIM_OK;
}

int launch_evict(const slim_cache_t *c, const float *w_in, float *w_out, const int32_t *pos_in, int32_t *pos_out, int stride,
                 const int32_t *kv_len, const int32_t *placed, const int32_t *seen, int B, int max_kv, int budget, int n_sink,
                 int n_recent, void *workspace, cudaStream_t stream)
{
    EvictParams p;
    p.codes = c->codes;
    p.scales = c->scales;
    p.block_table = c->block_table;
    p.w_in = w_in;
    p.w_out = w_out;
    p.pos_in = pos_in;
    p.pos_out = pos_out;
    p.kv_len = kv_len;
    p.placed = placed;
    p.seen = seen;
    p.n_moves = static_cast<int32_t *>(workspace);
    p.moves = p.n_moves + (size_t)B * c->num_kv_heads;
    p.stride = stride;
    p.max_kv = max_kv;
    p.budget = budget;
    p.n_sink = n_sink;
    p.n_recent = n_recent;
    p.cap = evict_cap(max_kv, budget);
    p.Hkv = c->num_kv_heads;
    p.max_pages_per_seq = c->max_pages_per_seq;
    p.num_pages = c->num_pages;
    // (cache rows are 32-bit numbers: 2^31 of them are 274 GB of codes)
    if ((long long)c->num_pages * c->num_kv_heads * 2 * kPageTokens > 0x7FFFFFFFLL) return SLIM_ERR_UNSUPPORTED;
    if ((long long)c->num_kv_heads * kEvMaxCluster > 0x7FFFFFFFLL) return SLIM_ERR_UNSUPPORTED;
    if (p.cap <= kEvBlockMoves && max_kv <= kEvBlockTokens) return launch_select_any<true>(p, B, stream);
    const int rc = launch_select_any<false>(p, B, stream);
    if (rc != SLIM_OK || p.cap == 0) return rc;
    const dim3 grid((unsigned)((p.cap + kEvBlockMoves - 1) / kEvBlockMoves), (unsigned)p.Hkv, (unsigned)B);
    SLIM_CUDA_TRY(launch_pdl(slim_evict_move_kernel, grid, dim3(256), 0, stream, p));
    return SLIM_OK;
}

}  // namespace slim

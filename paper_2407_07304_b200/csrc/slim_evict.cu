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
// Selection: one block per (sequence, kv head).  A weight is mapped to an unsigned integer of the same order (a
// protected token to the largest one), the budget-th largest key is found by three histogram passes over its 11, 11
// and 10 bits, and a second walk in slot order, 32 slots per warp and step, counts and then lists the freed and the
// moving slots.  The keys stay in shared memory between the passes where they fit (up to 53248 tokens), so the
// weights are read once.  Nothing depends on the order of the atomic additions (counts), so equal inputs give equal
// results.  Bound by latency: 4 bytes per token are read, beside 264 per moved token.
#include "slim_common.cuh"
#include "slim_tmap.cuh"

namespace slim {

constexpr int kEvBins = 2048;
constexpr int kEvSmemTokens = 53248;      // keys that fit the shared memory beside the histogram (208 KB)
constexpr int kEvMovesPerBlock = 64;      // moves of one block of the move kernel

struct EvictParams {
    int8_t *codes;
    float *scales;
    const int32_t *block_table;
    const float *w_in;
    float *w_out;
    const int32_t *pos_in;
    int32_t *pos_out;
    const int32_t *kv_len, *placed, *seen;
    int32_t *moves;        // [rows][2][cap]: freed slots, moving slots
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

// One token of (sequence b, kv head) from slot `from` to slot `to`, by sixteen lanes: the K row's eight 16-byte pieces,
// the V row's eight, the two scales.
struct EvRow {
    uint4 piece;
    float scale;
    int8_t *dst;
    float *dst_scale;
    bool ok;
};
__device__ __forceinline__ EvRow ev_fetch(const EvictParams &p, int b, int head, int from, int to, int l16)
{
    EvRow r;
    const int32_t *bt = p.block_table + (size_t)b * p.max_pages_per_seq;
    const int page_from = __ldg(bt + (from >> 7)), page_to = __ldg(bt + (to >> 7));
    r.ok = page_from >= 0 && page_from < p.num_pages && page_to >= 0 && page_to < p.num_pages;
    r.piece = make_uint4(0, 0, 0, 0);
    r.scale = 0.f;
    r.dst = nullptr;
    r.dst_scale = nullptr;
    if (r.ok) {
        const int kv = l16 >> 3, c = l16 & 7;
        const int sf = from & (kPageTokens - 1), st = to & (kPageTokens - 1);
        r.piece = *reinterpret_cast<const uint4 *>(p.codes + code_block_offset(page_from, head, kv, p.Hkv) + (size_t)sf * kHeadDim + 16 * c);
        r.dst = p.codes + code_block_offset(page_to, head, kv, p.Hkv) + (size_t)st * kHeadDim + 16 * c;
        if (c == 0) {
            r.scale = p.scales[scale_block_offset(page_from, head, kv, p.Hkv) + sf];
            r.dst_scale = p.scales + scale_block_offset(page_to, head, kv, p.Hkv) + st;
        }
    }
    return r;
}
__device__ __forceinline__ void ev_store(const EvRow &r)
{
    if (!r.ok) return;
    *reinterpret_cast<uint4 *>(r.dst) = r.piece;
    if (r.dst_scale != nullptr) *r.dst_scale = r.scale;
}

// Exclusive prefix of one value per warp over the block's warps (kWarps <= 32), for the calling warp; all threads call it.
template <int kWarps>
__device__ __forceinline__ int ev_warp_prefix(int *buf, int warp, int lane, int value)
{
    if (lane == 0) buf[warp] = value;
    __syncthreads();
    const int v = (lane < kWarps && lane < warp) ? buf[lane] : 0;
    const int sum = __reduce_add_sync(0xffffffffu, v);
    __syncthreads();   // buf may be used again
    return sum;
}

template <int kThreads, bool kInSmem, bool kMove>
__global__ void __launch_bounds__(kThreads)
slim_evict_select_kernel(const EvictParams p)
{
    constexpr int kWarps = kThreads / 32;
    extern __shared__ __align__(16) uint32_t ev_smem[];
    uint32_t *hist = ev_smem, *keys = ev_smem + kEvBins;
    __shared__ int buf[32];
    __shared__ uint32_t found[2];   // chosen bin, keys still to take from it
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.y, head = blockIdx.x;
    const int row = b * p.Hkv + head;
    pdl_launch_dependents();
    pdl_wait();
    const int len = min(min(max(__ldg(p.kv_len + b), 0), p.max_kv), p.max_pages_per_seq * kPageTokens);
    const int placed = (p.placed != nullptr) ? min(max(__ldg(p.placed + b), 0), len) : 0;
    const int seen = (p.seen != nullptr) ? __ldg(p.seen + b) : len;
    const float *w_in = p.w_in + (size_t)row * p.stride;
    float *w_out = p.w_out + (size_t)row * p.stride;
    const int32_t *pos_in = p.pos_in + (size_t)row * p.stride;
    int32_t *pos_out = p.pos_out + (size_t)row * p.stride;
    auto position = [&](int s) { return (s < placed) ? pos_in[s] : seen - len + s; };
    auto make_key = [&](int s) {
        const int pos = position(s);
        return (pos < p.n_sink || pos >= seen - p.n_recent) ? 0xFFFFFFFFu : ev_key(w_in[s]);
    };
    auto key = [&](int s) { return kInSmem ? keys[s] : make_key(s); };
    if (len <= p.budget) {
        // nothing leaves: weights and positions as they are
        for (int s = tid; s < len; s += kThreads) {
            const int pos = position(s);
            const float w = w_in[s];
            w_out[s] = w;
            pos_out[s] = pos;
        }
        if (tid == 0) p.n_moves[row] = 0;
        return;
    }

    // ---- the budget-th largest key
    uint32_t prefix = 0, mask = 0;
    int need = p.budget;   // keys to take among those that match the prefix
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = (pass == 0) ? 21 : (pass == 1) ? 10 : 0;
        const int bins = (pass == 2) ? 1024 : 2048;
        for (int i = tid; i < kEvBins; i += kThreads) hist[i] = 0;
        __syncthreads();
        for (int s = tid; s < len; s += kThreads) {
            uint32_t k;
            if (kInSmem && pass == 0) keys[s] = k = make_key(s);
            else k = key(s);
            if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (uint32_t)(bins - 1)], 1u);
        }
        __syncthreads();
        // the bins from the largest down, kEvBins / kThreads consecutive ones per thread
        constexpr int kPer = kEvBins / kThreads;
        int c[kPer], sum = 0;
#pragma unroll
        for (int i = 0; i < kPer; ++i) c[i] = (int)hist[kEvBins - 1 - (tid * kPer + i)], sum += c[i];   // (the upper half is empty in the last pass)
        int incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        int before = ev_warp_prefix<kWarps>(buf, warp, lane, __shfl_sync(0xffffffffu, incl, 31)) + incl - sum;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            if (before < need && need <= before + c[i]) {
                found[0] = (uint32_t)(kEvBins - 1 - (tid * kPer + i));
                found[1] = (uint32_t)(need - before);
            }
            before += c[i];
        }
        __syncthreads();
        prefix |= found[0] << shift;
        mask |= (uint32_t)(bins - 1) << shift;
        need = (int)found[1];
        // (found is written again only after the barriers of the next pass)
    }
    const uint32_t last = prefix;   // keys above it are kept, and the first `need` slots that hold it

    // ---- in slot order: every warp owns a contiguous run of slots
    const int run = ((len + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int s0 = min(warp * run, len), s1 = min(s0 + run, len);
    int equal = 0;
    for (int s = s0; s < s1; s += 32) equal += __popc(__ballot_sync(0xffffffffu, s + lane < s1 && key(s + lane) == last));
    const int equal0 = ev_warp_prefix<kWarps>(buf, warp, lane, equal);
    const unsigned lower = (1u << lane) - 1u;
    int free_n = 0, move_n = 0;
    {
        int rank = equal0;
        for (int s = s0; s < s1; s += 32) {
            const bool in = s + lane < s1;
            const uint32_t k = in ? key(s + lane) : 0u;
            const unsigned eq = __ballot_sync(0xffffffffu, in && k == last);
            const bool keep = in && (k > last || (k == last && rank + __popc(eq & lower) < need));
            rank += __popc(eq);
            const bool low = s + lane < p.budget;
            free_n += __popc(__ballot_sync(0xffffffffu, in && low && !keep));
            move_n += __popc(__ballot_sync(0xffffffffu, keep && !low));
        }
    }
    int free_at = ev_warp_prefix<kWarps>(buf, warp, lane, free_n);
    int move_at = ev_warp_prefix<kWarps>(buf, warp, lane, move_n);
    int32_t *freed = p.moves + (size_t)row * 2 * p.cap, *moving = freed + p.cap;
    {
        int rank = equal0;
        for (int s = s0; s < s1; s += 32) {
            const int slot = s + lane;
            const bool in = slot < s1;
            const uint32_t k = in ? key(slot) : 0u;
            const unsigned eq = __ballot_sync(0xffffffffu, in && k == last);
            const bool keep = in && (k > last || (k == last && rank + __popc(eq & lower) < need));
            rank += __popc(eq);
            const bool low = slot < p.budget;
            const unsigned fr = __ballot_sync(0xffffffffu, in && low && !keep), mv = __ballot_sync(0xffffffffu, keep && !low);
            if (in && low && !keep) freed[free_at + __popc(fr & lower)] = slot;
            if (keep && !low) moving[move_at + __popc(mv & lower)] = slot;
            if (keep && low) {
                const float w = w_in[slot];
                const int pos = position(slot);
                w_out[slot] = w;
                pos_out[slot] = pos;
            }
            free_at += __popc(fr);
            move_at += __popc(mv);
        }
    }
    __syncthreads();   // the lists are complete (written and read by this block only, up to here)
    const int n = [&] {   // as many slots move as were freed: the last warp's count
        if (warp == kWarps - 1 && lane == 0) buf[0] = move_at;
        __syncthreads();
        return buf[0];
    }();
    for (int i = tid; i < n; i += kThreads) {
        const int to = freed[i], from = moving[i];
        const float w = w_in[from];
        const int pos = position(from);
        w_out[to] = w;
        pos_out[to] = pos;
    }
    if (kMove) {
        for (int i = tid >> 4; i < n; i += kThreads / 16) ev_store(ev_fetch(p, b, head, moving[i], freed[i], tid & 15));
    } else if (tid == 0) {
        p.n_moves[row] = n;
    }
}

// The rows of every (sequence, kv head): sixteen lanes per row, four rows in flight.
__global__ void __launch_bounds__(256)
slim_evict_move_kernel(const EvictParams p)
{
    const int b = blockIdx.z, head = blockIdx.y;
    const int row = b * p.Hkv + head;
    const int l16 = threadIdx.x & 15, half = threadIdx.x >> 4;
    pdl_wait();
    const int n = __ldcg(p.n_moves + row);
    const int first = (int)blockIdx.x * kEvMovesPerBlock + half;
    const int32_t *freed = p.moves + (size_t)row * 2 * p.cap, *moving = freed + p.cap;
    EvRow r[kEvMovesPerBlock / 16];
#pragma unroll
    for (int u = 0; u < kEvMovesPerBlock / 16; ++u) {
        const int i = first + 16 * u;
        r[u].ok = false;
        if (i < n) r[u] = ev_fetch(p, b, head, __ldcg(moving + i), __ldcg(freed + i), l16);
    }
#pragma unroll
    for (int u = 0; u < kEvMovesPerBlock / 16; ++u) ev_store(r[u]);
}

// ---------------------------------------------------------------- host side
static int evict_cap(int max_kv, int budget) { return max_kv > budget ? (budget < max_kv - budget ? budget : max_kv - budget) : 0; }

size_t evict_workspace_bytes(int B, int Hkv, int max_kv, int budget)
{
    return (size_t)B * Hkv * (1 + 2 * (size_t)evict_cap(max_kv, budget)) * sizeof(int32_t);
}

template <int kThreads, bool kInSmem, bool kMove>
static int launch_select(const EvictParams &p, int B, cudaStream_t stream)
{
    const int bytes = (kEvBins + (kInSmem ? p.max_kv : 0)) * (int)sizeof(uint32_t);
    const int rc = allow_dynamic_smem(reinterpret_cast<const void *>(slim_evict_select_kernel<kThreads, kInSmem, kMove>),
                                      (kEvBins + (kInSmem ? kEvSmemTokens : 0)) * (int)sizeof(uint32_t));
    if (rc != SLIM_OK) return rc;
    SLIM_CUDA_TRY(launch_pdl(slim_evict_select_kernel<kThreads, kInSmem, kMove>, dim3((unsigned)p.Hkv, (unsigned)B), dim3(kThreads), bytes, stream, p));
    return SLIM_OK;
}

template <bool kMove>
static int launch_select_any(const EvictParams &p, int B, cudaStream_t stream)
{
    if (p.max_kv > kEvSmemTokens) return launch_select<1024, false, kMove>(p, B, stream);
    if (p.max_kv > 8192) return launch_select<1024, true, kMove>(p, B, stream);
    return launch_select<256, true, kMove>(p, B, stream);
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
    // few rows to move: by the block that chose them; many: by a second kernel over all the SMs
    if (p.cap <= kEvMovesPerBlock) return launch_select_any<true>(p, B, stream);
    const int rc = launch_select_any<false>(p, B, stream);
    if (rc != SLIM_OK) return rc;
    const dim3 grid((unsigned)((p.cap + kEvMovesPerBlock - 1) / kEvMovesPerBlock), (unsigned)p.Hkv, (unsigned)B);
    SLIM_CUDA_TRY(launch_pdl(slim_evict_move_kernel, grid, dim3(256), 0, stream, p));
    return SLIM_OK;
}

}  // namespace slim

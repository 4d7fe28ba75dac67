// Decode attention over the 4-bit KV cache (sm_100a).
//
// For every (sequence, kv head) pair, its G = Hq / Hkv query rows and cached tokens j with codes u, scale s and offset z:
//   score_j = c (s_j q.u_j + z_j sum q),   p = softmax(score),   o_d = sum_j (p_j s_j) u_jd + sum_j p_j z_j.
// The step is bound by memory: 136 bytes per token and kv head, read once.  At the copy rate an SM gets 22 of them per
// clock, which is what the design follows from:
//
//  * The codes are multiplied as they come out of shared memory, in registers (mma.sync m16n8k16, fp16 in, fp32 sums).
//    The tensor cores of tcgen05 take 4-bit integers from nowhere: the codes would have to be written back to shared
//    memory as bytes, and the copy engine's writes, that expansion (read and write) and the operand reads are 192 KB of
//    shared-memory traffic per 256 tokens, 1500 clocks against the 780 that the stream allows.  The product needs 352
//    multiply-adds per clock and SM (eight query rows), a third of what the register form gives.
//  * A code is made an fp16 operand by a mask alone: as the low bits of an fp16 number u is the subnormal u 2^-24, four
//    bits further up u 2^-20, and the tensor cores take subnormals as they are.  Eight codes cost four masks and a shift.
//    The powers of two go into the query (for the dims of the high halves 2^-4 less) and into the results.
//  * The order of dims inside a product is free, so a lane's 16 bytes of a K row are its share of eight products' operands;
//    the scores of S^T = K Q^T become the operand P^T of O^T = V^T P^T by an 8x8 transposition (movmatrix), and V's
//    token pairs by a byte permutation.  Nothing but raw rows passes through shared memory.
//  * Warps are independent: each has its own ring of 64-token units (the copy engine's boxes have rows of 1 KB: it takes a
//    box row by row, and rows of 64 bytes cost 1 us on 143 MB), its own contiguous range of the units of all pairs, and its own
//    running maximum, sum and O in registers.  A pair that begins and ends inside a warp's range is written as the result
//    at once; the others leave a record, merged by the block, and where a pair spans blocks, by the block that finishes it
//    last, or by a second kernel where few pairs span many blocks.
//  * A K product needs the query, then a softmax step, then V: with twelve warps per SM these phases overlap across warps
//    (32 x 4096 tokens, 64 / 8 heads: 34.9 us, with eight warps 36.8; 4 x 640 tokens, 32 / 32 heads: 7.8 and 10.4; only
//    where a few warps have work are eight faster: 272 tokens, 32 / 32 heads, 6.7 and 6.5.  Sixteen
//    warps at 128 registers, in an earlier form: 46 us where twelve took 37.)
//
// Measured (B200, calls back to back, three caches in turn; the copy rate is 6.57 TB/s): 16 x 2049 tokens, 32 / 32 heads 38 us
// for 143 MB, the new rows' append and their read-back included; 32 ragged sequences of up to 4096 tokens, 64 / 8 heads, 27.5 us
// for 93 MB; one of 32768 tokens, 32 / 2 heads, 17.5 us for 9 MB; one of 272 tokens, 32 / 32 heads, 6.8 us.  Between 144 and 573 MB
// with eight query heads per kv head the stream runs at 6.1 TB/s (573 MB: 108 us); a call
// carries 2.3 us to its first products and 5 to 8 us from the median warp's last unit to its end (the slowest warp, the block's
// merge, the round trips of the merge between blocks).  With more than eight query heads per kv head the products bound it:
// eight warps of 255 registers, 3.9 TB/s (64 x 32768 tokens, 32 / 2 heads, 571 MB: 147 us).
//
// Query rows are held as fp16 after division by a power of two near the row's largest value: exact down to 2^-24 of it.
// The weights p_j s_j are rounded to fp16 (2^-11 of each, 2^-34 of the largest scale at least), p_j itself, its sum and the offset's
// sum stay fp32.
// Every wait is bounded; a wait that runs out raises the status word and the warp writes nothing more.
#include <cuda.h>

#include "slim4_common.cuh"
#include "slim_decode_params.cuh"
#include "slim_tcgen05.cuh"
#include "slim_tmap.cuh"

namespace slim {

constexpr int kD4Unit = 64;                        // tokens whose scores a warp holds at a time
constexpr uint32_t kD4CodeBytes = kD4Unit * kRow4Bytes;
constexpr uint32_t kD4PairBytes = 2 * kD4Unit * 4;   // its (scale, offset) words, K's and then V's
constexpr float kD4Grow = 4.f;                     // the running maximum moves when it is exceeded by 2^4
constexpr float kD4Top = 512.f;                    // p s is scaled so that the largest s counts as 2^9 to 2^10 (with p <= 2^4 far below fp16's 2^16)
constexpr int kD4MaxBlocks = 160;
constexpr int kD4Few = 8;                          // blocks per pair up to which the last of them merges their records

struct Decode4Params {
    uint8_t *codes;
    uint32_t *pairs;
    const int32_t *block_table;
    const int32_t *kv_len;
    const __nv_bfloat16 *q, *k_new, *v_new;
    __nv_bfloat16 *out;
    int *status;
    int *counters;      // arrivals, per block for the pair that begins in it; null: a second kernel merges the pairs that span blocks
    float *parts;       // two records per block: of the pair at its start and of the one at its end, where they go on in others
    int B, Hq, Hkv, G, max_pages_per_seq, num_pages, cap_tokens;
    float scale_log2e;
};

// A record: O [G][128], then m [G] and l [G].
__host__ __device__ inline int d4_rec_floats(int G) { return (G * (kHeadDim + 2) + 3) / 4 * 4; }

// A pair that a block shares with others: where it lies and what the blocks leave of it.
struct D4Span {
    int pair, first, units;   // -1: none; its units in the order of all units
    int block, parts;         // the block in which it begins, the records that blocks leave of it
    int slot0;                // which of the two records of that first block it is (always the first one of the later blocks)
    int pad[2];
};

// What a block is made of, by the query heads that a kv head serves at most: NT groups of eight columns of the products.
// A warp's ring of S slots (the K or the V codes of a unit each): with four, units n and n + 1; with three, K(n) goes behind
// V(n - 2) and V(n) behind K(n - 1).
template <int kHeads>
struct D4 {
    static constexpr int NT = (kHeads + 7) / 8;
    static constexpr int kWarps = (kHeads <= 8) ? 12 : 8;
    static constexpr int S = (kHeads > 2 && kHeads <= 8) ? 3 : 4;   // (what shared memory holds beside the records)
    static constexpr uint32_t kWarpCodes = S * kD4CodeBytes;
    static constexpr uint32_t kPairs = kWarps * kWarpCodes;                      // two units' words per warp
    static constexpr uint32_t kRecBytes = kHeads * (kHeadDim + 2) * 4;
    static constexpr uint32_t kFirst = kPairs + kWarps * 2 * kD4PairBytes;       // records of the warps' first pairs
    static constexpr uint32_t kSpans = kFirst + kWarps * kRecBytes;               // D4Span [2]: of the block's first and last unit
    static constexpr uint32_t kLeft = kSpans + 2 * sizeof(D4Span);                // int [2 * warps]: the pair of a warp's first, last record
    // (record e: of warp e / 2, its first or its last one)
    static __host__ __device__ __forceinline__ constexpr uint32_t record(int e) { return (e & 1) ? (e >> 1) * kWarpCodes : kFirst + (e >> 1) * kRecBytes; }
    static constexpr uint32_t kBars = (kLeft + 2 * kWarps * 4 + 7) / 8 * 8;
    static constexpr uint32_t kFlags = (kBars + kWarps * S * 8 + 15) / 16 * 16;   // int[4]
    static constexpr uint32_t kBytes = kFlags + 16;
    static_assert(kRecBytes <= kWarpCodes, "a warp's last record goes into its ring");
    static_assert(2 * kWarps <= 32, "a warp's lanes look at all records of the block");
    static_assert(kBytes <= 232448, "shared memory of one block");
};

__device__ __forceinline__ void d4_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same from zero
__device__ __forceinline__ void d4_mma0(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// A wait that did not succeed at once; false where it ran out.
__device__ __noinline__ bool d4_wait(uint32_t bar, uint32_t parity, const volatile int *failed)
{
    return tc::mbar_wait(bar, parity, *failed != 0 ? 1u : (1u << 18), failed);
}
__device__ __forceinline__ uint32_t d4_transpose(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float d4_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
// a 16-byte load that stays where it is written
__device__ __forceinline__ uint4 ld_now(const uint4 *ptr)
{
    uint4 v;
    asm volatile("ld.global.nc.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(ptr));
    return v;
}
// order-preserving map between floats and signed integers (its own inverse)
__device__ __forceinline__ int d4_ordered_int(float x)
{
    const int i = __float_as_int(x);
    return i ^ ((i >> 31) & 0x7FFFFFFF);
}
__device__ __forceinline__ float d4_ordered_float(int i) { return __int_as_float(i ^ ((i >> 31) & 0x7FFFFFFF)); }
__device__ __forceinline__ float d4_max_rows(float v)   // over the lanes that hold other rows of the same columns
{
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float d4_sum_rows(float v)
{
#pragma unroll
    for (int o = 4; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// floor(n i / of) without leaving 32 bits (i <= of, of below 2^15): where part i of n things begins.
__device__ __forceinline__ int d4_cut(int n, int i, int of)
{
    const int q = n / of, r = n - q * of;
    return q * i + r * i / of;
}
// The block whose part of U units holds unit x: a first guess from the average part (off by few, in floating point), then steps.
__device__ __forceinline__ int d4_holder(int x, int U, int blocks)
{
    int i = min(blocks - 1, (int)((float)x * ((float)blocks / (float)U)));
    while (i > 0 && d4_cut(U, i, blocks) > x) --i;
    while (i + 1 < blocks && d4_cut(U, i + 1, blocks) <= x) ++i;
    return i;
}

__device__ __forceinline__ int d4_len(const Decode4Params &p, int b) { return min(max(__ldg(p.kv_len + b), 0), p.cap_tokens); }

// Where unit x of all units lies: the units in the order (sequence, kv head, unit); sequences without tokens have none.
struct D4Walk {
    int b, head, unit, units, len;
    __device__ __forceinline__ void next(const Decode4Params &p)
    {
        if (++unit < units) return;
        unit = 0;
        if (++head < p.Hkv) return;
        head = 0;
        units = 0;
        while (units == 0 && ++b < p.B) {
            len = d4_len(p, b);
            units = (len + kD4Unit - 1) / kD4Unit;
        }
    }
};

// All units, and where unit x lies.  Executed by a whole warp; first: the length of sequence `lane`, which both look at.
__device__ __forceinline__ int d4_units(int len) { return (len + kD4Unit - 1) / kD4Unit; }
__device__ __forceinline__ int d4_total(const Decode4Params &p, int lane, int first)
{
    int sum = __reduce_add_sync(0xffffffffu, d4_units(first));   // (the host has checked that all units fit 31 bits)
    for (int base = 32; base < p.B; base += 32) sum += __reduce_add_sync(0xffffffffu, (base + lane < p.B) ? d4_units(d4_len(p, base + lane)) : 0);
    return sum * p.Hkv;
}
__device__ __forceinline__ D4Walk d4_find(const Decode4Params &p, int lane, int first, int x)
{
    D4Walk w{0, 0, 0, 1, 0};
    int before = 0;
    for (int base = 0; base < p.B; base += 32) {
        const int len = (base == 0) ? first : ((base + lane < p.B) ? d4_len(p, base + lane) : 0);
        const int n = d4_units(len);
        int upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, (before + upto) * p.Hkv > x);
        if (hit != 0u) {
            const int at = __ffs(hit) - 1;
            const int n_at = __shfl_sync(0xffffffffu, n, at);
            const int r = x - (before + __shfl_sync(0xffffffffu, upto, at) - n_at) * p.Hkv;   // < Hkv * n_at
            w.b = base + at;
            w.head = r / n_at;
            w.unit = r - w.head * n_at;
            w.units = n_at;
            w.len = __shfl_sync(0xffffffffu, len, at);
            return w;
        }
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    return w;
}

// The new token's row in registers: lanes 0-15 hold K, 16-31 V; lane i of a half the dims 4 i .. and 64 + 4 i ...
__device__ __forceinline__ void d4_quantise(const __nv_bfloat16 *row, int i, uint32_t &codes, uint32_t &pair)
{
    const uint2 a = __ldg(reinterpret_cast<const uint2 *>(row) + i), c = __ldg(reinterpret_cast<const uint2 *>(row) + 16 + i);
    uint32_t lo2 = q4_min_bf16x2(q4_min_bf16x2(a.x, a.y), q4_min_bf16x2(c.x, c.y));
    uint32_t hi2 = q4_max_bf16x2(q4_max_bf16x2(a.x, a.y), q4_max_bf16x2(c.x, c.y));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
        lo2 = q4_min_bf16x2(lo2, __shfl_xor_sync(0xffffffffu, lo2, o));
        hi2 = q4_max_bf16x2(hi2, __shfl_xor_sync(0xffffffffu, hi2, o));
    }
    pair = q4_pair(q4_min_of(lo2), q4_max_of(hi2));
    const Q4Row q(pair);
    const uint32_t lo[2] = {a.x, a.y}, hi[2] = {c.x, c.y};
    uint32_t w[1];
    q.words<1>(lo, hi, w);
    codes = w[0];
}

__device__ __forceinline__ void d4_store(__nv_bfloat16 *dst, float4 o)
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(o.x, o.y), b = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// Log-sum-exp merge by one warp of head h of the records that its lanes name (rec: a lane's record, null: none), in lane
// order.  A lane owns four dims.  kGlobal: records of other blocks, read past the L1; at(x): record x's address (x a lane that
// names one).  kBatch outputs are requested together, the first ones before the maxima are known (inside the decode kernel
// four: with eight, the longer run through cold instructions cost the 64 / 8-head workload 0.7 us).
struct D4Merged {
    float m, l;
    float4 o;
};
__device__ __forceinline__ D4Merged d4_none() { return {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)}; }
template <bool kGlobal, int kBatch, class At>
__device__ __forceinline__ void d4_merge(D4Merged &r, const float *rec, int G, int h, int lane, At at)
{
    unsigned todo = __ballot_sync(0xffffffffu, rec != nullptr);
    if (todo == 0u) return;
    float m = -INFINITY, l = 0.f;
    if (rec != nullptr) {
        const float *ml = rec + G * kHeadDim + h;
        m = kGlobal ? __ldcg(ml) : ml[0], l = kGlobal ? __ldcg(ml + G) : ml[G];
    }
    float4 v[kBatch];
    int who[kBatch];
    auto load = [&]() {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            who[u] = (todo != 0u) ? __ffs(todo) - 1 : -1;
            v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (todo != 0u) {
                const float4 *src = reinterpret_cast<const float4 *>(at(who[u]) + h * kHeadDim) + lane;
                v[u] = kGlobal ? __ldcg(src) : *src;
            }
            todo &= todo - 1;
        }
    };
    load();
    const float top = fmaxf(r.m, d4_ordered_float(__reduce_max_sync(0xffffffffu, d4_ordered_int(m))));
    const float w = (m == -INFINITY) ? 0.f : d4_exp2(m - top), f = (r.m == -INFINITY) ? 0.f : d4_exp2(r.m - top);
    r.m = top;
    r.l = r.l * f + warp_sum(l * w);
    r.o = make_float4(r.o.x * f, r.o.y * f, r.o.z * f, r.o.w * f);
    for (;;) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const float wu = (who[u] >= 0) ? __shfl_sync(0xffffffffu, w, max(who[u], 0)) : 0.f;
            r.o.x = fmaf(v[u].x, wu, r.o.x);
            r.o.y = fmaf(v[u].y, wu, r.o.y);
            r.o.z = fmaf(v[u].z, wu, r.o.z);
            r.o.w = fmaf(v[u].w, wu, r.o.w);
        }
        if (todo == 0u) return;
        load();
    }
}
// Which of the blocks' records (two each) is a pair's record x; the pair's first unit lies in block `block`, whose record
// slot0 it is.  With fewer units than blocks every unit has a block of its own.
__device__ __forceinline__ int d4_part(int first, int block, int slot0, int x, int U, int n_blocks)
{
    if (U < n_blocks) return 2 * d4_holder(first + x, U, n_blocks);
    return 2 * (block + x) + (x == 0 ? slot0 : 0);
}
// Where a merge goes: a row of the result, or another record.
__device__ __forceinline__ void d4_put(const D4Merged &r, int G, int h, int lane, __nv_bfloat16 *out, float *part)
{
    if (out != nullptr) {
        const float inv = (r.l > 0.f) ? 1.f / r.l : 0.f;
        d4_store(out + h * kHeadDim + 4 * lane, make_float4(r.o.x * inv, r.o.y * inv, r.o.z * inv, r.o.w * inv));
    } else {
        __stcg(reinterpret_cast<float4 *>(part + h * kHeadDim) + lane, r.o);
        if (lane == 0) {
            __stcg(part + G * kHeadDim + h, r.m);
            __stcg(part + G * (kHeadDim + 1) + h, r.l);
        }
    }
}

template <int kHeads, bool kStep>
__global__ void __launch_bounds__(D4<kHeads>::kWarps * 32, 1)
slim4_decode_kernel(const __grid_constant__ CUtensorMap map_codes, const __grid_constant__ CUtensorMap map_pairs, const __grid_constant__ Decode4Params p)
{
    using L = D4<kHeads>;
    constexpr int NT = L::NT, NW = L::kWarps, S = L::S;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t sbase = smem_u32(smem);
    D4Span *spans = reinterpret_cast<D4Span *>(smem + L::kSpans);
    int *left_of = reinterpret_cast<int *>(smem + L::kLeft);
    volatile int *flags = reinterpret_cast<volatile int *>(smem + L::kFlags);   // [0]: a wait ran out; [1], [2]: what this block, arrived last, has to merge of its first, last pair
    const uint32_t ring = warp * L::kWarpCodes, pair_ring = L::kPairs + warp * 2 * kD4PairBytes;
    auto bar = [&](int s) { return sbase + L::kBars + 8u * (uint32_t)(warp * S + s); };

    pdl_launch_dependents();
    if (lane == 0) {
        if (warp == 0) tc::prefetch_tensormap(&map_codes), tc::prefetch_tensormap(&map_pairs);
        for (int s = 0; s < S; ++s) tc::mbar_init(bar(s), 1);
        tc::mbar_init_fence();
        left_of[2 * warp] = left_of[2 * warp + 1] = -1;
        if (warp == 0) {
            flags[0] = flags[1] = flags[2] = 0;
        }
    }
    __syncthreads();
    pdl_wait();   // from here on what earlier kernels of the stream wrote is read

    // ---- this warp's range of units
    const int len_first = (lane < p.B) ? d4_len(p, lane) : 0;
    const int U = d4_total(p, lane, len_first);
    const int n_blocks = (int)gridDim.x, block = (int)blockIdx.x;
    const int u0 = d4_cut(U, block * NW + warp, n_blocks * NW), cnt = d4_cut(U, block * NW + warp + 1, n_blocks * NW) - u0;
    const int G = p.G, rec_floats = d4_rec_floats(G);
    const uint64_t policy = tc::policy_evict_first();   // cache rows are read once per launch
    bool ok = true;
    const int block0 = d4_cut(U, block, n_blocks), block1 = d4_cut(U, block + 1, n_blocks);
    const bool sparse = U < n_blocks;   // (every unit has a block of its own)
    // ---- the pairs at the block's start and end, if they go on in other blocks (found here, where there is time: the first
    //      copies will be on their way)
    auto find_spans = [&]() {
        if (warp < NW - 2) return;
        const int which = warp - (NW - 2);
        D4Span span;
        span.pair = -1;
        if (block1 > block0) {
            const D4Walk x = d4_find(p, lane, len_first, which ? block1 - 1 : block0);
            span.first = (which ? block1 - 1 : block0) - x.unit;
            span.units = x.units;
            if ((which == 0 || span.first > block0) && (span.first < block0 || span.first + span.units > block1)) {
                span.pair = x.b * p.Hkv + x.head;
                span.block = d4_holder(span.first, U, n_blocks);
                span.parts = sparse ? span.units : d4_holder(span.first + span.units - 1, U, n_blocks) - span.block + 1;
                span.slot0 = (span.first <= d4_cut(U, span.block, n_blocks)) ? 0 : 1;
            }
        }
        if (lane == 0) spans[which] = span;
    };
    // ---- sequences without tokens: zeros
    for (int b = block; b < p.B; b += n_blocks) {
        if (d4_len(p, b) != 0) continue;
        uint4 *dst = reinterpret_cast<uint4 *>(p.out + (size_t)b * p.Hq * kHeadDim);
        for (int i = tid; i < p.Hq * (kHeadDim / 8); i += NW * 32) dst[i] = make_uint4(0, 0, 0, 0);
    }
    if (cnt == 0) find_spans();
    if (cnt > 0) {
        // ---- units n, n + 1 and n + 2 of the range; their page ids are asked for as far ahead
        auto page_of = [&](const D4Walk &x) { return __ldg(p.block_table + (size_t)x.b * p.max_pages_per_seq + (x.unit >> 1)); };
        D4Walk w = d4_find(p, lane, len_first, u0), w1 = w, w2;
        int page0 = page_of(w), page1 = 0, page2 = 0;
        if (cnt > 1) {
            w1.next(p);
            page1 = page_of(w1);
        }
        w2 = w1;
        if (cnt > 2) {
            w2.next(p);
            page2 = page_of(w2);
        }
        // ---- asks for the codes of a K or V half (whole units whatever the length: the page's other slots exist, and what they
        //      hold is masked), with K's for the words of both
        constexpr bool kWhole = S == 4;   // K and V by one copy, one wait
        int ask_slot = 0, blk = 0, row0 = 0;
        auto step_slot = [](int &slot) {
            slot += kWhole ? 2 : 1;
            if (slot == S) slot = 0;
        };
        auto ask_k = [&](const D4Walk &x, int page, int n) {
            page = (page >= 0 && page < p.num_pages) ? page : 0;
            blk = (page * p.Hkv + x.head) * 2, row0 = (x.unit & 1) * kD4Unit;
            if (lane == 0) {
                tc::mbar_arrive_expect_tx(bar(ask_slot), (kWhole ? 2 : 1) * kD4CodeBytes + kD4PairBytes);
                tc::tma_load_3d_hint(sbase + ring + ask_slot * kD4CodeBytes, &map_codes, 0, row0 / 16, blk, bar(ask_slot), policy);
                tc::tma_load_2d_hint(sbase + pair_ring + (n & 1) * kD4PairBytes, &map_pairs, row0, blk, bar(ask_slot), policy);
            }
            step_slot(ask_slot);
        };
        auto ask_v = [&]() {   // (of the unit whose K was asked for last)
            if (kWhole) return;
            if (lane == 0) {
                tc::mbar_arrive_expect_tx(bar(ask_slot), kD4CodeBytes);
                tc::tma_load_3d_hint(sbase + ring + ask_slot * kD4CodeBytes, &map_codes, 0, row0 / 16, blk + 1, bar(ask_slot), policy);
            }
            step_slot(ask_slot);
        };
        int take_slot = 0;
        uint32_t parity = 0;
        auto landed = [&]() {   // waits for the next half
            // (by vote: `ok` decides which way the whole warp goes, also where a wait runs out for some of its lanes only)
            if (!__all_sync(0xffffffffu, tc::mbar_try(bar(take_slot), parity)) &&
                !__all_sync(0xffffffffu, d4_wait(bar(take_slot), parity, flags))) {
                ok = false;
                flags[0] = 1;
            }
            __syncwarp();
            step_slot(take_slot);
            if (take_slot == 0) parity ^= 1u;
        };
        // the query rows of the pair that starts with the next unit, as they are.  They are requested before the copies that
        // fill the ring: a load behind those would wait until memory has delivered them
        uint4 qraw[NT][4];
        auto load_q = [&](int b, int head) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int h = nt * 8 + g;
#pragma unroll
                for (int i = 0; i < 4; ++i) qraw[nt][i] = make_uint4(0, 0, 0, 0);
                if (h < p.G) {
                    const uint4 *src = reinterpret_cast<const uint4 *>(p.q + ((size_t)b * p.Hq + (size_t)head * p.G + h) * kHeadDim);
                    qraw[nt][0] = ld_now(src + 2 * t), qraw[nt][1] = ld_now(src + 2 * t + 1);
                    qraw[nt][2] = ld_now(src + 8 + 2 * t), qraw[nt][3] = ld_now(src + 9 + 2 * t);
                }
            }
        };
        load_q(w.b, w.head);
        ask_k(w, page0, 0);

        uint32_t qf[NT][8][2];                  // Q^T operands: dims 16 t + 4 j .. (even steps), 64 further (odd steps)
        float rs[NT][2], qz[NT][2];             // of the columns 2 t, 2 t + 1: what a product and a row's offset count for
        float o[NT][8][4];                      // O^T: dim 8 g + i (first two) and that plus 16 times dim 64 + 8 g + i, of the columns 2 t, 2 t + 1
        float m[NT][2], l[NT][2], z[NT][2];     // running maximum; this lane's share of sum p and sum p z
        float r_cur = 0.f;                      // what the scales are multiplied with in P^T (0: nothing of the pair seen yet)
        bool fresh = true;
        int run_index = 0, run_unit0 = w.unit;
        const int row = g ^ ((g >> 1) & 1);     // token of this lane's row: neighbouring rows lie in opposite halves of the banks
        const int k_off = row * kRow4Bytes + t * 16;
        const int v_off0 = (2 * t ^ (t & 1)) * kRow4Bytes + 8 * g, v_off1 = ((2 * t + 1) ^ (t & 1)) * kRow4Bytes + 8 * g;

        for (int n = 0; n < cnt; ++n) {
            if (fresh) {
                fresh = false;
                if (NT > 1 && n > 0) load_q(w.b, w.head);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const uint4 (&v)[4] = qraw[nt];
                    float am = 0.f, sum = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float a = bf16_bits_to_float(x[k] & 0xFFFFu), b = __uint_as_float(x[k] & 0xFFFF0000u);
                            am = fmaxf(am, fmaxf(fabsf(a), fabsf(b)));
                            sum += a + b;
                        }
                    }
#pragma unroll
                    for (int x = 1; x <= 2; x <<= 1) {
                        am = fmaxf(am, __shfl_xor_sync(0xffffffffu, am, x));
                        sum += __shfl_xor_sync(0xffffffffu, sum, x);
                    }
                    const float p2 = pow2_floor(am), inv = pow2_recip(p2) * 16384.f;   // |q inv| < 2^15
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t x[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
                        const float f = (i < 2) ? inv : inv * 0.0625f;      // the high halves' codes count 2^4 more
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int step = 2 * (2 * (i & 1) + k) + (i >> 1);
                            qf[nt][step][0] = pack_half2(bf16_bits_to_float(x[2 * k] & 0xFFFFu) * f, bf16_bits_to_float(x[2 * k + 1] & 0xFFFFu) * f);
                            qf[nt][step][1] = pack_half2(__uint_as_float(x[2 * k] & 0xFFFF0000u) * f, __uint_as_float(x[2 * k + 1] & 0xFFFF0000u) * f);
                        }
                    }
                    const float mine = p2 * 1024.f * p.scale_log2e, sz = sum * p.scale_log2e;   // 2^24 / 2^14
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        rs[nt][k] = __shfl_sync(0xffffffffu, mine, 8 * t + 4 * k);
                        qz[nt][k] = __shfl_sync(0xffffffffu, sz, 8 * t + 4 * k);
                        m[nt][k] = l[nt][k] = z[nt][k] = 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
                }
                r_cur = 0.f;
                if (n == 0) {
                    find_spans();   // (the rest of the ring is filled once the query rows are there: they do not queue behind it)
                    ask_v();
                    if (cnt > 1) ask_k(w1, page1, 1);
                }
            }
            const int n_tok = min(kD4Unit, w.len - w.unit * kD4Unit);
            const bool ends = w.unit == w.units - 1;                            // the pair's last unit
            const bool complete = ends && run_unit0 == 0;
            const bool leaves = (ends && !complete) || (n == cnt - 1 && !ends); // a record is left behind this unit
            if (NT == 1 && ends && n + 1 < cnt) {   // the next pair's query rows, a unit ahead (with NT = 2 their 32 registers cost more)
                load_q(w1.b, w1.head);
            }
            unsigned char *kst = smem + ring + take_slot * kD4CodeBytes;
            landed();
            unsigned char *vst = kWhole ? kst + kD4CodeBytes : smem + ring + take_slot * kD4CodeBytes;
            uint32_t *kp = reinterpret_cast<uint32_t *>(smem + pair_ring + (n & 1) * kD4PairBytes), *vp = kp + kD4Unit;
            const bool appends = kStep && ends && ok && __ldg(p.kv_len + w.b) == w.len;
            uint32_t new_codes = 0;
            if (kStep && appends) {
                // ---- the new token: quantised here, stored in the cache and in the unit's copy of it
                const int kv = lane >> 4, i = lane & 15, at = n_tok - 1, pos = w.len - 1;
                uint32_t pair;
                d4_quantise((kv ? p.v_new : p.k_new) + ((size_t)w.b * p.Hkv + w.head) * kHeadDim, i, new_codes, pair);
                if (kv == 0) reinterpret_cast<uint32_t *>(kst + at * kRow4Bytes)[i] = new_codes;
                if (i == 0) kp[kv * kD4Unit + at] = pair;
                const int page = __ldg(p.block_table + (size_t)w.b * p.max_pages_per_seq + (pos >> 7));
                if (page >= 0 && page < p.num_pages) {
                    const int in_page = pos & (kPageTokens - 1);
                    uint8_t *dst = p.codes + code4_block_offset(page, w.head, kv, p.Hkv) + (size_t)in_page * kRow4Bytes;
                    reinterpret_cast<uint32_t *>(dst)[i] = new_codes;
                    if (i == 0) p.pairs[scale_block_offset(page, w.head, kv, p.Hkv) + in_page] = pair;
                }
                tc::fence_proxy_async();   // (the slot is filled by the copy engine again)
                __syncwarp();
            }
            if (n_tok < kD4Unit) {   // what lies behind the last token may be anything: words of zero
                if (lane + 32 >= n_tok) kp[lane + 32] = vp[lane + 32] = 0u;
                if (lane >= n_tok) kp[lane] = vp[lane] = 0u;
                tc::fence_proxy_async();
                __syncwarp();
            }

            // ---- S^T = K Q^T: rows g and g + 8 of every 16 tokens; then the scores less the running maximum
            //      (a tile's eight products form a chain: the four tiles' chains are issued in turn)
            float c[4][NT][4];
            uint32_t ka[4][4], kb[4][4];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                const uint4 a4 = *reinterpret_cast<const uint4 *>(kst + k_off + mt * 16 * kRow4Bytes);
                const uint4 b4 = *reinterpret_cast<const uint4 *>(kst + k_off + (mt * 16 + 8) * kRow4Bytes);
                ka[mt][0] = a4.x, ka[mt][1] = a4.y, ka[mt][2] = a4.z, ka[mt][3] = a4.w;
                kb[mt][0] = b4.x, kb[mt][1] = b4.y, kb[mt][2] = b4.z, kb[mt][3] = b4.w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
                    const uint32_t a = ka[mt][j], b = kb[mt][j], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if (j == 0) d4_mma0(c[mt][nt], a & 0x000F000Fu, b & 0x000F000Fu, a8 & 0x000F000Fu, b8 & 0x000F000Fu, qf[nt][2 * j][0], qf[nt][2 * j][1]);
                        else d4_mma(c[mt][nt], a & 0x000F000Fu, b & 0x000F000Fu, a8 & 0x000F000Fu, b8 & 0x000F000Fu, qf[nt][2 * j][0], qf[nt][2 * j][1]);
                    }
                }
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
                    const uint32_t a = ka[mt][j], b = kb[mt][j], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
                        d4_mma(c[mt][nt], a & 0x00F000F0u, b & 0x00F000F0u, a8 & 0x00F000F0u, b8 & 0x00F000F0u, qf[nt][2 * j + 1][0], qf[nt][2 * j + 1][1]);
                }
            }
            float top[NT][2];
            {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY;
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const uint32_t k2 = kp[mt * 16 + hf * 8 + row];
                        const float sk = pair_scale(k2), zk = pair_offset(k2);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                            for (int k = 0; k < 2; ++k) c[mt][nt][2 * hf + k] = fmaf(c[mt][nt][2 * hf + k], sk * rs[nt][k], fmaf(zk, qz[nt][k], -m[nt][k]));
                        }
                    }
                }
                if (n_tok < kD4Unit) {
#pragma unroll
                    for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                        for (int hf = 0; hf < 2; ++hf) {
                            if (mt * 16 + hf * 8 + row < n_tok) continue;
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) c[mt][nt][2 * hf] = c[mt][nt][2 * hf + 1] = -INFINITY;
                        }
                    }
                }
#pragma unroll
                for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) top[nt][k] = fmaxf(top[nt][k], fmaxf(c[mt][nt][k], c[mt][nt][2 + k]));
                    }
                }
            }
            if (!kWhole) {
                __syncwarp();          // every lane has read the K half
                if (n + 1 < cnt) ask_v();
                landed();
            }
            if (kStep && appends) {
                if (lane >= 16) reinterpret_cast<uint32_t *>(vst + (n_tok - 1) * kRow4Bytes)[lane & 15] = new_codes;
                tc::fence_proxy_async();
                __syncwarp();
            }
            // ---- a larger maximum, a much larger V scale (rarely, but for the pair's first unit)
            bool grow = r_cur == 0.f;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) grow |= fmaxf(top[nt][0], top[nt][1]) > kD4Grow;
            const uint2 v2 = *reinterpret_cast<const uint2 *>(vp + 2 * lane);
            const float sv_max = fmaxf(pair_scale(v2.x), pair_scale(v2.y));
            grow |= sv_max * r_cur >= 4.f * kD4Top;
            if (__any_sync(0xffffffffu, grow)) {
                const float sv_top = warp_max(sv_max);
                const float r_fit = pow2_recip(pow2_floor(sv_top)) * kD4Top;
                if (r_cur == 0.f) {
                    r_cur = r_fit;   // (nothing summed up yet)
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            m[nt][k] = d4_max_rows(top[nt][k]);
#pragma unroll
                            for (int mt = 0; mt < 4; ++mt) c[mt][nt][k] -= m[nt][k], c[mt][nt][2 + k] -= m[nt][k];
                        }
                    }
                } else {
                    const float r_new = (sv_top * r_cur >= 4.f * kD4Top) ? r_fit : r_cur, fr = r_new / r_cur;
                    r_cur = r_new;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float al[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float up = fmaxf(d4_max_rows(top[nt][k]), 0.f);
                            m[nt][k] += up;
                            al[k] = d4_exp2(-up);
                            l[nt][k] *= al[k];
                            z[nt][k] *= al[k];
                            al[k] *= fr;
#pragma unroll
                            for (int mt = 0; mt < 4; ++mt) c[mt][nt][k] -= up, c[mt][nt][2 + k] -= up;
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            o[nt][i][0] *= al[0];
                            o[nt][i][1] *= al[1];
                            o[nt][i][2] *= al[0];
                            o[nt][i][3] *= al[1];
                        }
                    }
                }
            }
            // ---- P^T of all four tiles, then O^T += V^T P^T
            uint32_t pt[4][NT][2];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const uint32_t pair = vp[mt * 16 + hf * 8 + row];
                    const float sr = pair_scale(pair) * r_cur, zv = pair_offset(pair);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float e[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            e[k] = d4_exp2(c[mt][nt][2 * hf + k]);
                            l[nt][k] += e[k];
                            z[nt][k] = fmaf(e[k], zv, z[nt][k]);
                        }
                        pt[mt][nt][hf] = d4_transpose(pack_half2(e[0] * sr, e[1] * sr));
                    }
                }
            }
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                // token rows 2 t and 2 t + 1 (this lane's column pair of the operand) and the two eight further
                const unsigned char *v0 = vst + v_off0 + mt * 16 * kRow4Bytes, *v1 = vst + v_off1 + mt * 16 * kRow4Bytes;
                const uint2 va = *reinterpret_cast<const uint2 *>(v0), vb = *reinterpret_cast<const uint2 *>(v1);
                const uint2 vc = *reinterpret_cast<const uint2 *>(v0 + 8 * kRow4Bytes), vd = *reinterpret_cast<const uint2 *>(v1 + 8 * kRow4Bytes);
#pragma unroll
                for (int w2 = 0; w2 < 2; ++w2) {
                    const uint32_t wa = w2 ? va.y : va.x, wb = w2 ? vb.y : vb.x, wc = w2 ? vc.y : vc.x, wd = w2 ? vd.y : vd.x;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x = __byte_perm(wa, wb, half ? 0x7632 : 0x5410), y = __byte_perm(wc, wd, half ? 0x7632 : 0x5410);
                        const uint32_t x8 = __byte_perm(x, 0u, 0x4341), y8 = __byte_perm(y, 0u, 0x4341);   // the odd bytes, whole
                        const int i = 4 * w2 + 2 * half;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            d4_mma(o[nt][i], x & 0x000F000Fu, x & 0x00FF00FFu, y & 0x000F000Fu, y & 0x00FF00FFu, pt[mt][nt][0], pt[mt][nt][1]);
                            d4_mma(o[nt][i + 1], x8 & 0x000F000Fu, x8, y8 & 0x000F000Fu, y8, pt[mt][nt][0], pt[mt][nt][1]);
                        }
                    }
                }
            }
            __syncwarp();              // every lane has read the V half
            if (n + 2 < cnt) ask_k(w2, page2, n);

            // ---- the end of the pair, or of the range
            if (complete || leaves) {
                const float f1 = 16777216.f / r_cur, f2 = f1 * 0.0625f;    // the codes counted 2^-24 and 2^-20
                float *rec = reinterpret_cast<float *>(smem + L::record(2 * warp + (run_index == 0 ? 0 : 1)));   // (a last one lies in the ring: nothing is in flight)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const int h = nt * 8 + 2 * t + k;
                        const float ls = d4_sum_rows(l[nt][k]), zs = d4_sum_rows(z[nt][k]);
                        float lo[8], hi[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            lo[i] = fmaf(o[nt][i][k], f1, zs);
                            hi[i] = fmaf(o[nt][i][2 + k] - o[nt][i][k], f2, zs);   // (whole bytes less their low halves)
                        }
                        if (h >= p.G || !ok) continue;
                        if (complete) {
                            const float inv = 1.f / ls;
                            __nv_bfloat16 *dst = p.out + ((size_t)w.b * p.Hq + (size_t)w.head * p.G + h) * kHeadDim + 8 * g;
                            d4_store(dst, make_float4(lo[0] * inv, lo[1] * inv, lo[2] * inv, lo[3] * inv));
                            d4_store(dst + 4, make_float4(lo[4] * inv, lo[5] * inv, lo[6] * inv, lo[7] * inv));
                            d4_store(dst + 64, make_float4(hi[0] * inv, hi[1] * inv, hi[2] * inv, hi[3] * inv));
                            d4_store(dst + 68, make_float4(hi[4] * inv, hi[5] * inv, hi[6] * inv, hi[7] * inv));
                        } else {
                            float4 *dst = reinterpret_cast<float4 *>(rec + h * kHeadDim + 8 * g);
                            dst[0] = make_float4(lo[0], lo[1], lo[2], lo[3]);
                            dst[1] = make_float4(lo[4], lo[5], lo[6], lo[7]);
                            dst[16] = make_float4(hi[0], hi[1], hi[2], hi[3]);
                            dst[17] = make_float4(hi[4], hi[5], hi[6], hi[7]);
                            if (g == 0) {
                                rec[G * kHeadDim + h] = m[nt][k];
                                rec[G * (kHeadDim + 1) + h] = ls;
                            }
                        }
                    }
                }
                if (leaves && lane == 0 && ok) {
                    left_of[2 * warp + (run_index == 0 ? 0 : 1)] = w.b * p.Hkv + w.head;
                }
                ++run_index;
                run_unit0 = 0;
                fresh = true;
            }
            w = w1;
            w1 = w2;
            if (n + 3 < cnt) {
                w2.next(p);
                page2 = page_of(w2);
            }
        }
        if (!ok) {   // copies still in flight get a bounded chance to land
            for (int s = 0; s < S; ++s) {
                tc::mbar_wait(bar(s), 0, 1u << 14);
                tc::mbar_wait(bar(s), 1, 1u << 14);
            }
        }
    }
    __syncthreads();
    if (flags[0] != 0) {
        if (tid == 0) atomicExch(p.status, SLIM_ERR_TIMEOUT);
        return;
    }

    // ---- records of the block's warps, in the order of the units: those of one pair are merged
    auto out_rows = [&](int pair) { return p.out + (size_t)pair * G * kHeadDim; };
    auto part = [&](int i) { return p.parts + (size_t)i * rec_floats; };
    {
        // lane e looks at record e; the first one of every pair stands for the pair
        const int pair = (lane < 2 * NW) ? left_of[lane] : -1;
        const unsigned valid = __ballot_sync(0xffffffffu, pair >= 0), below = valid & ((1u << lane) - 1u);
        const int before = __shfl_sync(0xffffffffu, pair, below != 0u ? 31 - __clz(below) : 0);
        unsigned firsts = __ballot_sync(0xffffffffu, pair >= 0 && (below == 0u || before != pair));
        auto at = [&](int e) { return reinterpret_cast<const float *>(smem + L::record(e)); };
        const int span0 = spans[0].pair, span1 = spans[1].pair;
        int h = warp;   // tasks (pair, head) are dealt to the warps in turn
        while (firsts != 0u) {
            const int of = __shfl_sync(0xffffffffu, pair, __ffs(firsts) - 1);
            firsts &= firsts - 1;
            for (; h < G; h += NW) {
                D4Merged r = d4_none();
                d4_merge<false, 4>(r, pair == of ? at(lane) : nullptr, G, h, lane, at);
                d4_put(r, G, h, lane, (of != span0 && of != span1) ? out_rows(of) : nullptr, part(2 * block + (of == span0 ? 0 : 1)));
            }
            h -= G;
        }
    }
    if (p.counters == nullptr) return;   // (the second kernel merges what blocks share)
    __syncthreads();
    // ---- pairs that span blocks: the block that arrives last merges their records
    if (warp < 2 && lane == 0 && spans[warp].pair >= 0) {
        const D4Span &span = spans[warp];
        int *counter = p.counters + span.block, before;
        // (releases the block's records, which were written before the barrier, and acquires those of the others)
        asm volatile("atom.acq_rel.gpu.global.add.s32 %0, [%1], 1;\n" : "=r"(before) : "l"(counter) : "memory");
        const bool last = before + 1 == span.parts;
        if (last) *counter = 0;   // ready for the next launch
        flags[1 + warp] = last ? 1 : 0;
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (flags[1 + which] == 0) continue;
        const D4Span span = spans[which];
        for (int h = (warp + NW - which * NW / 2) % NW; h < G; h += NW) {
            D4Merged r = d4_none();
            for (int x0 = 0; x0 < span.parts; x0 += 32) {
                const int x = x0 + lane;
                const int index = (x < span.parts) ? d4_part(span.first, span.block, span.slot0, x, U, n_blocks) : -1;
                d4_merge<true, 4>(r, (index >= 0) ? part(index) : nullptr, G, h, lane, [&](int e) { return part(__shfl_sync(0xffffffffu, index, e)); });
            }
            d4_put(r, G, h, lane, out_rows(span.pair), nullptr);
        }
    }
}

// The pairs that span blocks, where few pairs span many: a block per query row, four warps taking every fourth record.
constexpr int kD4MergeWarps = 4;
__global__ void __launch_bounds__(kD4MergeWarps * 32)
slim4_decode_merge_kernel(const __grid_constant__ Decode4Params p, const int n_blocks)
{
    __shared__ float4 o_s[kD4MergeWarps][32];
    __shared__ float m_s[kD4MergeWarps], l_s[kD4MergeWarps];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x, b = row / p.Hq, h = row % p.Hq % p.G, head = row % p.Hq / p.G;
    pdl_wait();
    int U = 0, before = 0;
    for (int base = 0; base < p.B; base += 32) {
        const int n = (base + lane < p.B) ? d4_units(d4_len(p, base + lane)) : 0;
        U += __reduce_add_sync(0xffffffffu, n);
        before += __reduce_add_sync(0xffffffffu, base + lane < b ? n : 0);
    }
    const int units = d4_units(d4_len(p, b)), first = before * p.Hkv + head * units;
    U *= p.Hkv;
    if (units == 0) return;
    const int block = d4_holder(first, U, n_blocks), last = d4_holder(first + units - 1, U, n_blocks);
    if (block == last) return;   // (the one block has written the result)
    const int parts = (U < n_blocks) ? units : last - block + 1, slot0 = (first <= d4_cut(U, block, n_blocks)) ? 0 : 1;
    const int rec_floats = d4_rec_floats(p.G);
    D4Merged r = d4_none();
    for (int x0 = 0; x0 < parts; x0 += 32 * kD4MergeWarps) {
        const int x = x0 + lane * kD4MergeWarps + warp;
        const int index = (x < parts) ? d4_part(first, block, slot0, x, U, n_blocks) : -1;
        d4_merge<true, 8>(r, (index >= 0) ? p.parts + (size_t)index * rec_floats : nullptr, p.G, h, lane,
                       [&](int e) { return p.parts + (size_t)__shfl_sync(0xffffffffu, index, e) * rec_floats; });
    }
    if (lane == 0) m_s[warp] = r.m, l_s[warp] = r.l;
    o_s[warp][lane] = r.o;
    __syncthreads();
    if (warp != 0) return;
    r = d4_none();
#pragma unroll
    for (int i = 0; i < kD4MergeWarps; ++i) r.m = fmaxf(r.m, m_s[i]);
#pragma unroll
    for (int i = 0; i < kD4MergeWarps; ++i) {
        const float w = (m_s[i] == -INFINITY) ? 0.f : d4_exp2(m_s[i] - r.m);
        const float4 v = o_s[i][lane];
        r.l = fmaf(l_s[i], w, r.l);
        r.o = make_float4(fmaf(v.x, w, r.o.x), fmaf(v.y, w, r.o.y), fmaf(v.z, w, r.o.z), fmaf(v.w, w, r.o.w));
    }
    d4_put(r, p.G, h, lane, p.out + ((size_t)b * p.Hq + (size_t)head * p.G) * kHeadDim, nullptr);
}

size_t decode4_workspace_bytes(int G)
{
    return kDecodeHeaderBytes + (size_t)kD4MaxBlocks * 2 * d4_rec_floats(G) * sizeof(float);
}

template <int kHeads, bool kStep>
static int launch_d4(const slim_cache4_t *c, const Decode4Params &p, int max_kv, cudaStream_t stream)
{
    int sms = 0;
    int rc = sm_count(&sms);
    if (rc != SLIM_OK) return rc;
    if (sms > kD4MaxBlocks) sms = kD4MaxBlocks;
    const long long pairs = (long long)p.B * p.Hkv, per_pair = (max_kv + kD4Unit - 1) / kD4Unit, units = pairs * per_pair;
    if (units > 0x7FFFFFFFLL) return SLIM_ERR_UNSUPPORTED;   // (units are counted in 32 bits)
    // One block per SM; where a pair is at most a unit for every warp and there is an SM for every pair, one block per pair:
    // nothing is merged between blocks then (one sequence, 32 / 32 heads, 272 tokens: 6.7 us, spread over all SMs 9.1; 32 / 8
    // heads, 768 tokens: 7.8 and 9.6; 32 / 2 heads, 512 tokens: 9.2 and 12.2)
    long long blocks = units < sms ? units : sms;
    if (per_pair <= D4<kHeads>::kWarps && pairs < blocks) blocks = pairs;
    if (blocks < 1) blocks = 1;
    CUtensorMap codes, scales;
    rc = unit4_tensor_maps(c, D4<kHeads>::S == 4 ? 2 : 1, &codes, &scales);
    if (rc != SLIM_OK) return rc;
    rc = allow_dynamic_smem(reinterpret_cast<const void *>(slim4_decode_kernel<kHeads, kStep>), (int)D4<kHeads>::kBytes);
    if (rc != SLIM_OK) return rc;
    // Few pairs on many blocks: a second kernel merges them.  In us, the last block merging / the second kernel, with one, eight
    // and sixteen query heads per kv head, one sequence of 32768 tokens: 74 blocks per pair 20.8 / 13.0, 23.4 / 15.6, 37.2 / 17.6;
    // 18.5 blocks 17.9 / 18.0, 20.2 / 18.1, 27.1 / 21.9; 9.2 blocks 22.2 / 23.4, 25.3 / 24.0, 35.7 / 29.9; 4.6 blocks 33.2 / 35.0 and
    // 36.4 / 36.5 (four sequences of 8192: 19.0 / 18.7).  With more pairs its launch costs more than it saves (32 ragged
    // sequences, 64 / 8 heads, 0.6 blocks: 28.3 / 32.5).
    const bool defer = blocks > kD4Few * pairs;
    Decode4Params q = p;
    if (defer) q.counters = nullptr;
    SLIM_CUDA_TRY(launch_pdl(slim4_decode_kernel<kHeads, kStep>, dim3((unsigned)blocks), dim3(D4<kHeads>::kWarps * 32), D4<kHeads>::kBytes, stream, codes, scales, q));
    if (defer) SLIM_CUDA_TRY(launch_pdl(slim4_decode_merge_kernel, dim3((unsigned)(p.B * p.Hq)), dim3(kD4MergeWarps * 32), 0, stream, q, (int)blocks));
    return SLIM_OK;
}

int launch_decode4(const slim_cache4_t *c, const void *q, const void *k_new, const void *v_new, void *out, const int32_t *kv_len, int B,
                   int max_kv, int Hq, float sm_scale, void *workspace, cudaStream_t stream)
{
    Decode4Params p;
    p.codes = c->codes;
    p.pairs = reinterpret_cast<uint32_t *>(c->scales);
    p.block_table = c->block_table;
    p.kv_len = kv_len;
    p.q = static_cast<const __nv_bfloat16 *>(q);
    p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = static_cast<const __nv_bfloat16 *>(v_new);
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.status = static_cast<int *>(workspace);
    p.counters = reinterpret_cast<int *>(static_cast<char *>(workspace) + kDecodeStatusBytes);
    p.parts = reinterpret_cast<float *>(static_cast<char *>(workspace) + kDecodeHeaderBytes);
    p.B = B;
    p.Hq = Hq;
    p.Hkv = c->num_kv_heads;
    p.G = Hq / c->num_kv_heads;
    p.max_pages_per_seq = c->max_pages_per_seq;
    p.num_pages = c->num_pages;
    p.cap_tokens = max_kv;   // (the caller has checked it against the page table)
    p.scale_log2e = sm_scale * kLog2e;
    const bool step = k_new != nullptr;
    if (p.G <= 2) return step ? launch_d4<2, true>(c, p, max_kv, stream) : launch_d4<2, false>(c, p, max_kv, stream);
    if (p.G <= 8) return step ? launch_d4<8, true>(c, p, max_kv, stream) : launch_d4<8, false>(c, p, max_kv, stream);
    return step ? launch_d4<16, true>(c, p, max_kv, stream) : launch_d4<16, false>(c, p, max_kv, stream);
}

}  // namespace slim

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
//  * Warps are independent: each has its own ring of 64-token units (two bulk copies for the codes, two for the scales),
//    its own contiguous range of the units of all pairs, and its own running maximum, sum and O in registers.  A pair that
//    begins and ends inside a warp's range is written as the result at once; the others leave a record, merged by the
//    block, and where a pair spans blocks, by the block that finishes it last.
//
// Query rows are held as fp16 after division by a power of two near the row's largest value: exact down to 2^-24 of it.
// The weights p_j s_j are rounded to fp16 (2^-11 of each), p_j itself, its sum and the offset's sum stay fp32.
// Every wait is bounded; a wait that runs out raises the status word and the warp writes nothing more.
#include "slim4_common.cuh"
#include "slim_decode_params.cuh"
#include "slim_tcgen05.cuh"
#include "slim_tmap.cuh"

namespace slim {

constexpr int kD4Unit = 64;                        // tokens of a ring stage
constexpr int kD4Warps = 8;
constexpr int kD4Stages = 2;
constexpr uint32_t kD4CodeBytes = kD4Unit * kRow4Bytes;
constexpr uint32_t kD4PairBytes = kD4Unit * 4;
constexpr uint32_t kD4StageBytes = 2 * (kD4CodeBytes + kD4PairBytes);
constexpr float kD4Grow = 4.f;                     // the running maximum moves when it is exceeded by 2^4
constexpr float kD4Top = 512.f;                    // p s is scaled so that the largest s counts as 2^9 to 2^10 (with p <= 2^4 far below fp16's 2^16)

struct Decode4Params {
    const uint8_t *codes;
    const uint32_t *pairs;
    const int32_t *block_table;
    const int32_t *kv_len;
    const __nv_bfloat16 *q, *k_new, *v_new;
    __nv_bfloat16 *out;
    int *status;
    int *counters;      // per block: arrivals for the pair that begins in it and ends in a later one
    float *parts;       // two records per block
    int B, Hq, Hkv, G, max_pages_per_seq, num_pages, cap_tokens;
    float scale_log2e;
};

// A pair's records: O [heads][128], then m [heads] and l [heads].
template <int NT>
struct D4 {
    static constexpr int kHeads = 8 * NT;
    static constexpr int kRecFloats = kHeads * (kHeadDim + 2);
    static constexpr uint32_t kRing = 0;
    static constexpr uint32_t kFirst = kD4Warps * kD4Stages * kD4StageBytes;     // a warp's record of its first pair
    static constexpr uint32_t kMeta = kFirst + kD4Warps * kRecFloats * 4;        // D4Run [2 * warps], then the block's [2]
    static constexpr uint32_t kBars = kMeta + (2 * kD4Warps + 2) * 16;
    static constexpr uint32_t kFlags = kBars + kD4Warps * kD4Stages * 8;         // int[4]
    static constexpr uint32_t kBytes = kFlags + 16;
    static_assert(kRecFloats * 4 <= kD4Stages * kD4StageBytes, "a warp's last record goes into its ring");
    static_assert(kBytes <= 232448, "shared memory of one block");
};

// Part of a pair that a warp (or block) has worked on.
struct __align__(16) D4Run {
    int pair, units;    // pair -1: nothing
    long long first;    // the pair's first unit in the order of all units
};

__device__ __forceinline__ void d4_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
__device__ __forceinline__ long long d4_div(long long a, long long b)
{
    if ((((unsigned long long)a | (unsigned long long)b) >> 32) == 0ull) return (long long)((unsigned)a / (unsigned)b);
    return a / b;
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

// All units, and where unit x lies.  Executed by a whole warp.
__device__ __forceinline__ long long d4_total(const Decode4Params &p, int lane)
{
    long long sum = 0;
    for (int base = 0; base < p.B; base += 32) {
        const int n = (base + lane < p.B) ? (d4_len(p, base + lane) + kD4Unit - 1) / kD4Unit : 0;
        sum += __reduce_add_sync(0xffffffffu, n);
    }
    return sum * p.Hkv;
}
__device__ __forceinline__ D4Walk d4_find(const Decode4Params &p, int lane, long long x)
{
    D4Walk w{0, 0, 0, 1, 0};
    long long before = 0;
    for (int base = 0; base < p.B; base += 32) {
        const int len = (base + lane < p.B) ? d4_len(p, base + lane) : 0;
        const int n = (len + kD4Unit - 1) / kD4Unit;
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
            const long long r = x - (before + __shfl_sync(0xffffffffu, upto, at) - n_at) * p.Hkv;   // < Hkv * n_at
            w.b = base + at;
            w.head = (int)d4_div(r, n_at);
            w.unit = (int)(r - (long long)w.head * n_at);
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
    uint32_t hi2 = ap_max_bf16x2(ap_max_bf16x2(a.x, a.y), ap_max_bf16x2(c.x, c.y));
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) {
        lo2 = q4_min_bf16x2(lo2, __shfl_xor_sync(0xffffffffu, lo2, o));
        hi2 = ap_max_bf16x2(hi2, __shfl_xor_sync(0xffffffffu, hi2, o));
    }
    pair = q4_pair(fminf(__uint_as_float(lo2 << 16), __uint_as_float(lo2 & 0xFFFF0000u)),
                   fmaxf(__uint_as_float(hi2 << 16), __uint_as_float(hi2 & 0xFFFF0000u)));
    const Q4Row q(pair);
    codes = q.codes4(a.x, a.y) | (q.codes4(c.x, c.y) << 4);
}

__device__ __forceinline__ void d4_store(__nv_bfloat16 *dst, float4 o)
{
    const __nv_bfloat162 a = __floats2bfloat162_rn(o.x, o.y), b = __floats2bfloat162_rn(o.z, o.w);
    *reinterpret_cast<uint2 *>(dst) = make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// A record's share of a merge: O and l relative to the largest maximum so far (a lane owns four dims of one head).
struct D4Merge {
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float m1, float l1, float4 o1)
    {
        const float M = fmaxf(m, m1);
        const float f = (m == M) ? 1.f : exp2f(m - M), f1 = (m1 == M) ? 1.f : exp2f(m1 - M);
        m = M;
        l = l * f + l1 * f1;
        o.x = o.x * f + o1.x * f1;
        o.y = o.y * f + o1.y * f1;
        o.z = o.z * f + o1.z * f1;
        o.w = o.w * f + o1.w * f1;
    }
    __device__ __forceinline__ void write(__nv_bfloat16 *dst) const
    {
        const float inv = (l > 0.f) ? 1.f / l : 0.f;
        d4_store(dst, make_float4(o.x * inv, o.y * inv, o.z * inv, o.w * inv));
    }
};

template <int NT, bool kStep>
__global__ void __launch_bounds__(kD4Warps * 32, 1)
slim4_decode_kernel(const Decode4Params p)
{
    using L = D4<NT>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
    const uint32_t sbase = smem_u32(smem);
    D4Run *runs = reinterpret_cast<D4Run *>(smem + L::kMeta);
    volatile int *flags = reinterpret_cast<volatile int *>(smem + L::kFlags);   // [0]: a wait ran out; [1], [2]: this block merges its first, last pair
    const uint32_t ring = sbase + L::kRing + warp * (kD4Stages * kD4StageBytes);
    auto bar = [&](int s) { return sbase + L::kBars + 8u * (uint32_t)(warp * kD4Stages + s); };

    pdl_launch_dependents();
    if (lane == 0) {
        for (int s = 0; s < kD4Stages; ++s) tc::mbar_init(bar(s), 1);
        tc::mbar_init_fence();
        runs[2 * warp].pair = runs[2 * warp + 1].pair = -1;
        if (warp == 0) {
            flags[0] = flags[1] = flags[2] = 0;
            runs[2 * kD4Warps].pair = runs[2 * kD4Warps + 1].pair = -1;
        }
    }
    __syncthreads();
    pdl_wait();   // from here on what earlier kernels of the stream wrote is read

    // ---- this warp's range of units
    const long long U = d4_total(p, lane);
    const long long W = (long long)gridDim.x * kD4Warps, gw = (long long)blockIdx.x * kD4Warps + warp;
    const long long u0 = d4_div(U * gw, W), u1 = d4_div(U * (gw + 1), W);
    const int cnt = (int)(u1 - u0);
    bool ok = true;
    int issued = 0;
    if (cnt > 0) {
        D4Walk w = d4_find(p, lane, u0), ahead = w;
        int page_next = __ldg(p.block_table + (size_t)ahead.b * p.max_pages_per_seq + (ahead.unit >> 1));
        // asks for the unit `ahead` stands on and steps ahead (the next page id is on its way while this unit's copies are)
        auto issue = [&]() {
            const int s = issued % kD4Stages;
            const int n_tok = min(kD4Unit, ahead.len - ahead.unit * kD4Unit);
            const int page = (page_next >= 0 && page_next < p.num_pages) ? page_next : 0;
            const int head = ahead.head, slot = (ahead.unit & 1) * kD4Unit;
            ++issued;
            if (issued < cnt) {
                ahead.next(p);
                page_next = __ldg(p.block_table + (size_t)ahead.b * p.max_pages_per_seq + (ahead.unit >> 1));
            }
            if (lane == 0) {
                const uint32_t dst = ring + s * kD4StageBytes;
                const uint32_t code_bytes = (uint32_t)n_tok * kRow4Bytes, pair_bytes = (uint32_t)((n_tok + 3) & ~3) * 4u;
                const uint8_t *c = p.codes + code4_block_offset(page, head, 0, p.Hkv) + (size_t)slot * kRow4Bytes;
                const uint32_t *sc = p.pairs + scale_block_offset(page, head, 0, p.Hkv) + slot;
                tc::mbar_arrive_expect_tx(bar(s), 2 * (code_bytes + pair_bytes));
                tc::bulk_load(dst, c, code_bytes, bar(s));
                tc::bulk_load(dst + 2 * kD4CodeBytes, sc, pair_bytes, bar(s));
                tc::bulk_load(dst + kD4CodeBytes, c + kPageTokens * kRow4Bytes, code_bytes, bar(s));
                tc::bulk_load(dst + 2 * kD4CodeBytes + kD4PairBytes, sc + kPageTokens, pair_bytes, bar(s));
            }
        };
        for (int i = 0; i < min(kD4Stages, cnt); ++i) issue();

        uint32_t qf[NT][8][2];                  // Q^T operands: dims 16 t + 4 j .. (even steps), 64 further (odd steps)
        float rs[NT][2], qz[NT][2];             // of the columns 2 t, 2 t + 1: what a product and a row's offset count for
        float o[NT][8][4];                      // O^T: dim 8 g + i (first two), 64 + 8 g + i, of the columns 2 t, 2 t + 1
        float m[NT][2], l[NT][2], z[NT][2];     // running maximum; this lane's share of sum p and sum p z
        float r_cur = 0.f;                      // what the scales are multiplied with in P^T
        bool fresh = true;
        int run_index = 0, run_unit0 = w.unit;

        for (int n = 0; n < cnt; ++n) {
            if (fresh) {
                fresh = false;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    const int h = nt * 8 + g;
                    uint4 v[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] = make_uint4(0, 0, 0, 0);
                    if (h < p.G) {
                        const uint4 *src = reinterpret_cast<const uint4 *>(p.q + ((size_t)w.b * p.Hq + (size_t)w.head * p.G + h) * kHeadDim);
                        v[0] = __ldg(src + 2 * t), v[1] = __ldg(src + 2 * t + 1), v[2] = __ldg(src + 8 + 2 * t), v[3] = __ldg(src + 9 + 2 * t);
                    }
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
                        m[nt][k] = -INFINITY;
                        l[nt][k] = z[nt][k] = 0.f;
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[nt][i][0] = o[nt][i][1] = o[nt][i][2] = o[nt][i][3] = 0.f;
                }
                r_cur = 0.f;
            }
            const int s = n % kD4Stages;
            const int n_tok = min(kD4Unit, w.len - w.unit * kD4Unit);
            if (!tc::mbar_wait(bar(s), (uint32_t)(n / kD4Stages) & 1u, ok ? (1u << 18) : 1u, flags)) {
                ok = false;
                flags[0] = 1;
            }
            __syncwarp();
            unsigned char *stage = smem + L::kRing + (warp * kD4Stages + s) * kD4StageBytes;
            if (kStep && ok && w.unit == w.units - 1 && __ldg(p.kv_len + w.b) == w.len) {
                // ---- the new token: quantised here, stored in the cache and in the unit's copy of it
                const int kv = lane >> 4, i = lane & 15, row = n_tok - 1, pos = w.len - 1;
                uint32_t codes, pair;
                d4_quantise((kv ? p.v_new : p.k_new) + ((size_t)w.b * p.Hkv + w.head) * kHeadDim, i, codes, pair);
                reinterpret_cast<uint32_t *>(stage + kv * kD4CodeBytes + row * kRow4Bytes)[i] = codes;
                if (i == 0) reinterpret_cast<uint32_t *>(stage + 2 * kD4CodeBytes + kv * kD4PairBytes)[row] = pair;
                const int page = __ldg(p.block_table + (size_t)w.b * p.max_pages_per_seq + (pos >> 7));
                if (page >= 0 && page < p.num_pages) {
                    const int slot = pos & (kPageTokens - 1);
                    uint8_t *dst = const_cast<uint8_t *>(p.codes) + code4_block_offset(page, w.head, kv, p.Hkv) + (size_t)slot * kRow4Bytes;
                    reinterpret_cast<uint32_t *>(dst)[i] = codes;
                    if (i == 0) const_cast<uint32_t *>(p.pairs)[scale_block_offset(page, w.head, kv, p.Hkv) + slot] = pair;
                }
                tc::fence_proxy_async();   // (the stage is filled by the copy engine again)
                __syncwarp();
            }
            const uint32_t *kp = reinterpret_cast<const uint32_t *>(stage + 2 * kD4CodeBytes), *vp = kp + kD4Unit;
            const int row = g ^ ((g >> 1) & 1);           // token of this lane's row: neighbouring rows lie in opposite halves of the banks
            const bool whole = n_tok == kD4Unit;

            // ---- S^T = K Q^T: rows g and g + 8 of every 16 tokens
            float c[4][NT][4];
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) c[mt][nt][0] = c[mt][nt][1] = c[mt][nt][2] = c[mt][nt][3] = 0.f;
                if (mt * 16 < n_tok) {
                    const uint4 a4 = *reinterpret_cast<const uint4 *>(stage + (mt * 16 + row) * kRow4Bytes + t * 16);
                    const uint4 b4 = *reinterpret_cast<const uint4 *>(stage + (mt * 16 + 8 + row) * kRow4Bytes + t * 16);
                    const uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w}, b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t a8 = a[j] >> 8, b8 = b[j] >> 8;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            d4_mma(c[mt][nt], a[j] & 0x000F000Fu, b[j] & 0x000F000Fu, a8 & 0x000F000Fu, b8 & 0x000F000Fu, qf[nt][2 * j][0], qf[nt][2 * j][1]);
                            d4_mma(c[mt][nt], a[j] & 0x00F000F0u, b[j] & 0x00F000F0u, a8 & 0x00F000F0u, b8 & 0x00F000F0u, qf[nt][2 * j + 1][0], qf[nt][2 * j + 1][1]);
                        }
                    }
                }
            }
            // ---- scores, their maxima, the largest V scale
            float mt_max[NT][2], sv_max = 0.f;
            float sv[4][2], zv[4][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) mt_max[nt][0] = mt_max[nt][1] = -INFINITY;
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int tok = mt * 16 + hf * 8 + row;
                    const bool seen = whole || tok < n_tok;   // (what lies behind the last token may be anything)
                    const uint32_t k2 = seen ? kp[tok] : 0u, v2 = seen ? vp[tok] : 0u;
                    const float sk = pair_scale(k2), zk = pair_offset(k2);
                    sv[mt][hf] = pair_scale(v2), zv[mt][hf] = pair_offset(v2);
                    sv_max = fmaxf(sv_max, sv[mt][hf]);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const float x = fmaf(c[mt][nt][2 * hf + k], sk * rs[nt][k], zk * qz[nt][k]);
                            c[mt][nt][2 * hf + k] = seen ? x : -INFINITY;
                            mt_max[nt][k] = fmaxf(mt_max[nt][k], c[mt][nt][2 * hf + k]);
                        }
                    }
                }
            }
            bool grow = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    mt_max[nt][k] = d4_max_rows(mt_max[nt][k]);
                    grow |= mt_max[nt][k] > m[nt][k] + kD4Grow;
                }
            }
            sv_max = d4_max_rows(sv_max);
            grow |= sv_max * r_cur >= 4.f * kD4Top || r_cur == 0.f;
            if (__any_sync(0xffffffffu, grow)) {
                const float top = (r_cur == 0.f) ? sv_max : fmaxf(sv_max, 0.f);
                const float r_new = (r_cur == 0.f || sv_max * r_cur >= 4.f * kD4Top) ? pow2_recip(pow2_floor(top)) * kD4Top : r_cur;
                const float fr = (r_cur == 0.f) ? 0.f : r_new / r_cur;
                r_cur = r_new;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) {
                    float al[2];
#pragma unroll
                    for (int k = 0; k < 2; ++k) {
                        const float m_new = fmaxf(m[nt][k], mt_max[nt][k]);
                        al[k] = d4_exp2(m[nt][k] - m_new);
                        m[nt][k] = m_new;
                        l[nt][k] *= al[k];
                        z[nt][k] *= al[k];
                        al[k] *= fr;
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
            // ---- P^T, and O^T += V^T P^T
#pragma unroll
            for (int mt = 0; mt < 4; ++mt) {
                if (mt * 16 >= n_tok) continue;
                uint32_t b[NT][2];
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const float sr = sv[mt][hf] * r_cur;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        float e[2];
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            e[k] = d4_exp2(c[mt][nt][2 * hf + k] - m[nt][k]);
                            l[nt][k] += e[k];
                            z[nt][k] = fmaf(e[k], zv[mt][hf], z[nt][k]);
                        }
                        b[nt][hf] = d4_transpose(pack_half2(e[0] * sr, e[1] * sr));
                    }
                }
                // token rows 2 t and 2 t + 1 (this lane's column pair of the operand) and the two eight further
                const unsigned char *v0 = stage + kD4CodeBytes + (mt * 16 + (2 * t ^ (t & 1))) * kRow4Bytes + 8 * g;
                const unsigned char *v1 = stage + kD4CodeBytes + (mt * 16 + ((2 * t + 1) ^ (t & 1))) * kRow4Bytes + 8 * g;
                const uint2 va = *reinterpret_cast<const uint2 *>(v0), vb = *reinterpret_cast<const uint2 *>(v1);
                const uint2 vc = *reinterpret_cast<const uint2 *>(v0 + 8 * kRow4Bytes), vd = *reinterpret_cast<const uint2 *>(v1 + 8 * kRow4Bytes);
#pragma unroll
                for (int w2 = 0; w2 < 2; ++w2) {
                    const uint32_t wa = w2 ? va.y : va.x, wb = w2 ? vb.y : vb.x, wc = w2 ? vc.y : vc.x, wd = w2 ? vd.y : vd.x;
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const uint32_t x = __byte_perm(wa, wb, half ? 0x7632 : 0x5410), y = __byte_perm(wc, wd, half ? 0x7632 : 0x5410);
                        const uint32_t x8 = x >> 8, y8 = y >> 8;
                        const int i = 4 * w2 + 2 * half;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            d4_mma(o[nt][i], x & 0x000F000Fu, x & 0x00F000F0u, y & 0x000F000Fu, y & 0x00F000F0u, b[nt][0], b[nt][1]);
                            d4_mma(o[nt][i + 1], x8 & 0x000F000Fu, x8 & 0x00F000F0u, y8 & 0x000F000Fu, y8 & 0x00F000F0u, b[nt][0], b[nt][1]);
                        }
                    }
                }
            }
            __syncwarp();              // every lane has read the stage
            if (issued < cnt) issue();

            // ---- the end of the pair, or of the range
            const bool ends = w.unit == w.units - 1;
            if (ends || n == cnt - 1) {
                const bool complete = ends && run_unit0 == 0;
                const float f1 = 16777216.f / r_cur, f2 = f1 * 0.0625f;    // the codes counted 2^-24 and 2^-20
                float *rec = reinterpret_cast<float *>(run_index == 0 ? smem + L::kFirst + warp * L::kRecFloats * 4
                                                                      : smem + L::kRing + warp * (kD4Stages * kD4StageBytes));
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
                            hi[i] = fmaf(o[nt][i][2 + k], f2, zs);
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
                                rec[L::kHeads * kHeadDim + h] = m[nt][k];
                                rec[L::kHeads * (kHeadDim + 1) + h] = ls;
                            }
                        }
                    }
                }
                if (!complete && lane == 0 && ok) {
                    D4Run &run = runs[2 * warp + (run_index == 0 ? 0 : 1)];
                    run.pair = w.b * p.Hkv + w.head;
                    run.units = w.units;
                    run.first = u0 + n - w.unit;
                }
                ++run_index;
                run_unit0 = 0;
                fresh = true;
            }
            if (n + 1 < cnt) w.next(p);
        }
        if (!ok) {   // copies still in flight get a bounded chance to land
            for (int i = max(0, issued - kD4Stages); i < issued; ++i) tc::mbar_wait(bar(i % kD4Stages), (uint32_t)(i / kD4Stages) & 1u, 1u << 14);
        }
    }
    // sequences without tokens: zeros
    for (int b = blockIdx.x; b < p.B; b += gridDim.x) {
        if (d4_len(p, b) != 0) continue;
        uint4 *dst = reinterpret_cast<uint4 *>(p.out + (size_t)b * p.Hq * kHeadDim);
        for (int i = tid; i < p.Hq * (kHeadDim / 8); i += kD4Warps * 32) dst[i] = make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    if (flags[0] != 0) {
        if (tid == 0) atomicExch(p.status, SLIM_ERR_TIMEOUT);
        return;
    }

    // ---- records of the block's warps, in the order of the units: consecutive ones of one pair are merged
    const long long block0 = d4_div(U * blockIdx.x, gridDim.x), block1 = d4_div(U * (blockIdx.x + 1), gridDim.x);
    auto record = [&](int e) {
        return reinterpret_cast<const float *>((e & 1) ? smem + L::kRing + (e >> 1) * (kD4Stages * kD4StageBytes)
                                                       : smem + L::kFirst + (e >> 1) * L::kRecFloats * 4);
    };
    int task = 0, prev = -1;
    for (int e = 0; e < 2 * kD4Warps; ++e) {
        const D4Run run = runs[e];
        if (run.pair < 0 || run.pair == prev) continue;
        prev = run.pair;
        const bool complete = run.first >= block0 && run.first + run.units <= block1;
        const int which = (run.first <= block0) ? 0 : 1;   // (of an incomplete one: the pair at the block's start, or at its end)
        float *part = p.parts + ((size_t)blockIdx.x * 2 + which) * L::kRecFloats;
        for (int h = 0; h < p.G; ++h) {
            if (task++ % kD4Warps != warp) continue;
            D4Merge acc;
            for (int x = e; x < 2 * kD4Warps; ++x) {
                if (runs[x].pair != run.pair) {
                    if (runs[x].pair >= 0) break;
                    continue;
                }
                const float *rec = record(x);
                acc.add(rec[L::kHeads * kHeadDim + h], rec[L::kHeads * (kHeadDim + 1) + h], reinterpret_cast<const float4 *>(rec + h * kHeadDim)[lane]);
            }
            if (complete) {
                acc.write(p.out + ((size_t)(run.pair / p.Hkv) * p.Hq + (size_t)(run.pair % p.Hkv) * p.G + h) * kHeadDim + 4 * lane);
            } else {
                __stcg(reinterpret_cast<float4 *>(part + h * kHeadDim) + lane, acc.o);
                if (lane == 0) {
                    __stcg(part + L::kHeads * kHeadDim + h, acc.m);
                    __stcg(part + L::kHeads * (kHeadDim + 1) + h, acc.l);
                }
            }
        }
        if (!complete && tid == 0) runs[2 * kD4Warps + which] = run;
    }
    __threadfence();   // this thread's part of a record is visible before the block's arrival is counted
    __syncthreads();
    // ---- pairs that span blocks: the block that arrives last merges them
    auto holder = [&](long long x) { return (int)(d4_div((x + 1) * gridDim.x - 1, U)); };   // the block whose range holds unit x
    if (tid < 2 && runs[2 * kD4Warps + tid].pair >= 0) {
        const D4Run run = runs[2 * kD4Warps + tid];
        const int i0 = holder(run.first), i1 = holder(run.first + run.units - 1);
        const int expected = (U >= gridDim.x) ? i1 - i0 + 1 : run.units;   // (with fewer units than blocks every one has a block of its own)
        if (atomicAdd(p.counters + i0, 1) + 1 == expected) {
            p.counters[i0] = 0;   // ready for the next launch
            __threadfence();
            flags[1 + tid] = 1;
        }
    }
    __syncthreads();
    for (int which = 0; which < 2; ++which) {
        if (flags[1 + which] == 0) continue;
        const D4Run run = runs[2 * kD4Warps + which];
        const int i0 = holder(run.first);
        const int n_parts = (U >= gridDim.x) ? holder(run.first + run.units - 1) - i0 + 1 : run.units;
        for (int h = warp; h < p.G; h += kD4Warps) {
            D4Merge acc;
            for (int x = 0; x < n_parts; ++x) {
                const int i = (U >= gridDim.x) ? i0 + x : holder(run.first + x);
                const int slot = (run.first <= d4_div(U * i, gridDim.x)) ? 0 : 1;
                const float *part = p.parts + ((size_t)i * 2 + slot) * L::kRecFloats;
                acc.add(__ldcg(part + L::kHeads * kHeadDim + h), __ldcg(part + L::kHeads * (kHeadDim + 1) + h),
                        __ldcg(reinterpret_cast<const float4 *>(part + h * kHeadDim) + lane));
            }
            acc.write(p.out + ((size_t)(run.pair / p.Hkv) * p.Hq + (size_t)(run.pair % p.Hkv) * p.G + h) * kHeadDim + 4 * lane);
        }
    }
}

constexpr int kD4MaxBlocks = 256;

size_t decode4_workspace_bytes(int G)
{
    const size_t heads = (G <= 8) ? 8 : 16;
    return kDecodeHeaderBytes + (size_t)kD4MaxBlocks * 2 * heads * (kHeadDim + 2) * sizeof(float);
}

template <int NT, bool kStep>
static int launch_d4(const Decode4Params &p, int blocks, cudaStream_t stream)
{
    const int rc = allow_dynamic_smem(reinterpret_cast<const void *>(slim4_decode_kernel<NT, kStep>), (int)D4<NT>::kBytes);
    if (rc != SLIM_OK) return rc;
    SLIM_CUDA_TRY(launch_pdl(slim4_decode_kernel<NT, kStep>, dim3((unsigned)blocks), dim3(kD4Warps * 32), D4<NT>::kBytes, stream, p));
    return SLIM_OK;
}

int launch_decode4(const slim_cache4_t *c, const void *q, const void *k_new, const void *v_new, void *out, const int32_t *kv_len, int B,
                   int max_kv, int Hq, float sm_scale, void *workspace, cudaStream_t stream)
{
    Decode4Params p;
    p.codes = c->codes;
    p.pairs = reinterpret_cast<const uint32_t *>(c->scales);
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
    int sms = 0;
    int rc = sm_count(&sms);
    if (rc != SLIM_OK) return rc;
    const long long units = (long long)B * p.Hkv * ((max_kv + kD4Unit - 1) / kD4Unit);
    long long blocks = units < sms ? units : sms;
    if (blocks > kD4MaxBlocks) blocks = kD4MaxBlocks;
    if (blocks < 1) blocks = 1;
    if (p.G <= 8)
        return k_new != nullptr ? launch_d4<1, true>(p, (int)blocks, stream) : launch_d4<1, false>(p, (int)blocks, stream);
    return k_new != nullptr ? launch_d4<2, true>(p, (int)blocks, stream) : launch_d4<2, false>(p, (int)blocks, stream);
}

}  // namespace slim

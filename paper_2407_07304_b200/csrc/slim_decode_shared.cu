// Decode attention of a batch whose sequences share a long prefix (the same pages in their page tables).
//
// Sequence b of a group attends over the prefix's tokens [0, shared_len[b]) and its own tail.  Attention over the prefix is
// computed once for all rows of the group: the G query heads of every sequence that read one kv head are stacked into
// the rows of one matrix, so the prefix's codes are read once instead of once per sequence and the products become
// matrix products:
//   prefix   (m, l, O)_row,split = softmax partial of the row over a part of the prefix     (kernel below)
//   tail     (m, l, O)_row,chunk = the split pass over the tokens behind the prefix          (slim_decode_stream.cu)
//   result   log-sum-exp merge of all of a row's partials                                    (slim_decode.cu)
//
// Prefix kernel: a block owns up to 256 stacked rows of one (group, kv head) and one contiguous part of the prefix's 128-key
// tiles; the number of parts fills the chip once.  The structure is that of the prefill kernel: TMA-staged INT8
// tiles, converted in registers into fp16 operands, scores and outputs on tcgen05 with accumulators in tensor memory, thread = row in the softmax, rescaling only when the maximum grows by more than 2^8.
// K's operand is the codes, exact in fp16, and so are the queries but for elements below 2^-17 of their row's largest; a key's
// scale is multiplied in the softmax.  So a score is as exact as fp32 sums are, whatever its size: rounded to fp16, 128 terms
// of a score of 350 move it by up to 0.1, and its weight by a tenth (with 2.6 us per key tile of 256 rows instead of 3.0).
// P and V are rounded to fp16 (V's scale, then its product with the code): each of a result's terms is off by 2^-10 at most,
// independently of one another, beside the 2^-8 of the result's own rounding to bf16.
// With more than 128 rows the block's two softmax groups take 128 rows each and every key tile serves both; with at
// most 128 rows both groups work on the same rows and take the key tiles in turn, so that the scores of one tile are
// formed while the softmax of the other runs, and their two partials are merged through shared memory at the end.
// The causal mask of the prefill kernel becomes a limit per row (a sequence may be shorter than the prefix).
//
// The tail kernel is launched as a programmatic dependent that does not wait for this one: its blocks run beside the
// prefix blocks, on the SMs left to them, and only their end waits for the prefix kernel (the merge kernel waits for the
// tail's).  What came before this kernel in the stream they see by a flag that it raises behind its own wait: about 1 us of
// a call, against 8 to 14 us for a tail behind the prefix.
#include <cuda.h>

#include <type_traits>

#include "slim_common.cuh"
#include "slim_decode_params.cuh"
#include "slim_quant.cuh"
#include "slim_tcgen05.cuh"
#include "slim_tmap.cuh"

namespace slim {

constexpr int kShThreads = 512;                // softmax groups 0 and 1, converters, {loader, MMA thread, two converter warps}
constexpr int kShTileRows = 128, kShKeys = 128;
constexpr int kShRows = 2 * kShTileRows;       // stacked rows per block
constexpr int kShConvWarps = 6;
constexpr uint32_t kShTmemCols = 512;
constexpr uint32_t kShTmemS = 0, kShTmemO = 256;   // S_t at columns 128 t, O_t at 256 + 128 t
constexpr float kShRescaleThreshold = 8.f;     // log2 units

namespace shl {   // shared-memory map
constexpr uint32_t kQ = 0;                      // two fp16 Q tiles; a tile = two 64-dim halves of [128 rows][128 B]
constexpr uint32_t kKf = 65536;                 // two fp16 K tiles (even / odd key tiles)
constexpr uint32_t kVf = kKf + 2 * 32768;       // two fp16 V tiles
constexpr uint32_t kRaw = kVf + 2 * 32768;      // raw INT8 tiles: stage 0 K, stage 1 V
constexpr uint32_t kRawScales = kRaw + 2 * 16384;   // of the raw V tile
// The keys' scales stay until the softmax of their tile has read them, and the loader is ahead of it: with 128 rows per
// group, when tile j is requested the products of tile j - 3 are done, which followed both groups' softmax of tile j - 4;
// with the tiles taken in turn, those of tiles j - 3 and j - 4, which followed the softmax of tiles j - 5 and j - 6.
constexpr uint32_t kKeyScales = kRawScales + 512;   // four key tiles
constexpr uint32_t kMisc = kKeyScales + 4 * 512;
// where the softmax groups take the key tiles in turn, the second Q tile is free: the keys' scales of eight key tiles, the
// rows' scales for group 1; and at the end, over the raw tiles, group 1's (m, l)
constexpr uint32_t kKeyScalesInTurn = kQ + 32768;
constexpr uint32_t kRowScale = kKeyScalesInTurn + 8 * 512;
constexpr uint32_t kMl = kRaw;
constexpr uint32_t kBytes = kMisc + 512;
// kMisc: floats by key tile mod 4: [0,4) log2 vexp, [4,8) 1 / vexp; byte 64: tensor-memory address;
//        byte 72: failure flag; byte 76: tokens of the prefix that any sequence of the group has; byte 128..: mbarriers
enum Bar { RAW_FULL = 0, RAW_EMPTY = 2, KF_FULL = 4, KF_EMPTY = 6, VF_FULL = 8, VF_EMPTY = 10,
           S_FULL = 12, P_FULL = 14, O_DONE = 16, Q_FULL = 18, VEXP_FULL = 20, NUM_BARS = 24 };
static_assert(128 + 8 * NUM_BARS <= 512, "mbarriers fit the misc area");
static_assert(kBytes <= 232448, "shared memory budget of one block");
}  // namespace shl

struct SharedParams {
    DecodeParams d;            // d.slot0 = parts of the prefix
    const int32_t *cu_group;   // [n_groups + 1]: the sequences of each group
    int B, max_group;
};

__device__ __forceinline__ float sh_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float sh_max3(float a, float b, float c)
{
    float m;
    asm("max.f32 %0, %1, %2, %3;\n" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
// halves: two fp16 numbers 1152 + code -> the codes, exactly, or code * factor
__device__ __forceinline__ uint32_t sh_code_pair(uint32_t halves)
{
    uint32_t d;
    asm("sub.rn.f16x2 %0, %1, %2;\n" : "=r"(d) : "r"(halves), "r"(0x64806480u));
    return d;
}
__device__ __forceinline__ uint32_t sh_value_pair(uint32_t halves, uint32_t factor)
{
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(sh_code_pair(halves)), "r"(factor));
    return r;
}

// The work of one block: rows m0 .. m0 + rows - 1 of the stack, key tiles j0 .. j0 + T - 1 of the prefix, T >= 1.
// by_rows: the softmax groups take 128 rows each; otherwise (at most 128 rows) they take the key tiles in turn, and T is
// even: behind the end of the prefix (`tiles`) an odd part gets one more tile, the last one's page again, all of it
// masked.  Two instances with equal step counts for both groups: with a flag at run time, or with counts T / 2 and
// (T + 1) / 2, the compiler spills the softmax group's score row (1.5 KB per thread against 100 bytes).
template <bool by_rows>
__device__ __forceinline__ void prefix_block(const CUtensorMap &codes_map, const SharedParams &sp, unsigned char *smem, int seq0, int seq1,
                                             int head, int m0, int rows, int j0, int T, int tiles)
{
    const DecodeParams &p = sp.d;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int split = blockIdx.x;
    // row m0 + r of the stack: sequence seq0 + (m0 + r) / G, query head head * G + (m0 + r) % G
    auto out_row = [&](int r) {
        const int s = (m0 + r) / p.G;
        return (size_t)(seq0 + s) * p.Hq + (size_t)head * p.G + (m0 + r - s * p.G);
    };
    const uint32_t sbase = smem_u32(smem);
    float *misc_f = reinterpret_cast<float *>(smem + shl::kMisc);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(smem + shl::kMisc + 64);
    volatile int *fail = reinterpret_cast<volatile int *>(smem + shl::kMisc + 72);
    int *known = reinterpret_cast<int *>(smem + shl::kMisc + 76);
    const uint32_t bar0 = sbase + shl::kMisc + 128;
    auto bar = [&](int which, int idx) { return bar0 + 8u * (uint32_t)(which + idx); };
    auto key_scales = [&](int j) { return by_rows ? shl::kKeyScales + (uint32_t)(j & 3) * 512u : shl::kKeyScalesInTurn + (uint32_t)(j & 7) * 512u; };

    // ---- the loader asks for the first raw tiles before the block's set-up is complete
    int raw_issued = 0;
    int page_next = 0;
    const int32_t *bt = p.block_table + (size_t)seq0 * p.max_pages_per_seq + j0;
    auto request_raw = [&](int i) {
        const int kv = i & 1, j = i >> 1;
        const int page = (page_next >= 0 && page_next < p.num_pages) ? page_next : 0;
        const uint32_t full = bar(shl::RAW_FULL, kv);
        tc::mbar_arrive_expect_tx(full, 16384 + 512);
        tc::tma_load_2d(sbase + shl::kRaw + kv * 16384, &codes_map, 0, ((page * p.Hkv + head) * 2 + kv) * kPageTokens, full);
        tc::bulk_load(sbase + (kv ? shl::kRawScales : key_scales(j)), p.scales + scale_block_offset(page, head, kv, p.Hkv), 512, full);
        if (kv == 1 && j + 1 < T) {
            // the next key tile's page id, and its two tiles on their way into the L2
            if (by_rows || j0 + j + 1 < tiles) page_next = __ldg(bt + j + 1);
            const int pn = (page_next >= 0 && page_next < p.num_pages) ? page_next : 0;
            tc::tma_prefetch_2d(&codes_map, 0, ((pn * p.Hkv + head) * 2) * kPageTokens);
            tc::tma_prefetch_2d(&codes_map, 0, ((pn * p.Hkv + head) * 2 + 1) * kPageTokens);
        }
        ++raw_issued;
    };
    if (warp == 12 && lane == 0) {
        for (int i = 0; i < 2; ++i) tc::mbar_init(bar(shl::RAW_FULL, i), 1);
        tc::mbar_init_fence();
        page_next = __ldg(bt);
        for (int i = 0; i < 2; ++i) request_raw(i);
    }
    // ---- query rows, sixteen lanes per row: warp w of group t brings in and converts rows 32 (w & 3) + 2 i + (lane >> 4) of
    //      its tile.  A row's 16-byte pieces go where their fp16 form will lie and are converted in place, so that both
    //      loops stay rolled: unrolled over registers they are 15 KB of instructions that every block runs once, and
    //      fetching those took longer than the rows.
    const bool has_q = warp < 8 && (warp < 4 || by_rows);
    const int q_row = (warp & 3) * 32 + (lane >> 4), q_piece = lane & 15;
    auto q_off = [&](int i) {   // (rows two apart: only the piece's slot depends on i beyond the stride)
        const int rr = q_row + 2 * i;
        return shl::kQ + (uint32_t)(warp >> 2) * 32768u + (uint32_t)(q_piece >> 3) * 16384u + (uint32_t)rr * 128u + (uint32_t)(((q_piece & 7) ^ (rr & 7)) << 4);
    };
    if (has_q) {
        const int r0 = (warp >> 2) * kShTileRows + q_row;
        int sq = (m0 + r0) / p.G, gq = m0 + r0 - sq * p.G;   // sequence and query head of row r0 + 2 i
        const __nv_bfloat16 *src = p.q + ((size_t)seq0 * p.Hq + (size_t)head * p.G) * kHeadDim + q_piece * 8;
#pragma unroll 4
        for (int i = 0; i < 16; ++i) {
            if (r0 + 2 * i < rows)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(sbase + q_off(i)),
                             "l"(src + ((size_t)sq * p.Hq + gq) * kHeadDim) : "memory");
            else
                *reinterpret_cast<uint4 *>(smem + q_off(i)) = make_uint4(0, 0, 0, 0);
            gq += 2;
            if (gq >= p.G) gq -= p.G, ++sq;
            if (gq >= p.G) gq -= p.G, ++sq;   // (one query head per kv head)
        }
        asm volatile("cp.async.commit_group;\n" ::: "memory");
    }
    if (warp == 14 && lane == 0) {   // (a warp that has nothing else to do here)
        for (int t = 0; t < 2; ++t) {
            tc::mbar_init(bar(shl::RAW_EMPTY, t), kShConvWarps);
            tc::mbar_init(bar(shl::KF_FULL, t), kShConvWarps);
            tc::mbar_init(bar(shl::KF_EMPTY, t), 1);
            tc::mbar_init(bar(shl::VF_FULL, t), kShConvWarps);
            tc::mbar_init(bar(shl::VF_EMPTY, t), 1);
            tc::mbar_init(bar(shl::S_FULL, t), 1);
            tc::mbar_init(bar(shl::P_FULL, t), 128);
            tc::mbar_init(bar(shl::O_DONE, t), 1);
            tc::mbar_init(bar(shl::Q_FULL, t), 128);
        }
        for (int i = 0; i < 4; ++i) tc::mbar_init(bar(shl::VEXP_FULL, i), 1);
        tc::mbar_init_fence();
        *fail = 0;
    }
    if (warp == 13) tc::tmem_alloc(smem_u32(tmem_slot), kShTmemCols);
    if (warp == 8) {
        // how many of the prefix's tokens any sequence of the group holds: rows behind them may hold anything
        int most = 0;
        for (int s = seq0 + lane; s < seq1; s += 32) most = max(most, min(__ldg(p.kv_len + s), decode_shared_tokens(p, s)));
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) *known = most;
    }
    tc::fence_before_sync();
    __syncthreads();
    tc::fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    bool ok = true;
    auto wait = [&](uint32_t mbar, uint32_t parity) {
        if (!tc::mbar_wait(mbar, parity, ok ? (1u << 18) : 1u, fail)) {
            ok = false;
            *fail = 1;
        }
    };
    // (2 * 160 + 96 + 96 = 4 * 128 registers per lane, as in the prefill kernel)
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 160;\n");
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 96;\n");
    }
    const int steps = by_rows ? T : T / 2;   // key tiles of each softmax group

    if (warp < 8) {
        // =========================================================== softmax of group t: thread = row
        const int t = warp >> 2;
        const int r = tid & 127;
        float *row_scale = reinterpret_cast<float *>(smem + shl::kRowScale);
        float rs = 0.f;   // row scale: sm_scale * log2(e) * the power of two that the row was divided by
        if (has_q) {
            // Q rows -> fp16, divided by a power of two near the row's absmax (the copy of bf16 is exact): thread = row, the
            // sixteen pieces in place
            unsigned char *at = smem + shl::kQ + (uint32_t)t * 32768u + (uint32_t)r * 128u;
            asm volatile("cp.async.wait_group 0;\n" ::: "memory");
            __syncwarp();   // the row was brought in by lanes of this warp
            uint32_t m2 = 0;
#pragma unroll 8
            for (int c = 0; c < 16; ++c) {
                const uint4 w = *reinterpret_cast<const uint4 *>(at + (c >> 3) * 16384 + (((c & 7) ^ (r & 7)) << 4));
                m2 = ap_max_bf16x2(m2, ap_max_bf16x2(ap_max_bf16x2(ap_abs_bf16x2(w.x), ap_abs_bf16x2(w.y)), ap_max_bf16x2(ap_abs_bf16x2(w.z), ap_abs_bf16x2(w.w))));
            }
            const float p2 = pow2_floor(fmaxf(__uint_as_float(m2 << 16), __uint_as_float(m2 & 0xFFFF0000u)));
            const float inv = copysignf(pow2_recip(p2), p.scale_log2e);   // (the factor c below is positive: a negative scale turns the row)
            const uint64_t inv2 = ap_pack(inv, inv);
#pragma unroll 4
            for (int c = 0; c < 16; ++c) {
                uint4 *piece = reinterpret_cast<uint4 *>(at + (c >> 3) * 16384 + (((c & 7) ^ (r & 7)) << 4));
                const uint4 raw = *piece;
                const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
                uint32_t hw[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    float x0, x1;
                    ap_unpack(ap_mul2(ap_pack(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u)), inv2), x0, x1);
                    hw[k] = pack_half2(x0, x1);
                }
                *piece = make_uint4(hw[0], hw[1], hw[2], hw[3]);
            }
            rs = p2 * fabsf(p.scale_log2e);
            if (!by_rows) row_scale[r] = rs;
            tc::fence_proxy_async();
        }
        if (!by_rows) {
            // group 1 works on group 0's rows
            tc::named_barrier(2, 256);
            rs = row_scale[r];
        }
        const int my_row = by_rows ? t * kShTileRows + r : r;      // row of the block
        const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t tS = tmem + lane_base + kShTmemS + (uint32_t)t * 128u;
        const uint32_t tO = tmem + lane_base + kShTmemO + (uint32_t)t * 128u;
        tc::mbar_arrive(bar(shl::Q_FULL, t));
        int limit = tiles * kShKeys;                               // keys that the row sees (rows of no sequence: their zero queries harm nothing)
        if (my_row < rows) {
            const int s = seq0 + (m0 + my_row) / p.G;
            limit = min(limit, min(__ldg(p.kv_len + s), decode_shared_tokens(p, s)));
        }
        const bool warp_rows = my_row - lane < rows;
        const float c = fmaxf(rs, 1e-37f);                         // (> 0)
        float m_run = -INFINITY, l_run = 0.f;
        for (int n = 0; n < steps; ++n) {
            const int j = by_rows ? n : 2 * n + t;                 // key tile of the block's part
            wait(bar(shl::S_FULL, t), (uint32_t)n & 1u);
            __syncwarp();
            tc::fence_after_sync();
            if (!warp_rows) {
                // no row of the stack in this warp: whatever lies in its score rows serves as P, nothing reads the result
                tc::fence_before_sync();
                tc::mbar_arrive(bar(shl::P_FULL, t));
                continue;
            }
            wait(bar(shl::VEXP_FULL, j & 3), (uint32_t)(j >> 2) & 1u);
            const float F = misc_f[j & 3];                         // log2 vexp
            const float vinv = misc_f[4 + (j & 3)];                // 1 / vexp
            const int key0 = (j0 + j) * kShKeys;
            uint32_t v[128];
            {
                uint32_t(&v0)[32] = *reinterpret_cast<uint32_t(*)[32]>(&v[0]);
                uint32_t(&v1)[32] = *reinterpret_cast<uint32_t(*)[32]>(&v[32]);
                uint32_t(&v2)[32] = *reinterpret_cast<uint32_t(*)[32]>(&v[64]);
                uint32_t(&v3)[32] = *reinterpret_cast<uint32_t(*)[32]>(&v[96]);
                tc::tmem_ld32(tS, v0);
                tc::tmem_ld32(tS + 32, v1);
                tc::tmem_ld32(tS + 64, v2);
                tc::tmem_ld32(tS + 96, v3);
                tc::tmem_ld_wait();
            }
            const float4 *ks = reinterpret_cast<const float4 *>(smem + key_scales(j));
#pragma unroll
            for (int i = 0; i < 128; i += 4) {
                const float4 k4 = ks[i / 4];
                float x0, x1, x2, x3;
                ap_unpack(ap_mul2(ap_pack(__uint_as_float(v[i]), __uint_as_float(v[i + 1])), ap_pack(k4.x, k4.y)), x0, x1);
                ap_unpack(ap_mul2(ap_pack(__uint_as_float(v[i + 2]), __uint_as_float(v[i + 3])), ap_pack(k4.z, k4.w)), x2, x3);
                v[i] = __float_as_uint(x0), v[i + 1] = __float_as_uint(x1), v[i + 2] = __float_as_uint(x2), v[i + 3] = __float_as_uint(x3);
            }
            if (__any_sync(0xffffffffu, key0 + kShKeys > limit)) {
#pragma unroll
                for (int i = 0; i < 128; ++i)
                    if (key0 + i >= limit) v[i] = 0xFF800000u;
            }
            float mx = -INFINITY, mx2 = -INFINITY;
#pragma unroll
            for (int i = 0; i < 128; i += 4) {
                mx = sh_max3(mx, __uint_as_float(v[i]), __uint_as_float(v[i + 1]));
                mx2 = sh_max3(mx2, __uint_as_float(v[i + 2]), __uint_as_float(v[i + 3]));
            }
            mx = fmaxf(mx, mx2);
            const float mt = (mx == -INFINITY) ? -INFINITY : fmaf(mx, c, F);
            const bool grow = (n == 0) ? true : (mt > m_run + kShRescaleThreshold);
            if (n > 0 && __any_sync(0xffffffffu, grow)) {
                const float alpha = grow ? sh_exp2(m_run - mt) : 1.f;   // m_run = -inf gives 0
                wait(bar(shl::O_DONE, t), (uint32_t)(n - 1) & 1u);
                __syncwarp();
                tc::fence_after_sync();
#pragma unroll 1
                for (int k = 0; k < 8; ++k) {
                    uint32_t o[16];
                    tc::tmem_ld16(tO + k * 16, o);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * alpha);
                    tc::tmem_st16(tO + k * 16, o);
                }
                tc::tmem_st_wait();
                l_run *= alpha;
            }
            if (grow) m_run = mt;
            const float bias = (m_run == -INFINITY) ? 0.f : F - m_run;
            const uint64_t c2 = ap_pack(c, c), bias2 = ap_pack(bias, bias);
            uint64_t sum2a = 0ull, sum2b = 0ull;
#pragma unroll
            for (int i = 0; i < 64; ++i) {
                float x0, x1;
                ap_unpack(ap_fma2(ap_pack(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1])), c2, bias2), x0, x1);
                const float e0 = sh_exp2(x0), e1 = sh_exp2(x1);
                if (i & 1) sum2b = ap_add2(sum2b, ap_pack(e0, e1)); else sum2a = ap_add2(sum2a, ap_pack(e0, e1));
                v[i] = pack_half2(e0, e1);
            }
            float rowsum, rowsum_hi;
            ap_unpack(ap_add2(sum2a, sum2b), rowsum, rowsum_hi);
            rowsum += rowsum_hi;
            {
                const uint32_t(&p0)[32] = *reinterpret_cast<const uint32_t(*)[32]>(&v[0]);
                const uint32_t(&p1)[32] = *reinterpret_cast<const uint32_t(*)[32]>(&v[32]);
                tc::tmem_st32(tS, p0);
                tc::tmem_st32(tS + 32, p1);
            }
            l_run = fmaf(rowsum, vinv, l_run);
            tc::tmem_st_wait();
            tc::fence_before_sync();
            tc::mbar_arrive(bar(shl::P_FULL, t));
        }

        // ---- epilogue: the rows go out through the operand buffers, 64 KB for each group, 16-byte piece c of row r in piece
        //      slot (c + r) mod 32 (no bank conflicts either way).  Behind group 0's last product all scores are complete, so
        //      the K buffers are free; behind group 1's, the block's last, the V buffers too.
        wait(bar(shl::O_DONE, t), (uint32_t)(steps - 1) & 1u);
        __syncwarp();
        tc::fence_after_sync();
        unsigned char *stage0 = smem + shl::kKf, *stage1 = smem + shl::kVf;
        float2 *ml1 = reinterpret_cast<float2 *>(smem + shl::kMl);
        if (!by_rows && t == 1) ml1[r] = make_float2(m_run, l_run);   // group 1 stages its rows first, group 0 adds them to its own
        if ((by_rows || t == 1) && warp_rows) {
            unsigned char *stage = (by_rows && t == 0) ? stage0 : stage1;
#pragma unroll
            for (int c4 = 0; c4 < 4; ++c4) {
                uint32_t o[32];
                tc::tmem_ld32(tO + c4 * 32, o);
                tc::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    *reinterpret_cast<uint4 *>(stage + r * 512 + (((c4 * 8 + i + r) & 31) << 4)) = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
        }
        if (!by_rows) {
            tc::named_barrier(1, 256);
            if (t == 0 && warp_rows) {
                const float2 other = ml1[r];
                const float M = fmaxf(m_run, other.x);
                const bool use_other = other.x != -INFINITY;
                const float w_own = (m_run == -INFINITY) ? 0.f : exp2f(m_run - M);
                const float w_other = use_other ? exp2f(other.x - M) : 0.f;
                l_run = l_run * w_own + (use_other ? other.y * w_other : 0.f);
                m_run = M;
#pragma unroll
                for (int c4 = 0; c4 < 4; ++c4) {
                    uint32_t o[32];
                    tc::tmem_ld32(tO + c4 * 32, o);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t at = r * 512 + (((c4 * 8 + i + r) & 31) << 4);
                        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
                        if (use_other) a = *reinterpret_cast<const float4 *>(stage1 + at);
                        float4 x;
                        x.x = fmaf(__uint_as_float(o[4 * i]), w_own, a.x * w_other);
                        x.y = fmaf(__uint_as_float(o[4 * i + 1]), w_own, a.y * w_other);
                        x.z = fmaf(__uint_as_float(o[4 * i + 2]), w_own, a.z * w_other);
                        x.w = fmaf(__uint_as_float(o[4 * i + 3]), w_own, a.w * w_other);
                        *reinterpret_cast<float4 *>(stage0 + at) = x;
                    }
                }
            }
        }
        if (by_rows || t == 0) {
            // coalesced: a warp writes one of its rows' 512 bytes per store
            const unsigned char *stage = t ? stage1 : stage0;
            __syncwarp();
            const size_t ps = my_row < rows ? out_row(my_row) * p.n_slots + split : 0;
            const bool all_ok = __all_sync(0xffffffffu, ok);   // (after a wait that ran out nothing is written, by no lane of the warp)
            if (my_row < rows && all_ok) *reinterpret_cast<float2 *>(p.part_ml + ps * 2) = make_float2(m_run, l_run);
            const int n_out = all_ok ? min(32, rows - (my_row - lane)) : 0;   // rows of this warp
#pragma unroll 4
            for (int i = 0; i < n_out; ++i) {
                const int rr = (warp & 3) * 32 + i;
                const size_t to = (size_t)__shfl_sync(0xffffffffu, (unsigned long long)ps, i);
                reinterpret_cast<float4 *>(p.part_o + to * kHeadDim)[lane] = *reinterpret_cast<const float4 *>(stage + rr * 512 + (((lane + rr) & 31) << 4));
            }
        }
    } else if (warp < 12 || warp >= 14) {
        // =========================================================== dequantise (as in the prefill kernel)
        const bool main_cv = warp < 12;
        const int r0 = main_cv ? tid - 256 : tid - 448;
        const int n_rows = main_cv ? 1 : 2, c_first = main_cv ? 0 : 6, c_last = main_cv ? 6 : 8;
        const bool announces = warp == 8 && lane == 0;
        const int kept = min(*known, tiles * kShKeys) - j0 * kShKeys;      // tokens of the block's part that exist
        auto convert = [&](auto kind, int j) {
            constexpr int kv = decltype(kind)::value;
            constexpr bool is_k = kv == 0;
            const int buf = j & 1;
            wait(bar(shl::RAW_FULL, kv), (uint32_t)j & 1u);
            const unsigned char *raw = smem + shl::kRaw + kv * 16384;
            const float *scales = reinterpret_cast<const float *>(smem + shl::kRawScales);
            const int n_valid = min(kShKeys, kept - j * kShKeys);
            float rex = 0.f;
            if (is_k) {
                wait(bar(shl::KF_EMPTY, buf), ((uint32_t)(j >> 1) & 1u) ^ 1u);
            } else {
                float wm = 0.f;
                const float4 s4 = *reinterpret_cast<const float4 *>(scales + 4 * lane);
                const float sv[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (4 * lane + k < n_valid) wm = fmaxf(wm, sv[k]);
                wm = warp_max(wm);
                const float ex = (wm > 0.f) ? pow2_floor(wm) : 1.f;
                rex = pow2_recip(ex);
                if (announces) {
                    misc_f[j & 3] = (float)((int)(__float_as_uint(ex) >> 23) - 127);
                    misc_f[4 + (j & 3)] = rex;
                    tc::mbar_arrive(bar(shl::VEXP_FULL, j & 3));   // (the keys' scales, too, have been seen to arrive)
                }
                wait(bar(shl::VF_EMPTY, buf), ((uint32_t)(j >> 1) & 1u) ^ 1u);
            }
            unsigned char *dst_tile = smem + (is_k ? shl::kKf : shl::kVf) + buf * 32768;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                if (q >= n_rows) break;
                const int r = r0 + 64 * q;
                uint32_t fac2 = 0;   // a value's scale / 2^e in [0, 2)
                if (!is_k) {
                    const float f = ((r < n_valid) ? scales[r] : 0.f) * rex;
                    fac2 = pack_half2(f, f);
                }
                unsigned char *dstb = dst_tile + r * 128;
                for (int c = c_first; c < c_last; ++c) {
                    const uint4 w4 = *reinterpret_cast<const uint4 *>(raw + r * 128 + ((c ^ (r & 7)) << 4));
                    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
                    uint32_t hh[8];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t x = w[k] ^ 0x80808080u;   // byte code ^ 0x80 under 0x64 is the fp16 number 1152 + code
                        const uint32_t h0 = __byte_perm(x, 0x64646464u, 0x4140), h1 = __byte_perm(x, 0x64646464u, 0x4342);
                        hh[2 * k] = is_k ? sh_code_pair(h0) : sh_value_pair(h0, fac2);
                        hh[2 * k + 1] = is_k ? sh_code_pair(h1) : sh_value_pair(h1, fac2);
                    }
                    const uint32_t hf = (uint32_t)(c >> 2) * 16384u;
                    const int oc = 2 * (c & 3);
                    *reinterpret_cast<uint4 *>(dstb + hf + ((oc ^ (r & 7)) << 4)) = make_uint4(hh[0], hh[1], hh[2], hh[3]);
                    *reinterpret_cast<uint4 *>(dstb + hf + (((oc + 1) ^ (r & 7)) << 4)) = make_uint4(hh[4], hh[5], hh[6], hh[7]);
                }
            }
            tc::fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                tc::mbar_arrive(bar(is_k ? shl::KF_FULL : shl::VF_FULL, buf));
                tc::mbar_arrive(bar(shl::RAW_EMPTY, kv));
            }
        };
        for (int j = 0; j < T; ++j) {
            convert(std::integral_constant<int, 0>(), j);
            convert(std::integral_constant<int, 1>(), j);
        }
    } else if (warp == 12) {
        // =========================================================== loader (one thread)
        if (lane == 0) {
            for (int i = 2; i < 2 * T; ++i) {
                wait(bar(shl::RAW_EMPTY, i & 1), ((uint32_t)(i >> 1) & 1u) ^ 1u);
                request_raw(i);
            }
        }
    } else {
        // =========================================================== MMA issue (one thread)
        if (lane == 0) {
            constexpr uint32_t idesc_qk = tc::instr_desc(1, 0, 0, false, false, 128, 128);
            constexpr uint32_t idesc_pv = tc::instr_desc(1, 0, 0, false, true, 128, 128);
            const uint64_t dq0 = tc::smem_desc(sbase + shl::kQ, 16, 1024, tc::kSwizzle128B);
            const uint64_t dk0 = tc::smem_desc(sbase + shl::kKf, 16, 1024, tc::kSwizzle128B);
            const uint64_t dv0 = tc::smem_desc(sbase + shl::kVf, 16384, 1024, tc::kSwizzle128B);
            auto issue_qk = [&](int t, int buf) {   // S_t = Q . K^T (the group's own rows, or both groups the same rows)
                const uint64_t dq = dq0 + (uint64_t)((by_rows ? t : 0) * (32768 >> 4));
                const uint64_t dk = dk0 + (uint64_t)(buf * (32768 >> 4));
                const uint32_t d = tmem + kShTmemS + (uint32_t)t * 128u;
#pragma unroll
                for (int ks = 0; ks < 8; ++ks) {
                    const uint64_t koff = (uint64_t)(((ks >> 2) * 16384 + (ks & 3) * 32) >> 4);
                    tc::mma_f16(d, dq + koff, dk + koff, idesc_qk, ks > 0);
                }
                tc::commit(bar(shl::S_FULL, t));
            };
            auto issue_pv = [&](int t, bool first, int buf) {   // O_t (+)= P_t . V
                const uint32_t d = tmem + kShTmemO + (uint32_t)t * 128u, a = tmem + kShTmemS + (uint32_t)t * 128u;
                const uint64_t dv = dv0 + (uint64_t)(buf * (32768 >> 4));
#pragma unroll
                for (int ks = 0; ks < 8; ++ks)
                    tc::mma_f16_ts(d, a + ks * 8, dv + (uint64_t)((ks * 2048) >> 4), idesc_pv, !first || ks > 0);
                tc::commit(bar(shl::O_DONE, t));
            };
            wait(bar(shl::Q_FULL, 0), 0);
            wait(bar(shl::Q_FULL, 1), 0);
            wait(bar(shl::KF_FULL, 0), 0);
            tc::fence_after_sync();
            issue_qk(0, 0);
            if (by_rows) {
                issue_qk(1, 0);
                tc::commit(bar(shl::KF_EMPTY, 0));
                for (int j = 0; j < T; ++j) {
                    const uint32_t ph = (uint32_t)j & 1u;
                    const int buf = j & 1, bufn = buf ^ 1;
                    const uint32_t bph = (uint32_t)(j >> 1) & 1u, bphn = (uint32_t)((j + 1) >> 1) & 1u;
                    const bool more = j + 1 < T;
                    wait(bar(shl::VF_FULL, buf), bph);
                    wait(bar(shl::P_FULL, 0), ph);
                    tc::fence_after_sync();
                    issue_pv(0, j == 0, buf);
                    if (more) {
                        wait(bar(shl::KF_FULL, bufn), bphn);
                        tc::fence_after_sync();
                        issue_qk(0, bufn);
                    }
                    wait(bar(shl::P_FULL, 1), ph);
                    tc::fence_after_sync();
                    issue_pv(1, j == 0, buf);
                    tc::commit(bar(shl::VF_EMPTY, buf));
                    if (more) {
                        issue_qk(1, bufn);
                        tc::commit(bar(shl::KF_EMPTY, bufn));
                    }
                }
            } else {
                // group t takes key tiles t, t + 2, ...: tile j lies in operand buffers j & 1 = t
                tc::commit(bar(shl::KF_EMPTY, 0));
                wait(bar(shl::KF_FULL, 1), 0);
                tc::fence_after_sync();
                issue_qk(1, 1);
                tc::commit(bar(shl::KF_EMPTY, 1));
                for (int j = 0; j < T; ++j) {
                    const int t = j & 1;
                    const uint32_t ph = (uint32_t)(j >> 1) & 1u;
                    wait(bar(shl::VF_FULL, t), ph);
                    wait(bar(shl::P_FULL, t), ph);
                    tc::fence_after_sync();
                    issue_pv(t, j < 2, t);
                    tc::commit(bar(shl::VF_EMPTY, t));
                    if (j + 2 < T) {
                        wait(bar(shl::KF_FULL, t), (uint32_t)((j + 2) >> 1) & 1u);
                        tc::fence_after_sync();
                        issue_qk(t, t);
                        tc::commit(bar(shl::KF_EMPTY, t));
                    }
                }
            }
        }
    }

    tc::fence_before_sync();
    __syncthreads();
    if (warp == 12 && lane == 0 && *fail != 0) {
        // a wait ran out somewhere: give the copies still in flight a bounded chance to land before the block exits
        for (int i = max(0, raw_issued - 2); i < raw_issued; ++i)
            tc::mbar_wait(bar(shl::RAW_FULL, i & 1), (uint32_t)(i >> 1) & 1u, 1u << 14);
        if (p.status != nullptr) atomicExch(p.status, SLIM_ERR_TIMEOUT);
    }
    if (warp == 13) {
        __syncwarp();
        tc::fence_after_sync();
        tc::tmem_dealloc(tmem, kShTmemCols);
    }
}

// grid = (parts of the prefix, kv heads * row blocks, groups)
__global__ void __launch_bounds__(kShThreads, 1)
slim_decode_prefix_kernel(const __grid_constant__ CUtensorMap codes_map, const __grid_constant__ SharedParams sp)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    // The tail's blocks may start on the SMs that this kernel does not use once all of its blocks are here, behind the
    // wait.  They must not wait for this kernel's end, so the flag tells them that what came before it in the stream has
    // ended, and makes it visible to them.
    pdl_wait();
    if (blockIdx.x + blockIdx.y + blockIdx.z != 0) {
        pdl_launch_dependents();
    } else if (threadIdx.x == kShThreads - 32) {   // (a warp with nothing else to do yet; the tail starts behind this block's call, too)
        flag_raise(sp.d.begun);
        pdl_launch_dependents();
    }
    const DecodeParams &p = sp.d;
    const int head = (int)blockIdx.y % p.Hkv, m0 = (int)blockIdx.y / p.Hkv * kShRows;
    // (one group is all the sequences: nothing to look up)
    const bool one = gridDim.z == 1;
    const int seq0 = one ? 0 : min(max(__ldg(sp.cu_group + blockIdx.z), 0), sp.B);
    const int seq_end = one ? sp.B : min(max(__ldg(sp.cu_group + blockIdx.z + 1), 0), sp.B);
    const int seq1 = min(seq_end, seq0 + sp.max_group);      // (the launch has row blocks for max_group sequences)
    // what the merge finds for rows r0 .. r1 - 1 of the stack that begins at sequence s0: no keys, weight 0
    auto leave_empty = [&](int s0, int r0, int r1) {
        const int lane = threadIdx.x & 31;
        for (int r = r0 + (threadIdx.x >> 5); r < r1; r += kShThreads / 32) {
            const int s = r / p.G;
            const size_t ps = ((size_t)(s0 + s) * p.Hq + (size_t)head * p.G + (r - s * p.G)) * p.n_slots + blockIdx.x;
            reinterpret_cast<float4 *>(p.part_o + ps * kHeadDim)[lane] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (lane == 0) *reinterpret_cast<float2 *>(p.part_ml + ps * 2) = make_float2(-INFINITY, 0.f);
        }
    };
    if (m0 == 0 && !one) {
        // sequences beyond max_group of their group, and those of no group: the merge must not find what an earlier call left
        leave_empty(seq1, 0, (seq_end - seq1) * p.G);
        if (blockIdx.z == 0) leave_empty(0, 0, seq0 * p.G);
        if (blockIdx.z == gridDim.z - 1) leave_empty(max(seq_end, seq0), 0, (sp.B - max(seq_end, seq0)) * p.G);
    }
    const int R = (seq1 - seq0) * p.G;                       // stacked rows of the group and kv head
    if (m0 >= R) return;
    const int rows = min(kShRows, R - m0);
    const int split = blockIdx.x, tiles = decode_shared_tokens(p, seq0) / kShKeys;
    // the part's key tiles; where the softmax groups take them in turn, the prefix is cut into pairs of tiles
    const bool by_rows = rows > kShTileRows;
    const int unit = by_rows ? 1 : 2;
    const long long units = (tiles + unit - 1) / unit;
    const int j0 = unit * (int)(units * split / p.slot0), T = unit * (int)(units * (split + 1) / p.slot0) - j0;
    if (T <= 0) {
        leave_empty(seq0, m0, m0 + rows);   // a part without keys
        return;
    }
    if (by_rows) prefix_block<true>(codes_map, sp, smem, seq0, seq1, head, m0, rows, j0, T, tiles);
    else prefix_block<false>(codes_map, sp, smem, seq0, seq1, head, m0, rows, j0, T, tiles);
}

// ---------------------------------------------------------------- host side
struct SharedShape {
    int row_blocks, splits, slots, tail_blocks;
};

constexpr int kShSms = 148;

// How the work is divided over the SMs.  Prefix and tail blocks take an SM each and run side by side, so the number of
// parts of the prefix is chosen for the earliest end of both, by what their blocks were measured to take (us):
//   prefix block   10 + 3.0 per key tile of 256 rows; 13 + 1.4 where the softmax groups take the tiles in turn
//   tail           7 + (2 per 256-token chunk, 4 with more than eight query heads per kv head) / blocks
// The tails' lengths are device data: half of max_tail is taken for their mean, so where all tails are as long as max_tail
// the tails' SMs end later than the prefix's.  (Prefixes of 2048 / 8192 / 16384 tokens for 16 / 32 / 64 sequences: 27.7 / 34.1
// / 53 us.  When this was built, with the prefix on all SMs and the tail behind it 38.6 / 47.9 / 67.1, side by side 30.9 /
// 34.8 / 53.7.)
static SharedShape shared_shape(int B, int Hq, int Hkv, int n_groups, int max_group, int max_shared, int max_tail)
{
    SharedShape s;
    const int G = Hq / Hkv;
    const long long rows = (long long)max_group * G;
    s.row_blocks = (int)((rows + kShRows - 1) / kShRows);
    const bool by_rows = rows > kShTileRows;
    const int tiles = max_shared / kShKeys, unit = by_rows ? 1 : 2, units = (tiles + unit - 1) / unit;
    const long long per_part = (long long)Hkv * s.row_blocks * n_groups;
    const double chunks = (double)B * Hkv * (max_tail + 255) / 512, tail_work = chunks * (G <= 8 ? 2.0 : 4.0);
    s.splits = tiles > 0 ? 1 : 0;
    s.tail_blocks = kShSms;
    double best = 1e30;
    for (int n = 1; n <= units && n * per_part < kShSms; ++n) {
        const int tail_blocks = kShSms - (int)(n * per_part);
        const int part = unit * ((units + n - 1) / n);
        const double prefix = by_rows ? 10.0 + 3.0 * part : 13.0 + 1.4 * part;
        const double tail = max_tail > 0 ? 7.0 + tail_work / tail_blocks : 0.0;
        const double end = prefix > tail ? prefix : tail;
        if (end < best) best = end, s.splits = n, s.tail_blocks = tail_blocks;
    }
    s.slots = s.splits + (max_tail + 255) / 256 + 1;
    return s;
}

// Room for the partials of every call with at most these sequences, groups and bounds, so that a workspace made for the
// largest serves the smaller ones too.  The division above does not grow with them (a shorter tail leaves more SMs to the
// prefix, and so more parts), so the prefix's partials are bounded by what any division of such a call can have: one part, or
// n parts with n * Hkv * row_blocks * n_groups < kShSms, never more than the prefix has units; and as B <= n_groups * max_group,
//   n * B * Hq < kShSms * max_group * G / row_blocks <= kShSms * min(max_group * G, kShRows).
size_t shared_workspace_bytes(int B, int Hq, int Hkv, int n_groups, int max_group, int max_shared, int max_tail)
{
    const long long rows = (long long)B * Hq, stack = (long long)max_group * (Hq / Hkv);
    const int tiles = max_shared / kShKeys, units = stack > kShTileRows ? tiles : (tiles + 1) / 2;
    long long prefix = 0;
    if (tiles > 0) {
        prefix = kShSms * (stack < kShRows ? stack : kShRows);
        if (prefix > rows * units) prefix = rows * units;
        if (prefix < rows) prefix = rows;
    }
    const long long tail = rows * (((long long)max_tail + 255) / 256 + 1);
    return kDecodeHeaderBytes + (size_t)(prefix + tail) * (kHeadDim + 2) * sizeof(float);
}

int launch_decode_shared(const slim_cache_t *c, const void *q, const void *k_new, const void *v_new, void *out, const int32_t *cu_group,
                         const int32_t *shared_len, const int32_t *kv_len, int n_groups, int B, int max_group, int max_shared,
                         int max_tail, int Hq, float sm_scale, void *workspace, cudaStream_t stream)
{
    const SharedShape s = shared_shape(B, Hq, c->num_kv_heads, n_groups, max_group, max_shared, max_tail);
    // no prefix of a page or more: ordinary decode
    if (s.splits == 0) return launch_decode(c, q, k_new, v_new, out, kv_len, B, max_tail, Hq, sm_scale, workspace, stream);
    if ((long long)c->num_kv_heads * s.row_blocks > 65535) return SLIM_ERR_UNSUPPORTED;
    DecodeParams p = make_decode_params(c, q, kv_len, B, max_tail, Hq, sm_scale, workspace);
    p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = static_cast<const __nv_bfloat16 *>(v_new);
    p.shared_len = shared_len;
    p.max_shared_pages = max_shared / kPageTokens;
    p.begun = p.status + 1;
    p.slot0 = s.splits;
    p.n_slots = s.slots;
    p.max_blocks = s.tail_blocks;
    p.part_ml = p.part_o + (size_t)B * Hq * p.n_slots * kHeadDim;
    SharedParams sp;
    sp.d = p;
    sp.cu_group = cu_group;
    sp.B = B;
    sp.max_group = max_group;
    CUtensorMap map;
    int rc = codes_tensor_map(c, kShKeys, &map);
    if (rc != SLIM_OK) return rc;
    rc = allow_dynamic_smem(reinterpret_cast<const void *>(slim_decode_prefix_kernel), (int)shl::kBytes);
    if (rc != SLIM_OK) return rc;
    const dim3 grid((unsigned)s.splits, (unsigned)(c->num_kv_heads * s.row_blocks), (unsigned)n_groups);
    SLIM_CUDA_TRY(launch_pdl(slim_decode_prefix_kernel, grid, dim3(kShThreads), (size_t)shl::kBytes, stream, map, sp));
    if (p.n_chunks > 0) {
        rc = launch_decode_split_stream(c, p, B, stream);
        if (rc != SLIM_OK) return rc;
    }
    return launch_merge_rows(p, B, out, nullptr, stream);
}

}  // namespace slim

// Norm of every query and key head and rotation by position, in one pass over the rows, and the same pass with the
// keys and values quantised into the INT8 cache (Section 2.2) instead of being written back.
//
//   n_d   = x_d * w_d / sqrt(mean_e x_e^2 + eps)                       (without a weight: n = x)
//   a_i   = position[axis_i] * inv_freq_i                              i < rotary_dim / 2
//   (y_f, y_s) = (n_f cos a_i - n_s sin a_i, n_f sin a_i + n_s cos a_i) for the i-th pair (f, s) of dimensions
//   out   = bf16(y);  cached row: code = round_half_even(127 y_d / max|y|), scale = max|y| / 127
//
// Everything between the bf16 input and the result is fp32; a value is rounded once, to bf16 or to its code (the key
// that goes into the cache is never rounded to bf16 on the way).  The angle is formed in fp64 as a number of turns,
// whole turns are dropped there, and only the remaining fraction is rounded to fp32: at position 2^20 an fp32 angle
// would be off by 2^-4, this one by 2^-22 of a turn.
//
// The kernel is bound by memory traffic (read and write every row once).  Four lanes own a row, as in the append
// kernel: lane l holds the 16-byte pieces l, l + 4, l + 8, l + 12, so a load instruction of a warp covers eight rows
// in whole 64-byte sectors, and the two halves of a 128- or 64-dimension rotation lie in the same lane.  Narrower
// rotations in halves (rotary_dim other than 64 and 128) read the partner piece a second time, from the L1.
// A block takes 32 consecutive rows (token-major: the token's query heads, key heads, value heads); the cosines and
// sines of the few tokens that it touches are computed once per block, by all its threads, while the rows are on
// their way, so no table of angles is read from memory.
#include "slim_common.cuh"
#include "slim_quant.cuh"

namespace slim {

// (Blocks of 128 threads, nine per SM: 54 us for a prompt of 16384 tokens with 32 query heads on 2 kv heads, 5.4 TB/s;
// 256 threads 61 us, 64 threads 58 us; several batches of rows per block, or the weights folded into the angles' table
// with packed arithmetic, take registers and with them blocks, and were 5 to 25 % slower.)
constexpr int kNrThreads = 128;
constexpr int kNrLanes = 4;                             // lanes per row
constexpr int kNrRows = kNrThreads / kNrLanes;          // rows per block

// how the pairs of a rotation lie in a row
constexpr int kNrHalvesInLane = 0;   // pair (i, i + half), half a multiple of 32: both in one lane
constexpr int kNrAdjacent = 1;       // pair (2 i, 2 i + 1)
constexpr int kNrHalvesReload = 2;   // pair (i, i + half), half a multiple of 8

struct NormRopeParams {
    const __nv_bfloat16 *src[3];      // query, key and value rows; tokens src_stride elements apart
    long long src_stride[3];
    __nv_bfloat16 *dst[2];            // bf16 [token][heads][128] of the queries and (without a cache) the keys
    const __nv_bfloat16 *weight[2];   // norm weights of queries and keys, or null
    const double *inv_freq;
    const uint8_t *axis;
    const int32_t *positions;         // [n_axes][n_tokens], or null: the token's position in its cache
    // the cache (append only)
    int8_t *codes;
    float *scales;
    const int32_t *block_table, *cu_new, *start_pos;
    int B, max_pages_per_seq, num_pages;
    int n_tokens, Hq, Hkv, rows_per_token, half, n_axes, span;
    float eps;
};

// The sequence that row `tok` of the concatenated new tokens belongs to: the last b with cu[b] <= tok (sequences without
// new tokens repeat a start).  One warp; every round divides the candidates by 32.
__device__ __forceinline__ int nr_find_sequence(const int32_t *cu, int B, int tok, int lane)
{
    int lo = 0, n = B;   // the answer is one of lo .. lo + n - 1, and cu[lo] <= tok
    while (n > 1) {
        const int step = (n + 31) / 32;
        const int i = lo + lane * step;
        const bool le = lane * step < n && __ldg(cu + i) <= tok;
        const unsigned hits = __ballot_sync(0xffffffffu, le);
        const int last = hits ? 31 - __clz((int)hits) : 0;   // starts ascend, so the hits are the first lanes
        const int end = lo + n;
        lo += last * step;
        n = min(step, end - lo);
    }
    return lo;
}

// 32 values of a row of 128 owned by four consecutive lanes -> the codes of its four pieces and the row's scale: the
// quantiser of slim_quant.cuh on fp32 values (for values that are bf16 the same codes and scale bit for bit; for others
// 127 x is rounded to fp32 before the quotient, 2^-24 of it).  All lanes of a warp call it together.
__device__ __forceinline__ void nr_quantize(const float (&x)[32], uint2 (&pk)[4], float &scale)
{
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) amax = fmaxf(amax, fabsf(x[i]));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    float f = 1.f;
    if (amax < 0x1p-60f) f = 0x1p64f;
    else if (amax > 0x1p60f) f = 0x1p-64f;
    const float as = __fmul_rn(amax, f), m127 = __fmul_rn(127.f, f);
    const float rc = (amax > 0.f) ? __frcp_rn(as) : 0.f;
    const uint64_t m127_2 = ap_pack(m127, m127), rc2 = ap_pack(rc, rc), nas2 = ap_pack(-as, -as), magic2 = ap_pack(kRoundMagic, kRoundMagic);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        uint32_t tb[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint64_t y2 = ap_mul2(ap_pack(x[8 * v + 2 * k], x[8 * v + 2 * k + 1]), m127_2);
            const uint64_t p2 = ap_mul2(y2, rc2);
            const uint64_t t2 = ap_add2(ap_fma2(ap_fma2(nas2, p2, y2), rc2, p2), magic2);
            tb[2 * k] = (uint32_t)t2;
            tb[2 * k + 1] = (uint32_t)(t2 >> 32);
        }
        pk[v].x = __byte_perm(__byte_perm(tb[0], tb[1], 0x0040), __byte_perm(tb[2], tb[3], 0x0040), 0x5410);
        pk[v].y = __byte_perm(__byte_perm(tb[4], tb[5], 0x0040), __byte_perm(tb[6], tb[7], 0x0040), 0x5410);
    }
    constexpr float c127 = 1.f / 127.f;
    const float sq = __fmul_rn(amax, c127);
    scale = (f != 1.f) ? __fdiv_rn(amax, 127.f) : fmaf(fmaf(-127.f, sq, amax), c127, sq);
}

__device__ __forceinline__ void nr_unpack(const uint4 raw, float *x)
{
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        x[2 * k] = __uint_as_float(w[k] << 16);
        x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
    }
}

template <int kMode, bool kAppend>
__global__ void __launch_bounds__(kNrThreads, 9)
slim_norm_rope_kernel(const NormRopeParams p)
{
    extern __shared__ __align__(16) float nr_smem[];
    // cosines [span][half], sines [span][half], then (append) the tokens' sequence and cache position
    float *cos_s = nr_smem, *sin_s = nr_smem + p.span * p.half;
    int2 *where_s = reinterpret_cast<int2 *>(nr_smem + 2 * p.span * p.half);
    pdl_launch_dependents();   // an attention kernel queued behind this one may run its set-up meanwhile
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = tid / kNrLanes, l = tid % kNrLanes;
    const int R = p.rows_per_token;
    const int first = (int)blockIdx.x * kNrRows;             // (the host checks that the row count fits 32 bits)
    const int tok0 = (int)((unsigned)first / (unsigned)R);
    const int row = first + g;
    const int tok = (int)((unsigned)row / (unsigned)R);
    const int slot = row - tok * R;
    const int kind = (slot < p.Hq) ? 0 : ((slot < p.Hq + p.Hkv) ? 1 : 2);   // query, key, value
    const int head = slot - (kind == 0 ? 0 : (kind == 1 ? p.Hq : p.Hq + p.Hkv));
    const bool valid = tok < p.n_tokens;
    pdl_wait();

    // ---- the rows' loads, before anything else (plain loads: the output may be the input itself)
    uint4 raw[4], raw2[4];
    const __nv_bfloat16 *src = p.src[kind] + (long long)tok * p.src_stride[kind] + (long long)head * kHeadDim;
    const int hp = p.half / 8;   // pieces in half a rotation
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        raw[v] = raw2[v] = make_uint4(0, 0, 0, 0);
        if (valid) {
            const int piece = 4 * v + l;
            raw[v] = reinterpret_cast<const uint4 *>(src)[piece];
            if (kMode == kNrHalvesReload && kind != 2 && piece < 2 * hp)
                raw2[v] = reinterpret_cast<const uint4 *>(src)[piece < hp ? piece + hp : piece - hp];
        }
    }

    // ---- where the block's tokens go, then their angles
    if (kAppend) {
        // (by the block's last warps, while the first ones compute angles)
        for (int t = kNrThreads / 32 - 1 - warp; t < p.span; t += kNrThreads / 32) {
            int2 at = make_int2(-1, 0);
            if (tok0 + t < p.n_tokens && tok0 + t < __ldg(p.cu_new + p.B)) {   // tokens behind the last sequence go nowhere
                const int b = nr_find_sequence(p.cu_new, p.B, tok0 + t, lane);
                at = make_int2(b, __ldg(p.start_pos + b) + tok0 + t - __ldg(p.cu_new + b));
            }
            if (lane == 0) where_s[t] = at;
        }
        if (p.positions == nullptr) __syncthreads();   // (the angles wait for the positions then)
    }
    for (int i = tid; i < p.span * p.half; i += kNrThreads) {
        const int t = i / p.half, k = i - t * p.half;
        float s = 0.f, c = 1.f;
        if (tok0 + t < p.n_tokens) {
            int pos;
            if (p.positions != nullptr) {
                const int axis = (p.n_axes > 1) ? min((int)__ldg(p.axis + k), p.n_axes - 1) : 0;
                pos = __ldg(p.positions + (size_t)axis * p.n_tokens + tok0 + t);
            } else {
                pos = where_s[t].y;
            }
            // (positions are only optional with a cache; the host checks that)
            const double turns = (double)pos * (__ldg(p.inv_freq + k) * 0.15915494309189535);   // 1 / (2 pi)
            sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        }
        cos_s[i] = c;
        sin_s[i] = s;
    }
    __syncthreads();

    const int t = valid ? tok - tok0 : 0;
    const bool placed = !kAppend || (valid && where_s[t].x >= 0);
    float x[32];
#pragma unroll
    for (int v = 0; v < 4; ++v) nr_unpack(raw[v], x + 8 * v);

    // ---- norm
    const __nv_bfloat16 *weight = (kind == 2) ? nullptr : p.weight[kind];
    float norm = 1.f;
    {
        float ss = 0.f;
#pragma unroll
        for (int i = 0; i < 32; ++i) ss = fmaf(x[i], x[i], ss);
        ss += __shfl_xor_sync(0xffffffffu, ss, 1);
        ss += __shfl_xor_sync(0xffffffffu, ss, 2);
        if (weight != nullptr) norm = rsqrtf(fmaf(ss, 1.f / kHeadDim, p.eps));
    }
    if (weight != nullptr) {
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            float w[8];
            nr_unpack(__ldg(reinterpret_cast<const uint4 *>(weight) + 4 * v + l), w);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[8 * v + e] *= norm * w[e];
        }
    }

    // ---- rotation
    if (kind != 2) {
        const float *cs = cos_s + t * p.half, *sn = sin_s + t * p.half;
        if (kMode == kNrHalvesInLane) {
            // half = 64: pieces v and v + 2 of the lane; half = 32: pieces 0 and 1; half = 0: none
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const bool wide = p.half == 64;
                if (!wide && (u == 1 || p.half == 0)) break;
                const int piece = 4 * u + l;
#pragma unroll
                for (int e4 = 0; e4 < 2; ++e4) {
                    const float4 c4 = *reinterpret_cast<const float4 *>(cs + 8 * piece + 4 * e4);
                    const float4 s4 = *reinterpret_cast<const float4 *>(sn + 8 * piece + 4 * e4);
                    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 8 * u + 4 * e4 + e;
                        const float a = x[i], b = wide ? x[16 + i] : x[8 + i % 8];
                        const float ya = a * c[e] - b * s[e], yb = fmaf(a, s[e], b * c[e]);
                        x[i] = ya;
                        if (wide) x[16 + i] = yb; else x[8 + i % 8] = yb;
                    }
                }
            }
        } else if (kMode == kNrAdjacent) {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int piece = 4 * v + l;
                if (4 * piece < p.half) {
                    const float4 c4 = *reinterpret_cast<const float4 *>(cs + 4 * piece), s4 = *reinterpret_cast<const float4 *>(sn + 4 * piece);
                    const float c[4] = {c4.x, c4.y, c4.z, c4.w}, s[4] = {s4.x, s4.y, s4.z, s4.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float a = x[8 * v + 2 * e], b = x[8 * v + 2 * e + 1];
                        x[8 * v + 2 * e] = a * c[e] - b * s[e];
                        x[8 * v + 2 * e + 1] = fmaf(a, s[e], b * c[e]);
                    }
                }
            }
        } else {
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int piece = 4 * v + l;
                if (piece < 2 * hp) {
                    const bool low = piece < hp;
                    const int other = low ? piece + hp : piece - hp, i0 = 8 * (low ? piece : other);
                    float o[8];
                    nr_unpack(raw2[v], o);
                    if (weight != nullptr) {
                        float w[8];
                        nr_unpack(__ldg(reinterpret_cast<const uint4 *>(weight) + other), w);
#pragma unroll
                        for (int e = 0; e < 8; ++e) o[e] *= norm * w[e];
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float c = cs[i0 + e], s = low ? -sn[i0 + e] : sn[i0 + e];
                        x[8 * v + e] = fmaf(o[e], s, x[8 * v + e] * c);
                    }
                }
            }
        }
    }

    // ---- results
    uint2 pk[4];
    float scale;
    if (kAppend) nr_quantize(x, pk, scale);   // (all lanes together; query rows do not use it)
    __syncwarp();                             // every lane of the row has read its input: the output may be the same memory
    if (!valid) return;
    if (kind == 0 || !kAppend) {
        const int heads = (kind == 0) ? p.Hq : p.Hkv;
        uint4 *dst = reinterpret_cast<uint4 *>(p.dst[kind == 0 ? 0 : 1] + ((size_t)tok * heads + head) * kHeadDim);
        if (!placed) return;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            uint32_t o[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                __nv_bfloat162 y = __floats2bfloat162_rn(x[8 * v + 2 * k], x[8 * v + 2 * k + 1]);
                o[k] = *reinterpret_cast<uint32_t *>(&y);
            }
            dst[4 * v + l] = make_uint4(o[0], o[1], o[2], o[3]);
        }
    } else if (placed) {
        const int2 at = where_s[t];
        const int page_idx = at.y >> 7;
        if (at.y < 0 || page_idx >= p.max_pages_per_seq) return;
        const int page = __ldg(p.block_table + (size_t)at.x * p.max_pages_per_seq + page_idx);
        if (page < 0 || page >= p.num_pages) return;
        const int kv = kind - 1, in_page = at.y & (kPageTokens - 1);
        uint2 *dst = reinterpret_cast<uint2 *>(p.codes + code_block_offset(page, head, kv, p.Hkv) + (size_t)in_page * kHeadDim);
#pragma unroll
        for (int v = 0; v < 4; ++v) dst[4 * v + l] = pk[v];
        if (l == 0) p.scales[scale_block_offset(page, head, kv, p.Hkv) + in_page] = scale;
    }
}

template <bool kAppend>
static int launch_mode(const NormRopeParams &p, bool interleaved, cudaStream_t stream)
{
    const long long rows = (long long)p.n_tokens * p.rows_per_token;
    const unsigned blocks = (unsigned)((rows + kNrRows - 1) / kNrRows);
    const size_t smem = (size_t)p.span * (2 * p.half * sizeof(float) + sizeof(int2));   // 17 KB at most (one row per token)
    if (interleaved)
        SLIM_CUDA_TRY(launch_pdl(slim_norm_rope_kernel<kNrAdjacent, kAppend>, dim3(blocks), dim3(kNrThreads), smem, stream, p));
    else if (p.half % 32 == 0)
        SLIM_CUDA_TRY(launch_pdl(slim_norm_rope_kernel<kNrHalvesInLane, kAppend>, dim3(blocks), dim3(kNrThreads), smem, stream, p));
    else
        SLIM_CUDA_TRY(launch_pdl(slim_norm_rope_kernel<kNrHalvesReload, kAppend>, dim3(blocks), dim3(kNrThreads), smem, stream, p));
    return SLIM_OK;
}

// Arguments have been checked (slim_abi.cu).  cache null: queries and keys to q_out and k_out.
int launch_norm_rope(const slim_cache_t *c, const slim_norm_rope_t *nr, const void *q, int64_t q_stride, void *q_out, const void *k,
                     int64_t k_stride, void *k_out, const void *v, int64_t v_stride, const int32_t *positions, const int32_t *cu_new,
                     const int32_t *start_pos, int B, int n_tokens, int Hq, int Hkv, cudaStream_t stream)
{
    // (the kernel indexes rows with 32-bit integers)
    const long long per_token = Hq + (c != nullptr ? 2LL : 1LL) * Hkv;
    if (per_token > 0x7FFFFF00LL / n_tokens) return SLIM_ERR_UNSUPPORTED;
    NormRopeParams p = {};
    p.src[0] = static_cast<const __nv_bfloat16 *>(q);
    p.src[1] = static_cast<const __nv_bfloat16 *>(k);
    p.src[2] = static_cast<const __nv_bfloat16 *>(v);
    p.src_stride[0] = q_stride, p.src_stride[1] = k_stride, p.src_stride[2] = v_stride;
    p.dst[0] = static_cast<__nv_bfloat16 *>(q_out);
    p.dst[1] = static_cast<__nv_bfloat16 *>(k_out);
    p.weight[0] = static_cast<const __nv_bfloat16 *>(nr->q_weight);
    p.weight[1] = static_cast<const __nv_bfloat16 *>(nr->k_weight);
    p.inv_freq = nr->inv_freq;
    p.axis = nr->axis;
    p.positions = positions;
    p.n_tokens = n_tokens;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.half = nr->rotary_dim / 2;
    p.n_axes = nr->n_axes;
    p.eps = nr->eps;
    p.rows_per_token = (int)per_token;
    p.span = (kNrRows - 1 + p.rows_per_token - 1) / p.rows_per_token + 1;   // tokens that a block's consecutive rows touch at most
    if (c == nullptr) return launch_mode<false>(p, nr->interleaved != 0, stream);
    p.codes = c->codes;
    p.scales = c->scales;
    p.block_table = c->block_table;
    p.max_pages_per_seq = c->max_pages_per_seq;
    p.num_pages = c->num_pages;
    p.cu_new = cu_new;
    p.start_pos = start_pos;
    p.B = B;
    return launch_mode<true>(p, nr->interleaved != 0, stream);
}

}  // namespace slim

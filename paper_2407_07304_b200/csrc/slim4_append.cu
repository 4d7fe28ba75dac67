// Quantise-and-append into the 4-bit cache, and the way back to bf16 rows.
//
// Both kernels are bound by memory traffic (256 bytes of bf16 and 68 of codes, scale and offset per row).  Four lanes own
// a row: lane l holds the eight-dim pieces l, 4 + l, 8 + l and 12 + l, so that the two dims that share a byte (i and
// 64 + i) lie in one lane and a row's loads and stores stay contiguous across its lanes.
//
// Measured (16 ragged prompts of 256 to 4096 tokens, 8 kv heads, 291,000 rows each of K and V, 189 MB a call): append 36.2 us =
// 5.2 TB/s (68 % of the issue slots; constants held as packed pairs and the rows of extreme scales apart took it from 39.3),
// read-back 35.2 us = 5.4 TB/s, 79 and 82 % of the copy rate.  Blocks of 128 threads: 35.3 and
// 35.2 us, within the spread of such runs; of 512, with an earlier form of the append that took 40.2: 44.6 and 37.1.
#include "slim4_common.cuh"

namespace slim {

constexpr int kAp4Threads = 256;
constexpr int kAp4Rows = kAp4Threads / 4;   // rows of a block: row = token * Hkv + head within the sequence's new rows

// Where row r of sequence b lies: false outside the page table or the pool.
struct Row4 {
    size_t code, pair;   // byte offset of the codes, index of the (scale, offset) word
};
__device__ __forceinline__ bool row4_find(const int32_t *block_table, int b, int pos, int head, int kv, int Hkv, int max_pages_per_seq,
                                          int num_pages, Row4 &at)
{
    const int page_idx = pos >> 7;
    if (pos < 0 || page_idx >= max_pages_per_seq) return false;
    const int page = __ldg(block_table + (size_t)b * max_pages_per_seq + page_idx);
    if (page < 0 || page >= num_pages) return false;
    const int slot = pos & (kPageTokens - 1);
    at.code = code4_block_offset(page, head, kv, Hkv) + (size_t)slot * kRow4Bytes;
    at.pair = scale_block_offset(page, head, kv, Hkv) + slot;
    return true;
}

// grid = (blocks of rows, B, 2 [K, V]).  The first new token of sequence b goes to position start_pos[b], or, without
// start_pos, to len_after[b] minus the sequence's new tokens.
__global__ void __launch_bounds__(kAp4Threads)
slim4_append_kernel(uint8_t *__restrict__ codes, uint32_t *__restrict__ pairs, const int32_t *__restrict__ block_table,
                    const __nv_bfloat16 *__restrict__ k_new, const __nv_bfloat16 *__restrict__ v_new,
                    const int32_t *__restrict__ cu_new, const int32_t *__restrict__ start_pos, const int32_t *__restrict__ len_after,
                    int Hkv, int max_pages_per_seq, int num_pages)
{
    pdl_launch_dependents();   // an attention kernel queued behind this one may run its set-up meanwhile
    const int b = blockIdx.y, kv = blockIdx.z, l = threadIdx.x & 3;
    const int row0 = __ldg(cu_new + b), n_tok = __ldg(cu_new + b + 1) - row0;
    const long long n_rows = (long long)n_tok * Hkv;
    const long long r = (long long)blockIdx.x * kAp4Rows + (threadIdx.x >> 2);
    if ((long long)blockIdx.x * kAp4Rows >= n_rows) return;
    const bool real = r < n_rows;
    uint4 raw[4];
#pragma unroll
    for (int v = 0; v < 4; ++v) raw[v] = make_uint4(0, 0, 0, 0);
    Row4 at;
    bool stored = false;
    if (real) {
        const uint4 *src = reinterpret_cast<const uint4 *>((kv ? v_new : k_new) + ((size_t)row0 * Hkv + (size_t)r) * kHeadDim);
#pragma unroll
        for (int v = 0; v < 4; ++v) raw[v] = __ldg(src + v * 4 + l);
        const int tok = (int)((unsigned)r / (unsigned)Hkv), head = (int)r - tok * Hkv;   // (the host checks that the rows fit 32 bits)
        const int start = (start_pos != nullptr) ? __ldg(start_pos + b) : __ldg(len_after + b) - n_tok;
        stored = row4_find(block_table, b, start + tok, head, kv, Hkv, max_pages_per_seq, num_pages, at);
    }
    // smallest and largest value on the packed pairs, then across the row's lanes
    uint32_t lo2 = raw[0].x, hi2 = raw[0].x;
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        lo2 = q4_min_bf16x2(lo2, q4_min_bf16x2(q4_min_bf16x2(raw[v].x, raw[v].y), q4_min_bf16x2(raw[v].z, raw[v].w)));
        hi2 = q4_max_bf16x2(hi2, q4_max_bf16x2(q4_max_bf16x2(raw[v].x, raw[v].y), q4_max_bf16x2(raw[v].z, raw[v].w)));
    }
#pragma unroll
    for (int o = 1; o <= 2; o <<= 1) {
        lo2 = q4_min_bf16x2(lo2, __shfl_xor_sync(0xffffffffu, lo2, o));
        hi2 = q4_max_bf16x2(hi2, __shfl_xor_sync(0xffffffffu, hi2, o));
    }
    const uint32_t pair = q4_pair(q4_min_of(lo2), q4_max_of(hi2));
    const Q4Row q(pair);
    if (!stored) return;
    // dims 8 (4 v + l) .. + 7 low, 64 further high, v = 0, 1
    const uint32_t low[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
    const uint32_t high[8] = {raw[2].x, raw[2].y, raw[2].z, raw[2].w, raw[3].x, raw[3].y, raw[3].z, raw[3].w};
    uint32_t w[4];
    q.words<4>(low, high, w);
    reinterpret_cast<uint2 *>(codes + at.code)[l] = make_uint2(w[0], w[1]);
    reinterpret_cast<uint2 *>(codes + at.code)[4 + l] = make_uint2(w[2], w[3]);
    if (l == 0) pairs[at.pair] = pair;
}

// Four values z + u s (u in the bytes of w) as bf16 pairs.
__device__ __forceinline__ uint2 row4_values(uint32_t w, float s, float z)
{
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __fadd_rn(__fmul_rn((float)((w >> (8 * i)) & 0xFu), s), z);
    const __nv_bfloat162 a = __floats2bfloat162_rn(x[0], x[1]), b = __floats2bfloat162_rn(x[2], x[3]);
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

__global__ void __launch_bounds__(kAp4Threads)
slim4_read_kernel(const uint8_t *__restrict__ codes, const uint32_t *__restrict__ pairs, const int32_t *__restrict__ block_table,
                  __nv_bfloat16 *__restrict__ k_out, __nv_bfloat16 *__restrict__ v_out, const int32_t *__restrict__ cu,
                  const int32_t *__restrict__ start_pos, int Hkv, int max_pages_per_seq, int num_pages)
{
    const int b = blockIdx.y, kv = blockIdx.z, l = threadIdx.x & 3;
    pdl_wait();
    const int row0 = __ldg(cu + b);
    const long long n_rows = (long long)(__ldg(cu + b + 1) - row0) * Hkv;
    const long long r = (long long)blockIdx.x * kAp4Rows + (threadIdx.x >> 2);
    if (r >= n_rows) return;
    const int tok = (int)((unsigned)r / (unsigned)Hkv), head = (int)r - tok * Hkv;
    Row4 at;
    if (!row4_find(block_table, b, __ldg(start_pos + b) + tok, head, kv, Hkv, max_pages_per_seq, num_pages, at)) return;
    uint2 w[2];
#pragma unroll
    for (int v = 0; v < 2; ++v) w[v] = reinterpret_cast<const uint2 *>(codes + at.code)[v * 4 + l];
    const uint32_t pair = pairs[at.pair];
    const float s = pair_scale(pair), z = pair_offset(pair);
    uint4 *dst = reinterpret_cast<uint4 *>((kv ? v_out : k_out) + ((size_t)row0 * Hkv + (size_t)r) * kHeadDim);
#pragma unroll
    for (int v = 0; v < 4; ++v) {
        const uint2 a = row4_values((w[v & 1].x >> (v < 2 ? 0 : 4)) & 0x0F0F0F0Fu, s, z);
        const uint2 c = row4_values((w[v & 1].y >> (v < 2 ? 0 : 4)) & 0x0F0F0F0Fu, s, z);
        dst[v * 4 + l] = make_uint4(a.x, a.y, c.x, c.y);
    }
}

int launch_append4(const slim_cache4_t *c, const void *k_new, const void *v_new, const int32_t *cu_new, const int32_t *start_pos,
                   int B, int max_new, cudaStream_t stream, const int32_t *len_after)
{
    const long long rows = (long long)max_new * c->num_kv_heads;
    if (rows > 0x7FFFFF00LL) return SLIM_ERR_UNSUPPORTED;   // the kernel divides rows in 32 bits
    dim3 grid((unsigned)((rows + kAp4Rows - 1) / kAp4Rows), (unsigned)B, 2);
    slim4_append_kernel<<<grid, kAp4Threads, 0, stream>>>(
        c->codes, reinterpret_cast<uint32_t *>(c->scales), c->block_table, static_cast<const __nv_bfloat16 *>(k_new),
        static_cast<const __nv_bfloat16 *>(v_new), cu_new, start_pos, len_after, c->num_kv_heads, c->max_pages_per_seq, c->num_pages);
    SLIM_CUDA_TRY(cudaGetLastError());
    return SLIM_OK;
}

int launch_read4(const slim_cache4_t *c, void *k_out, void *v_out, const int32_t *cu, const int32_t *start_pos, int B, int max_rows,
                 cudaStream_t stream)
{
    const long long rows = (long long)max_rows * c->num_kv_heads;
    if (rows > 0x7FFFFF00LL) return SLIM_ERR_UNSUPPORTED;
    dim3 grid((unsigned)((rows + kAp4Rows - 1) / kAp4Rows), (unsigned)B, 2);
    SLIM_CUDA_TRY(launch_pdl(slim4_read_kernel, grid, dim3(kAp4Threads), 0, stream, c->codes, reinterpret_cast<const uint32_t *>(c->scales),
                             c->block_table, static_cast<__nv_bfloat16 *>(k_out), static_cast<__nv_bfloat16 *>(v_out), cu, start_pos,
                             c->num_kv_heads, c->max_pages_per_seq, c->num_pages));
    return SLIM_OK;
}

}  // namespace slim

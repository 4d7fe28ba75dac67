// The log-sum-exp merge of a row's partials by one warp, and what the merge kernels share.
#pragma once
#include "slim_common.cuh"
#include "slim_decode_params.cuh"

namespace slim {

constexpr int kChunkTok = 256;   // tokens per partial result (two pages)

// Partials of a row of `len` cached tokens (never more than cap_tokens): one per 256-token chunk of the
// tokens before the last one, then the last token's own.
__device__ __forceinline__ int merge_row_partials(int len, int cap_tokens)
{
    const int L = min(max(len, 0), cap_tokens);
    return (L == 0) ? 0 : (L - 1 + kChunkTok - 1) / kChunkTok + 1;
}

// How many partials the merge kernels find for a sequence.  (They are passed by value with every launch: the plain form
// stays as small as it can be.)
struct PlainRows {
    const int32_t *kv_len;
    int cap_tokens;
    __device__ __forceinline__ void done(bool) const {}
    __device__ __forceinline__ int length(int b) const { return __ldg(kv_len + b); }
    __device__ __forceinline__ int partials(int b, int len) const { return merge_row_partials(len, cap_tokens); }
};

// Behind a shared prefix: the prefix's slots (every one of them is filled, those without a key with weight 0), then the
// tail's partials; cap_tokens bounds the tail.
struct SharedRows {
    const int32_t *kv_len, *shared_len;
    int *begun;
    int slot0, max_pages, max_shared_pages, cap_tokens;
    // (both kernels before this one have ended: the workspace's header goes back to zero)
    __device__ __forceinline__ void done(bool one_thread) const
    {
        if (one_thread) *begun = 0;
    }
    __device__ __forceinline__ int length(int b) const { return __ldg(kv_len + b); }
    __device__ __forceinline__ int partials(int b, int len) const
    {
        const int start = shared_tokens(shared_len, max_shared_pages, b);
        const int tail = merge_row_partials(len - start, min(max_pages * kPageTokens - start, cap_tokens));
        return (tail == 0 && min(len, start) <= 0) ? 0 : slot0 + tail;
    }
};

// Tokens that a launch attends over at most (behind the prefix, where there is one).
inline int merge_cap_tokens(const DecodeParams &p)
{
    const long long pages = (long long)p.max_pages_per_seq * kPageTokens, chunks = (long long)p.n_chunks * kChunkTok;
    return (int)(pages < chunks ? pages : chunks);
}

// A row's merged partial (what slim_attn_decode_partial returns): O relative to M, then M and l; a lane owns four dims.
__device__ __forceinline__ void store_raw_partial(float *raw, int row, int lane, float4 o, float M, float l)
{
    float *dst = raw + (size_t)row * SLIM_PARTIAL_FLOATS;
    reinterpret_cast<float4 *>(dst)[lane] = o;
    if (lane == 0) *reinterpret_cast<float2 *>(dst + kHeadDim) = make_float2(M, l);
}

// The same merge for rows of fewer than 32 chunks: one warp per (sequence, query head) row, a lane owns four head
// dims, lane c owns chunk c's (m, l).  Once the row's length has arrived, the (m, l) pairs and the first sixteen
// partial outputs of the row are requested together, so a row costs two round trips to memory instead of one per
// step of the reduction.  (Asking for the sixteen slots before the length is known, as the block-per-row kernel below
// does, read half as much again on ragged batches and was 0.5 us slower on the 64 / 8-head workload.)
constexpr int kMergeWarpBatch = 16;
__device__ __forceinline__ void merge_row_by_warp(const float *part_o, const float *part_ml, int nc, __nv_bfloat16 *out,
                                                  float *raw, int row, int n_slots, int lane)
{
    const float2 *ml = reinterpret_cast<const float2 *>(part_ml) + (size_t)row * n_slots;
    const float4 *po = reinterpret_cast<const float4 *>(part_o + (size_t)row * n_slots * kHeadDim) + lane;
    float4 o[kMergeWarpBatch];
#pragma unroll
    for (int u = 0; u < kMergeWarpBatch; ++u)
        o[u] = (u < nc) ? __ldcg(po + (size_t)u * (kHeadDim / 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
    float2 v = (lane < nc) ? __ldcg(ml + lane) : make_float2(-INFINITY, 0.f);
    if (lane >= nc) v = make_float2(-INFINITY, 0.f);
    const float M = warp_max(v.x);
    const float w = (v.x != -INFINITY) ? exp2f(v.x - M) : 0.f;   // (slots without keys: weight 0, also where no slot has any)
    const float l = warp_sum(v.y * w);
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int c0 = 0; c0 < nc; c0 += kMergeWarpBatch) {
        if (c0 > 0) {
#pragma unroll
            for (int u = 0; u < kMergeWarpBatch; ++u)
                o[u] = (c0 + u < nc) ? __ldcg(po + (size_t)(c0 + u) * (kHeadDim / 4)) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int u = 0; u < kMergeWarpBatch; ++u) {
            const float wj = __shfl_sync(0xffffffffu, w, (c0 + u) & 31);
            if (c0 + u < nc) {
                acc.x = fmaf(o[u].x, wj, acc.x);
                acc.y = fmaf(o[u].y, wj, acc.y);
                acc.z = fmaf(o[u].z, wj, acc.z);
                acc.w = fmaf(o[u].w, wj, acc.w);
            }
        }
    }
    if (raw != nullptr) {
        store_raw_partial(raw, row, lane, nc > 0 ? acc : make_float4(0.f, 0.f, 0.f, 0.f), nc > 0 ? M : -INFINITY, nc > 0 ? l : 0.f);
        return;
    }
    const float inv = (nc > 0 && l > 0.f) ? 1.f / l : 0.f;
    __nv_bfloat162 lo = __floats2bfloat162_rn(acc.x * inv, acc.y * inv), hi = __floats2bfloat162_rn(acc.z * inv, acc.w * inv);
    uint2 packed;
    packed.x = *reinterpret_cast<uint32_t *>(&lo);
    packed.y = *reinterpret_cast<uint32_t *>(&hi);
    *reinterpret_cast<uint2 *>(out + (size_t)row * kHeadDim + lane * 4) = packed;
}

}  // namespace slim

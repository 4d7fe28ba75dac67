// Parameters shared by the decode split kernels and the merge kernel.
#pragma once
#include "slim_common.cuh"

namespace slim {

// The plain split pass.  (It is passed by value with every launch: 32 bytes more of it cost a decode step 0.5 us.)
struct SplitParams {
    const int8_t *codes;
    const float *scales;
    const int32_t *block_table;
    const int32_t *kv_len;
    const __nv_bfloat16 *q;   // [B][Hq][128]
    int *status;              // first word of the workspace: set to a SLIM_ERR_* code by a kernel whose wait ran out
    float *part_o;            // [B][Hq][n_slots][128] unnormalised partial outputs: a row's chunks, then its last token
    float *part_ml;           // [B][Hq][n_slots][2]   (max in log2 units, sum)
    // one-kernel append + split (optional): the new token of every sequence, [B][Hkv][128], quantised into slot
    // kv_len - 1 by the warp that attends the sequence's last token (null: nothing to append)
    const __nv_bfloat16 *k_new, *v_new;
    // merge at the end of the split kernel (optional, both or neither): the result [B][Hq][128] and the counters
    // [B * Hkv] of chunks counted so far per (sequence, kv head); zero before and after every launch
    __nv_bfloat16 *out;
    int *counters;
    int Hq, Hkv, G;
    int max_pages_per_seq, num_pages;
    int n_chunks;             // 256-token chunks that max_kv tokens need
    int n_slots;              // partial slots per row: n_chunks + 1 (the last token of a row has a partial of its own)
    float scale_log2e;        // sm_scale * log2(e)
};

// What the other forms of the pass take beside it.
struct DecodeParams : SplitParams {
    // kept for the attention weights (optional): [B][Hq][share_stride], position by position a token's share of the
    // denominator l of its partial, 2^(s - m)
    float *shares;
    int share_stride;
    // tokens behind a shared prefix (optional): the prefix's length per sequence, and the partial slots in front of
    // the tail's that the prefix kernel fills
    const int32_t *shared_len;
    int max_shared_pages;   // the launch's bound on the prefix, never beyond the page table
    int *begun;             // in the workspace's header: raised once everything before the prefix kernel is visible, lowered by the merge
    int slot0;
    int max_blocks;   // of the split pass (0: one per SM)
};

// The length of the prefix that sequence b shares: whole pages, never more than the launch was made for (what is shared
// beyond that counts as the sequence's own).
__device__ __forceinline__ int shared_tokens(const int32_t *shared_len, int max_shared_pages, int b)
{
    return min(max(__ldg(shared_len + b), 0) / kPageTokens, max_shared_pages) * kPageTokens;
}
__device__ __forceinline__ int decode_shared_tokens(const DecodeParams &p, int b)
{
    return shared_tokens(p.shared_len, p.max_shared_pages, b);
}

// Workspace header in front of the partials: the status word (16 bytes; the second int of them is the shared decode's
// flag), then the counters of the in-kernel merge.  The header has one size for every shape, so a workspace zeroed once
// stays valid when the shapes of the calls that use it change.
constexpr size_t kDecodeStatusBytes = 16;
constexpr int kDecodeCounterRows = 16384;   // (sequence, kv head) pairs the in-kernel merge can count
constexpr size_t kDecodeHeaderBytes = kDecodeStatusBytes + (size_t)kDecodeCounterRows * sizeof(int);

// Parameters of a split pass over `workspace` (slim_decode.cu); what is optional is left out.
DecodeParams make_decode_params(const slim_cache_t *c, const void *q, const int32_t *kv_len, int B, int max_kv, int Hq,
                                float sm_scale, void *workspace);
size_t decode_workspace_bytes(int B, int Hq, int Hkv, int max_kv);
int launch_decode_split_stream(const slim_cache_t *c, const DecodeParams &p, int B, cudaStream_t stream);
// Whether the split kernel merges its own partials (few per pair); p.out and p.counters are set then.
bool merge_in_split_kernel(DecodeParams &p, int B, void *out);
int launch_decode(const slim_cache_t *c, const void *q, const void *k_new, const void *v_new, void *out, const int32_t *kv_len, int B,
                  int max_kv, int Hq, float sm_scale, void *workspace, cudaStream_t stream);
// The merge kernel: out (bf16 rows) or, where raw is given, the rows' merged partials.
int launch_merge_rows(const DecodeParams &p, int B, void *out, float *raw, cudaStream_t stream);

}  // namespace slim

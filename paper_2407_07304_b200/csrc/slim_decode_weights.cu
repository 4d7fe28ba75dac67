// Decode attention that also accumulates every cached token's attention weight (what an eviction by weight needs).
//
//   p_h[j]   = softmax_j(sm_scale q_h . k^_j)                       query head h of sequence b
//   W'[g][j] = decay * W[g][j] + sum over the query heads h of kv head g of p_h[j]
//
// A token's weight needs the row's final maximum M and denominator l, which are known only once every chunk of the row
// has been attended, and the scores of a long row do not fit on chip.  The split pass (slim_decode_stream.cu) therefore
// leaves, beside each chunk's (m_c, l_c, O_c), every token's share of l_c, e_j = 2^(s_j - m_c): 4 bytes per query head
// and token beside the 264 bytes of cache that it reads per kv head and token.  The kernel below reads them back, mostly
// out of the L2, and p_j = e_j * 2^(m_c - M) / l: one factor per chunk and query head, no exponential per token, no
// second pass over the keys.  Shares, factors and weights are fp32.
// The same launch merges the rows' outputs where the split kernel has not done it (blocks behind the weights' blocks).
#include "slim_common.cuh"
#include "slim_decode_params.cuh"
#include "slim_merge.cuh"

namespace slim {

constexpr int kDwThreads = 256;
constexpr int kDwChunks = 4;                                  // chunks per block: a thread has one token of each
constexpr int kDwBlockTokens = kDwChunks * kChunkTok;
constexpr int kDwMaxGroup = 16;                               // query heads per kv head
constexpr int kDwBatch = 8;                                   // query heads whose shares are requested together
static_assert(kDwThreads == kChunkTok, "thread = position in the chunk");

// grid = (token blocks [+ 1: merge], kv heads, sequences)
__global__ void __launch_bounds__(kDwThreads, 3)
slim_decode_weights_kernel(const DecodeParams p, const PlainRows rows, const float *w_in, float *w_out, int w_stride, const int32_t *weighed,
                           float decay, int max_kv, int token_blocks, __nv_bfloat16 *out)
{
    __shared__ float factor[kDwMaxGroup][kDwChunks + 1];      // per query head: the block's chunks, then the row's last token
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.z, head = blockIdx.y;
    const int row0 = b * p.Hq + head * p.G;
    pdl_launch_dependents();
    pdl_wait();
    if ((int)blockIdx.x == token_blocks) {
        for (int h = warp; h < p.G; h += kDwThreads / 32) merge_row_by_warp(p.part_o, p.part_ml, rows.partials(b, rows.length(b)), out, nullptr, row0 + h, p.n_slots, lane);
        return;
    }
    const int len = min(max(__ldg(p.kv_len + b), 0), rows.cap_tokens);
    // The attention takes whole chunks (a length beyond max_kv is cut at the end of max_kv's last chunk), but a row of weights
    // has room for max_kv of them.
    const int w_len = min(len, max_kv);
    const int first = (int)blockIdx.x * kDwBlockTokens;
    if (first >= w_len) return;
    // ---- requested before anything is waited for: the first query heads' shares and the old weights
    const float *src = p.shares + (size_t)row0 * p.share_stride + first + tid;   // (a row's shares reach to the end of its last chunk)
    const int old_len = (w_in == nullptr) ? 0 : (weighed != nullptr) ? __ldg(weighed + b) : len - 1;
    const size_t w_row = ((size_t)b * p.Hkv + head) * w_stride + first + tid;
    float sum[kDwChunks], old[kDwChunks], e[kDwBatch][kDwChunks];
#pragma unroll
    for (int i = 0; i < kDwChunks; ++i) {
        const int j = first + tid + i * kChunkTok;
        old[i] = (j < w_len && j < old_len) ? w_in[w_row + i * kChunkTok] : 0.f;
        sum[i] = 0.f;
    }
    auto fetch = [&](int h0) {
#pragma unroll
        for (int h = 0; h < kDwBatch; ++h) {
#pragma unroll
            for (int i = 0; i < kDwChunks; ++i)
                e[h][i] = (h0 + h < p.G && first + tid + i * kChunkTok < len) ? __ldcg(src + (size_t)(h0 + h) * p.share_stride + i * kChunkTok) : 0.f;
        }
    };
    if (len > 1) fetch(0);
    // ---- every query head's factors, one warp per head, from the split pass's partials: the chunks, then the last token
    //      (a sequence of one token has weight 1 and, where the split kernel merges, no partial)
    const int last = len > 1 ? (len - 1 + kChunkTok - 1) / kChunkTok : 0;   // the last token's partial
    if (len > 1) {
        for (int h = warp; h < p.G; h += kDwThreads / 32) {
            const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml) + (size_t)(row0 + h) * p.n_slots;
            const int mine = (lane < kDwChunks) ? min(first / kChunkTok + lane, last) : last;
            const float m_mine = (lane <= kDwChunks) ? __ldcg(ml + mine).x : 0.f;
            float2 v = (lane <= last) ? __ldcg(ml + lane) : make_float2(-INFINITY, 0.f);
            float M = v.x;
            for (int c = lane + 32; c <= last; c += 32) M = fmaxf(M, __ldcg(ml + c).x);
            M = warp_max(M);
            float l = v.y * exp2f(v.x - M);
            for (int c = lane + 32; c <= last; c += 32) {
                v = __ldcg(ml + c);
                l = fmaf(v.y, exp2f(v.x - M), l);
            }
            l = warp_sum(l);
            if (lane <= kDwChunks) factor[h][lane] = exp2f(m_mine - M) / l;
        }
    }
    __syncthreads();
    if (len > 1) {
        for (int h0 = 0; h0 < p.G; h0 += kDwBatch) {
            if (h0 > 0) fetch(h0);
#pragma unroll
            for (int h = 0; h < kDwBatch; ++h) {
                if (h0 + h < p.G) {
#pragma unroll
                    for (int i = 0; i < kDwChunks; ++i)
                        sum[i] = fmaf(e[h][i], factor[h0 + h][first + tid + i * kChunkTok == len - 1 ? kDwChunks : i], sum[i]);
                }
            }
        }
    } else {
        sum[0] = (float)p.G;
    }
#pragma unroll
    for (int i = 0; i < kDwChunks; ++i)
        if (first + tid + i * kChunkTok < w_len) w_out[w_row + i * kChunkTok] = fmaf(decay, old[i], sum[i]);
}

// The shares follow the split pass's workspace.
static size_t shares_offset(int B, int Hq, int Hkv, int max_kv)
{
    return (decode_workspace_bytes(B, Hq, Hkv, max_kv) + 255) / 256 * 256;
}

size_t weights_workspace_bytes(int B, int Hq, int Hkv, int max_kv)
{
    const size_t stride = (size_t)(max_kv + kChunkTok - 1) / kChunkTok * kChunkTok;
    return shares_offset(B, Hq, Hkv, max_kv) + (size_t)B * Hq * stride * sizeof(float);
}

int launch_decode_weights(const slim_cache_t *c, const void *q, const void *k_new, const void *v_new, void *out, const float *w_in,
                          float *w_out, int w_stride, const int32_t *weighed, const int32_t *kv_len, int B, int max_kv, int Hq,
                          float sm_scale, float decay, void *workspace, cudaStream_t stream)
{
    DecodeParams p = make_decode_params(c, q, kv_len, B, max_kv, Hq, sm_scale, workspace);
    if (p.n_chunks == 0) return launch_merge_rows(p, B, out, nullptr, stream);   // rows of zeros
    p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = static_cast<const __nv_bfloat16 *>(v_new);
    p.shares = reinterpret_cast<float *>(static_cast<char *>(workspace) + shares_offset(B, Hq, c->num_kv_heads, max_kv));
    p.share_stride = p.n_chunks * kChunkTok;
    const bool merged = merge_in_split_kernel(p, B, out);
    int rc = launch_decode_split_stream(c, p, B, stream);
    if (rc != SLIM_OK) return rc;
    // rows of up to 31 partials are merged by the weights' launch, longer ones by the kernels made for them
    const bool merge_here = !merged && p.n_slots < 32;
    if (!merged && !merge_here) {
        rc = launch_merge_rows(p, B, out, nullptr, stream);
        if (rc != SLIM_OK) return rc;
    }
    const int token_blocks = (max_kv + kDwBlockTokens - 1) / kDwBlockTokens;
    const dim3 grid((unsigned)(token_blocks + (merge_here ? 1 : 0)), (unsigned)p.Hkv, (unsigned)B);
    SLIM_CUDA_TRY(launch_pdl(slim_decode_weights_kernel, grid, dim3(kDwThreads), 0, stream, p, PlainRows{kv_len, merge_cap_tokens(p)}, w_in, w_out, w_stride, weighed, decay,
                             max_kv, token_blocks, static_cast<__nv_bfloat16 *>(out)));
    return SLIM_OK;
}

}  // namespace slim

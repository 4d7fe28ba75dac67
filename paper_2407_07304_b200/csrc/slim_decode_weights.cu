// Decode attention that also accumulates every cached token's attention weight (what an eviction by weight needs).
//
//   p_h[j]   = softmax_j(sm_scale q_h . k^_j)                       query head h of sequence b
//   W'[g][j] = decay * W[g][j] + sum over the query heads h of kv head g of p_h[j]
//
// A token's weight needs the row's final maximum and denominator, which are known only once every chunk of the row has
// been attended, and the scores of a long row do not fit on chip.  The split pass (slim_decode_stream.cu) therefore
// writes each score it forms, 4 bytes per query head and token beside the 264 bytes of cache that it reads per kv head
// and token, and the kernel below reads them back, mostly out of the L2: no second pass over the keys.
// Scores, maxima, denominators and weights are fp32 throughout.
#include "slim_common.cuh"
#include "slim_decode_params.cuh"

namespace slim {

constexpr int kDwThreads = 256;
constexpr int kDwTokens = 4;                                  // tokens per thread, 256 apart
constexpr int kDwBlockTokens = kDwThreads * kDwTokens;
constexpr int kDwMaxGroup = 16;                               // query heads per kv head
constexpr int kDwChunk = 256;                                 // tokens per partial of the split pass

// grid = (token blocks, kv heads, sequences).  Every block finds the maxima and denominators of its kv head's query
// rows itself from the split pass's partials (one warp per row).
__global__ void __launch_bounds__(kDwThreads)
slim_decode_weights_kernel(const DecodeParams p, const float *w_in, float *w_out, int w_stride, const int32_t *weighed, float decay)
{
    __shared__ float max_s[kDwMaxGroup], inv_s[kDwMaxGroup];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.z, head = blockIdx.y;
    pdl_wait();
    const int len = min(max(__ldg(p.kv_len + b), 0), min(p.max_pages_per_seq * kPageTokens, p.n_chunks * kDwChunk));
    const int first = (int)blockIdx.x * kDwBlockTokens;
    if (first >= len) return;
    const size_t row0 = (size_t)b * p.Hq + (size_t)head * p.G;
    // ---- the rows' maxima and denominators (a sequence of one token has weight 1 and, where the split kernel merges,
    //      no partial)
    if (len > 1) {
        const int nc = (len - 1 + kDwChunk - 1) / kDwChunk + 1;
        for (int h = warp; h < p.G; h += kDwThreads / 32) {
            const float2 *ml = reinterpret_cast<const float2 *>(p.part_ml) + (row0 + h) * p.n_slots;
            float M = -INFINITY;
            for (int c = lane; c < nc; c += 32) M = fmaxf(M, __ldcg(ml + c).x);
            M = warp_max(M);
            float l = 0.f;
            for (int c = lane; c < nc; c += 32) {
                const float2 v = __ldcg(ml + c);
                l = fmaf(v.y, exp2f(v.x - M), l);
            }
            l = warp_sum(l);
            if (lane == 0) max_s[h] = M, inv_s[h] = 1.f / l;
        }
    }
    __syncthreads();
    const int old_len = (weighed != nullptr) ? __ldg(weighed + b) : len - 1;
    const size_t w_row = ((size_t)b * p.Hkv + head) * w_stride;
    float sum[kDwTokens];
#pragma unroll
    for (int i = 0; i < kDwTokens; ++i) sum[i] = 0.f;
    if (len > 1) {
        const float *src = p.scores + row0 * p.score_stride + first + tid;   // (a row's scores reach to the end of its last chunk)
        for (int h = 0; h < p.G; ++h, src += p.score_stride) {
            const float M = max_s[h], inv = inv_s[h];
#pragma unroll
            for (int i = 0; i < kDwTokens; ++i) {
                const int j = first + tid + i * kDwThreads;
                if (j < len) sum[i] = fmaf(exp2f(__ldcg(src + i * kDwThreads) - M), inv, sum[i]);
            }
        }
    } else {
        sum[0] = (float)p.G;
    }
#pragma unroll
    for (int i = 0; i < kDwTokens; ++i) {
        const int j = first + tid + i * kDwThreads;
        if (j < len) {
            const float old = (w_in != nullptr && j < old_len) ? w_in[w_row + j] : 0.f;
            w_out[w_row + j] = fmaf(decay, old, sum[i]);
        }
    }
}

// The scores follow the split pass's workspace, which is a multiple of 8 bytes.
static size_t scores_offset(int B, int Hq, int Hkv, int max_kv)
{
    return (decode_workspace_bytes(B, Hq, Hkv, max_kv) + 255) / 256 * 256;
}

size_t weights_workspace_bytes(int B, int Hq, int Hkv, int max_kv)
{
    const size_t stride = (size_t)(max_kv + kDwChunk - 1) / kDwChunk * kDwChunk;
    return scores_offset(B, Hq, Hkv, max_kv) + (size_t)B * Hq * stride * sizeof(float);
}

int launch_decode_weights(const slim_cache_t *c, const void *q, const void *k_new, const void *v_new, void *out, const float *w_in,
                          float *w_out, int w_stride, const int32_t *weighed, const int32_t *kv_len, int B, int max_kv, int Hq,
                          float sm_scale, float decay, void *workspace, cudaStream_t stream)
{
    DecodeParams p = make_decode_params(c, q, kv_len, B, max_kv, Hq, sm_scale, workspace);
    p.k_new = static_cast<const __nv_bfloat16 *>(k_new);
    p.v_new = static_cast<const __nv_bfloat16 *>(v_new);
    p.scores = reinterpret_cast<float *>(static_cast<char *>(workspace) + scores_offset(B, Hq, c->num_kv_heads, max_kv));
    p.score_stride = p.n_chunks * kDwChunk;
    const int rc = launch_decode_params(c, p, B, out, stream);
    if (rc != SLIM_OK || p.n_chunks == 0) return rc;
    const dim3 grid((unsigned)((max_kv + kDwBlockTokens - 1) / kDwBlockTokens), (unsigned)p.Hkv, (unsigned)B);
    SLIM_CUDA_TRY(launch_pdl(slim_decode_weights_kernel, grid, dim3(kDwThreads), 0, stream, p, w_in, w_out, w_stride, weighed, decay));
    return SLIM_OK;
}

}  // namespace slim

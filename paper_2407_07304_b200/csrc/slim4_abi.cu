// C ABI of the 4-bit cache and of the page tables: argument validation and dispatch (declared in include/slim.h).
#include "slim_common.cuh"

#define SLIM_EXPORT extern "C" __attribute__((visibility("default")))

namespace slim {

int launch_append4(const slim_cache4_t *c, const void *k_new, const void *v_new, const int32_t *cu_new, const int32_t *start_pos, int B,
                   int max_new, cudaStream_t stream, const int32_t *len_after);
int launch_read4(const slim_cache4_t *c, void *k_out, void *v_out, const int32_t *cu, const int32_t *start_pos, int B, int max_rows,
                 cudaStream_t stream);
int launch_decode4(const slim_cache4_t *c, const void *q, const void *k_new, const void *v_new, void *out, const int32_t *kv_len, int B,
                   int max_kv, int Hq, float sm_scale, void *workspace, cudaStream_t stream);
size_t decode4_workspace_bytes(int G);
int launch_prefill4_tc(const slim_cache4_t *c, const void *q, void *out, const int32_t *cu_q, const int32_t *kv_len, int B, int max_q,
                       int Hq, float sm_scale, void *workspace, cudaStream_t stream, bool after_append);
size_t prefill_workspace_bytes();
int launch_pages_fork(const slim_pages_t *from, const slim_pages_t *to, const int32_t *parent, const int32_t *kv_len, int32_t *len_out,
                      const slim_layer_t *layers, int n_layers, int32_t *result, void *workspace, cudaStream_t stream);
int launch_pages_grow(const slim_pages_t *pages, const int32_t *kv_len, int room, int32_t *result, void *workspace, cudaStream_t stream);
int launch_pages_compact(const slim_pages_t *from, const slim_pages_t *to, const slim_layer_t *layers, int n_layers, int32_t *result,
                         void *workspace, cudaStream_t stream);
size_t pages_workspace_bytes(int num_pages, int rows);

static bool misaligned(const void *ptr, uintptr_t bytes) { return ((uintptr_t)ptr & (bytes - 1)) != 0; }

static int check_cache4(const slim_cache4_t *c)
{
    if (c == nullptr || c->codes == nullptr || c->scales == nullptr || c->block_table == nullptr) return SLIM_ERR_INVALID_ARG;
    if (c->num_pages <= 0 || c->num_kv_heads <= 0 || c->max_pages_per_seq <= 0) return SLIM_ERR_INVALID_ARG;
    if (c->page_tokens != SLIM_PAGE_TOKENS || c->head_dim != SLIM_HEAD_DIM) return SLIM_ERR_UNSUPPORTED;
    if (misaligned(c->codes, 16) || misaligned(c->scales, 16)) return SLIM_ERR_INVALID_ARG;
    return SLIM_OK;
}
static bool beyond_pages(const slim_cache4_t *c, int32_t tokens)
{
    return (long long)tokens > (long long)c->max_pages_per_seq * SLIM_PAGE_TOKENS;
}
static int check_scratch(const void *workspace, size_t bytes, size_t need)
{
    if (need > 0 && (workspace == nullptr || bytes < need)) return SLIM_ERR_WORKSPACE;
    return misaligned(workspace, 16) ? SLIM_ERR_INVALID_ARG : SLIM_OK;
}

// Shared by the calls that go through rows of new (or held) tokens; *launch is false for a valid no-op.
static int check_rows4(const slim_cache4_t *cache, const void *k, const void *v, const int32_t *cu, const int32_t *start_pos, int32_t B,
                       int32_t max_rows, bool *launch)
{
    *launch = false;
    const int rc = check_cache4(cache);
    if (rc != SLIM_OK) return rc;
    if (B < 0 || max_rows < 0) return SLIM_ERR_INVALID_ARG;
    if (B == 0 || max_rows == 0) return SLIM_OK;
    if (k == nullptr || v == nullptr || cu == nullptr || start_pos == nullptr) return SLIM_ERR_INVALID_ARG;
    if (misaligned(k, 16) || misaligned(v, 16)) return SLIM_ERR_INVALID_ARG;
    if (B > 65535) return SLIM_ERR_UNSUPPORTED;
    *launch = true;
    return SLIM_OK;
}

}  // namespace slim

using namespace slim;

SLIM_EXPORT int slim_kv4_append(const slim_cache4_t *cache, const void *k_new, const void *v_new, const int32_t *cu_new,
                                const int32_t *start_pos, int32_t B, int32_t max_new, void *stream)
{
    bool launch;
    const int rc = check_rows4(cache, k_new, v_new, cu_new, start_pos, B, max_new, &launch);
    if (rc != SLIM_OK || !launch) return rc;
    return launch_append4(cache, k_new, v_new, cu_new, start_pos, B, max_new, (cudaStream_t)stream, nullptr);
}

SLIM_EXPORT int slim_kv4_read(const slim_cache4_t *cache, void *k_out, void *v_out, const int32_t *cu, const int32_t *start_pos, int32_t B,
                              int32_t max_rows, void *stream)
{
    bool launch;
    const int rc = check_rows4(cache, k_out, v_out, cu, start_pos, B, max_rows, &launch);
    if (rc != SLIM_OK || !launch) return rc;
    return launch_read4(cache, k_out, v_out, cu, start_pos, B, max_rows, (cudaStream_t)stream);
}

static int check_prefill4(const slim_cache4_t *cache, const void *q, const void *out, const int32_t *cu_q, const int32_t *kv_len, int32_t B,
                          int32_t max_q, int32_t max_kv, int32_t Hq, const void *workspace, size_t workspace_bytes, bool *launch)
{
    *launch = false;
    const int rc = check_cache4(cache);
    if (rc != SLIM_OK) return rc;
    if (B < 0 || max_q < 0 || max_kv < 0 || Hq <= 0) return SLIM_ERR_INVALID_ARG;
    if (Hq % cache->num_kv_heads != 0) return SLIM_ERR_UNSUPPORTED;
    if (B == 0 || max_q == 0) return SLIM_OK;
    if (q == nullptr || out == nullptr || cu_q == nullptr || kv_len == nullptr) return SLIM_ERR_INVALID_ARG;
    if (misaligned(q, 16) || misaligned(out, 16)) return SLIM_ERR_INVALID_ARG;
    if (B > 65535 || Hq > 65535) return SLIM_ERR_UNSUPPORTED;
    if (beyond_pages(cache, max_kv)) return SLIM_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < prefill_workspace_bytes()) return SLIM_ERR_WORKSPACE;
    if (misaligned(workspace, 4)) return SLIM_ERR_INVALID_ARG;
    *launch = true;
    return SLIM_OK;
}

SLIM_EXPORT int slim_attn4_prefill(const slim_cache4_t *cache, const void *q, void *out, const int32_t *cu_q, const int32_t *kv_len, int32_t B,
                                   int32_t max_q, int32_t max_kv, int32_t Hq, float sm_scale, void *workspace, size_t workspace_bytes,
                                   void *stream)
{
    bool launch;
    const int rc = check_prefill4(cache, q, out, cu_q, kv_len, B, max_q, max_kv, Hq, workspace, workspace_bytes, &launch);
    if (rc != SLIM_OK || !launch) return rc;
    return launch_prefill4_tc(cache, q, out, cu_q, kv_len, B, max_q, Hq, sm_scale, workspace, (cudaStream_t)stream, false);
}

SLIM_EXPORT int slim_prefill4_step(const slim_cache4_t *cache, const void *q, const void *k_new, const void *v_new, void *out,
                                   const int32_t *cu_q, const int32_t *kv_len, int32_t B, int32_t max_q, int32_t max_kv, int32_t Hq,
                                   float sm_scale, void *workspace, size_t workspace_bytes, void *stream)
{
    bool launch;
    int rc = check_prefill4(cache, q, out, cu_q, kv_len, B, max_q, max_kv, Hq, workspace, workspace_bytes, &launch);
    if (rc != SLIM_OK || !launch) return rc;
    if (k_new == nullptr || v_new == nullptr || misaligned(k_new, 16) || misaligned(v_new, 16)) return SLIM_ERR_INVALID_ARG;
    // the new rows of sequence b go to positions kv_len[b] - q_len[b] ... kv_len[b] - 1
    rc = launch_append4(cache, k_new, v_new, cu_q, nullptr, B, max_q, (cudaStream_t)stream, kv_len);
    if (rc != SLIM_OK) return rc;
    return launch_prefill4_tc(cache, q, out, cu_q, kv_len, B, max_q, Hq, sm_scale, workspace, (cudaStream_t)stream, true);
}

SLIM_EXPORT int slim_attn4_decode(const slim_cache4_t *cache, const void *q, const void *k_new, const void *v_new, void *out,
                                  const int32_t *kv_len, int32_t B, int32_t max_kv, int32_t Hq, float sm_scale, void *workspace,
                                  size_t workspace_bytes, void *stream)
{
    int rc = check_cache4(cache);
    if (rc != SLIM_OK) return rc;
    if (B < 0 || max_kv < 0 || Hq <= 0) return SLIM_ERR_INVALID_ARG;
    if (Hq % cache->num_kv_heads != 0 || Hq / cache->num_kv_heads > 16) return SLIM_ERR_UNSUPPORTED;
    if (B == 0) return SLIM_OK;
    if (B > 65535 || (long long)B * cache->num_kv_heads > 0x7FFFFFFFLL) return SLIM_ERR_UNSUPPORTED;   // (pairs are counted in 32 bits)
    if (beyond_pages(cache, max_kv)) return SLIM_ERR_INVALID_ARG;
    if (q == nullptr || out == nullptr || kv_len == nullptr || misaligned(q, 16) || misaligned(out, 16)) return SLIM_ERR_INVALID_ARG;
    if ((k_new == nullptr) != (v_new == nullptr) || misaligned(k_new, 16) || misaligned(v_new, 16)) return SLIM_ERR_INVALID_ARG;
    rc = check_scratch(workspace, workspace_bytes, slim_attn4_workspace_bytes(Hq, cache->num_kv_heads));
    if (rc != SLIM_OK) return rc;
    return launch_decode4(cache, q, k_new, v_new, out, kv_len, B, max_kv, Hq, sm_scale, workspace, (cudaStream_t)stream);
}

SLIM_EXPORT size_t slim_attn4_workspace_bytes(int32_t Hq, int32_t Hkv)
{
    if (Hq <= 0 || Hkv <= 0 || Hq % Hkv != 0 || Hq / Hkv > 16) return 0;
    return decode4_workspace_bytes(Hq / Hkv);
}
SLIM_EXPORT size_t slim_cache4_code_bytes(int32_t num_pages, int32_t num_kv_heads)
{
    if (num_pages <= 0 || num_kv_heads <= 0) return 0;
    return (size_t)num_pages * num_kv_heads * 2 * SLIM_PAGE_TOKENS * (SLIM_HEAD_DIM / 2);
}
SLIM_EXPORT size_t slim_cache4_scale_bytes(int32_t num_pages, int32_t num_kv_heads)
{
    if (num_pages <= 0 || num_kv_heads <= 0) return 0;
    return (size_t)num_pages * num_kv_heads * 2 * SLIM_PAGE_TOKENS * 4;
}

// ---------------------------------------------------------------- page tables
static int check_pages(const slim_pages_t *p)
{
    if (p == nullptr || p->num_pages <= 0 || p->rows < 0 || p->stride <= 0) return SLIM_ERR_INVALID_ARG;
    if (p->refs == nullptr || misaligned(p->refs, 4)) return SLIM_ERR_INVALID_ARG;
    if (p->rows > 0 && (p->table == nullptr || p->held == nullptr || misaligned(p->table, 4) || misaligned(p->held, 4))) return SLIM_ERR_INVALID_ARG;
    if (p->num_pages > (1 << 23) || p->rows > (1 << 23)) return SLIM_ERR_UNSUPPORTED;   // (sums over either stay inside 32 bits)
    return SLIM_OK;
}
// Whether two arrays of 32-bit numbers share one.
static bool overlap(const int32_t *a, size_t n_a, const int32_t *b, size_t n_b)
{
    return n_a > 0 && n_b > 0 && (uintptr_t)a < (uintptr_t)(b + n_b) && (uintptr_t)b < (uintptr_t)(a + n_a);
}
static bool overlap_in_part(const int32_t *a, const int32_t *b, size_t n) { return a != b && overlap(a, n, b, n); }
static size_t entries(const slim_pages_t *p) { return (size_t)p->rows * p->stride; }
static int check_layers(const slim_layer_t *layers, int32_t n_layers)
{
    if (n_layers < 0 || (n_layers > 0 && layers == nullptr)) return SLIM_ERR_INVALID_ARG;
    for (int i = 0; i < n_layers; ++i) {
        const slim_layer_t &l = layers[i];
        if (l.codes == nullptr || l.scales == nullptr || misaligned(l.codes, 16) || misaligned(l.scales, 16)) return SLIM_ERR_INVALID_ARG;
        if (l.num_kv_heads <= 0) return SLIM_ERR_INVALID_ARG;
        if (l.num_kv_heads > 65535 || (l.row_bytes != SLIM_HEAD_DIM && l.row_bytes != SLIM_HEAD_DIM / 2)) return SLIM_ERR_UNSUPPORTED;
    }
    return SLIM_OK;
}

SLIM_EXPORT int slim_pages_fork(const slim_pages_t *from, const slim_pages_t *to, const int32_t *parent, const int32_t *kv_len, int32_t *len_out,
                                const slim_layer_t *layers, int32_t n_layers, int32_t *result, void *workspace, size_t workspace_bytes,
                                void *stream)
{
    int rc = check_pages(from);
    if (rc == SLIM_OK) rc = check_pages(to);
    if (rc == SLIM_OK) rc = check_layers(layers, n_layers);
    if (rc != SLIM_OK) return rc;
    if (from->num_pages != to->num_pages || from->stride != to->stride) return SLIM_ERR_INVALID_ARG;
    if (result == nullptr || (to->rows > 0 && (parent == nullptr || len_out == nullptr)) || (from->rows > 0 && kv_len == nullptr)) return SLIM_ERR_INVALID_ARG;
    // (rows of `from`, lengths and parents are read while those of `to` are written)
    if (overlap(from->table, entries(from), to->table, entries(to)) || overlap(from->held, from->rows, to->held, to->rows)) return SLIM_ERR_INVALID_ARG;
    if (overlap(kv_len, from->rows, len_out, to->rows) || overlap(parent, to->rows, len_out, to->rows)) return SLIM_ERR_INVALID_ARG;
    if (overlap_in_part(from->refs, to->refs, from->num_pages)) return SLIM_ERR_INVALID_ARG;
    rc = check_scratch(workspace, workspace_bytes, slim_pages_workspace_bytes(from->num_pages, from->rows > to->rows ? from->rows : to->rows));
    if (rc != SLIM_OK) return rc;
    return launch_pages_fork(from, to, parent, kv_len, len_out, layers, n_layers, result, workspace, (cudaStream_t)stream);
}

SLIM_EXPORT int slim_pages_grow(const slim_pages_t *pages, const int32_t *kv_len, int32_t room, int32_t *result, void *workspace,
                                size_t workspace_bytes, void *stream)
{
    int rc = check_pages(pages);
    if (rc != SLIM_OK) return rc;
    if (room < 0 || result == nullptr || (pages->rows > 0 && kv_len == nullptr)) return SLIM_ERR_INVALID_ARG;
    rc = check_scratch(workspace, workspace_bytes, slim_pages_workspace_bytes(pages->num_pages, pages->rows));
    if (rc != SLIM_OK) return rc;
    return launch_pages_grow(pages, kv_len, room, result, workspace, (cudaStream_t)stream);
}

SLIM_EXPORT int slim_pages_compact(const slim_pages_t *from, const slim_pages_t *to, const slim_layer_t *layers, int32_t n_layers, int32_t *result,
                                   void *workspace, size_t workspace_bytes, void *stream)
{
    int rc = check_pages(from);
    if (rc == SLIM_OK) rc = check_pages(to);
    if (rc == SLIM_OK) rc = check_layers(layers, n_layers);
    if (rc != SLIM_OK) return rc;
    if (from->num_pages != to->num_pages || from->stride != to->stride || from->rows != to->rows || result == nullptr) return SLIM_ERR_INVALID_ARG;
    if (overlap_in_part(from->table, to->table, entries(from)) || overlap_in_part(from->held, to->held, from->rows) ||
        overlap_in_part(from->refs, to->refs, from->num_pages)) return SLIM_ERR_INVALID_ARG;
    rc = check_scratch(workspace, workspace_bytes, slim_pages_workspace_bytes(from->num_pages, from->rows));
    if (rc != SLIM_OK) return rc;
    return launch_pages_compact(from, to, layers, n_layers, result, workspace, (cudaStream_t)stream);
}

SLIM_EXPORT size_t slim_pages_workspace_bytes(int32_t num_pages, int32_t rows)
{
    if (num_pages <= 0 || rows < 0) return 0;
    return pages_workspace_bytes(num_pages, rows);
}

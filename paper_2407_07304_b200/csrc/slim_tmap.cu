// TMA tensor maps of the INT8 code pool (host side).
//
// The pool [num_pages][Hkv][2][128 slots][128 dims] is described to the copy engine as a 2-D
// byte tensor [rows][128] with rows = num_pages * Hkv * 2 * 128: one row per cached (token, kv
// head, K|V) vector.  A box of `box_rows` rows lands in shared memory with the 128-byte swizzle,
// which is the layout the tensor cores read directly.  x is always 0 (16-byte rule trivially met).
#include <cuda.h>

#include <mutex>

#include "slim_common.cuh"
#include "slim_tmap.cuh"

namespace slim {

namespace {
typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// What a map is made of: a pool seen as rows (2-D) or as blocks of rows (3-D).
struct Shape {
    const void *ptr;
    CUtensorMapDataType type;
    int dims;
    cuuint64_t size[3], stride[2];   // elements; bytes
    cuuint32_t box[3];
    CUtensorMapSwizzle swizzle;
};
struct Entry {
    Shape shape;
    CUtensorMap map;
};
constexpr int kEntries = 256;

bool same_shape(const Shape &a, const Shape &b)
{
    if (a.ptr != b.ptr || a.type != b.type || a.dims != b.dims || a.swizzle != b.swizzle) return false;
    for (int i = 0; i < a.dims; ++i)
        if (a.size[i] != b.size[i] || a.box[i] != b.box[i] || (i > 0 && a.stride[i - 1] != b.stride[i - 1])) return false;
    return true;
}

// Maps are cached by their shape; thread-safe.
int tensor_map(const Shape &want, CUtensorMap *out)
{
    static std::mutex mu;
    static EncodeTiledFn encode = nullptr;
    static Entry cache[kEntries];
    static int used = 0, next = 0;
    std::lock_guard<std::mutex> lock(mu);
    if (encode == nullptr) {
        void *fn = nullptr;
        cudaDriverEntryPointQueryResult qres;
        SLIM_CUDA_TRY(cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres));
        if (fn == nullptr || qres != cudaDriverEntryPointSuccess) return SLIM_ERR_UNSUPPORTED;
        encode = reinterpret_cast<EncodeTiledFn>(fn);
    }
    for (int i = 0; i < used; ++i) {
        if (same_shape(cache[i].shape, want)) {
            *out = cache[i].map;
            return SLIM_OK;
        }
    }
    Entry e;
    e.shape = want;
    const cuuint32_t estr[3] = {1, 1, 1};
    const CUresult r = encode(&e.map, want.type, (cuuint32_t)want.dims, const_cast<void *>(want.ptr), want.size, want.stride, want.box, estr,
                              CU_TENSOR_MAP_INTERLEAVE_NONE, want.swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return SLIM_ERR_CUDA;
    cache[next] = e;
    next = (next + 1) % kEntries;
    if (used < kEntries) ++used;
    *out = e.map;
    return SLIM_OK;
}

Shape rows_shape(const void *ptr, long long rows, int box_rows)
{
    Shape s = {};
    s.ptr = ptr;
    s.type = CU_TENSOR_MAP_DATA_TYPE_UINT8;
    s.dims = 2;
    s.size[0] = s.stride[0] = s.box[0] = kHeadDim;
    s.size[1] = (cuuint64_t)rows;
    s.box[1] = (cuuint32_t)box_rows;
    s.swizzle = CU_TENSOR_MAP_SWIZZLE_128B;
    return s;
}
template <class Cache>
long long pool_blocks(const Cache *c)   // (page, head, K|V)
{
    return (long long)c->num_pages * c->num_kv_heads * 2;
}
}  // namespace

int codes_tensor_map(const slim_cache_t *c, int box_rows, CUtensorMap *out)
{
    return tensor_map(rows_shape(c->codes, pool_blocks(c) * kPageTokens, box_rows), out);
}

int unit4_tensor_maps(const slim_cache4_t *c, int blocks, CUtensorMap *codes, CUtensorMap *pairs)
{
    // (rows of 1 KB, sixteen slots each: the copy engine takes a box row by row)
    constexpr int kBlock = kPageTokens * kHeadDim / 2, kRow = 1024;
    Shape s = {};
    s.ptr = c->codes;
    s.type = CU_TENSOR_MAP_DATA_TYPE_UINT32;
    s.dims = 3;
    s.size[0] = s.box[0] = kRow / 4;
    s.stride[0] = kRow;
    s.size[1] = kBlock / kRow;
    s.stride[1] = kBlock;
    s.size[2] = (cuuint64_t)pool_blocks(c);
    s.box[1] = kBlock / kRow / 2;
    s.box[2] = (cuuint32_t)blocks;
    s.swizzle = CU_TENSOR_MAP_SWIZZLE_NONE;
    const int rc = tensor_map(s, codes);
    if (rc != SLIM_OK) return rc;
    s.ptr = c->scales;
    s.dims = 2;
    s.size[0] = kPageTokens;
    s.stride[0] = kPageTokens * 4;
    s.size[1] = (cuuint64_t)pool_blocks(c);
    s.box[0] = kPageTokens / 2;
    s.box[1] = 2;
    return tensor_map(s, pairs);
}

int sm_count(int *out)
{
    static int cached[64];
    int dev = 0;
    SLIM_CUDA_TRY(cudaGetDevice(&dev));
    if (dev < 0 || dev >= 64) return SLIM_ERR_UNSUPPORTED;
    if (cached[dev] == 0) {
        int n = 0;
        SLIM_CUDA_TRY(cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev));
        cached[dev] = n;
    }
    *out = cached[dev];
    return SLIM_OK;
}

int allow_dynamic_smem(const void *func, int bytes)
{
    struct Done {
        int dev;
        const void *func;
    };
    static std::mutex mu;
    static Done done[64];
    static int n_done = 0;
    int dev = 0;
    SLIM_CUDA_TRY(cudaGetDevice(&dev));
    std::lock_guard<std::mutex> lock(mu);
    for (int i = 0; i < n_done; ++i)
        if (done[i].dev == dev && done[i].func == func) return SLIM_OK;
    SLIM_CUDA_TRY(cudaFuncSetAttribute(func, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes));
    if (n_done < 64) done[n_done++] = Done{dev, func};
    return SLIM_OK;
}

}  // namespace slim

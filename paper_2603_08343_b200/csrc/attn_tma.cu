// Tensor maps of the paged caches.
#include "attn_host.h"
#include "attn_kernels.cuh"

namespace wht_host {

using namespace wht;

namespace {

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                 const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                 CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_function(EncodeTiled* out) {
    static EncodeTiled cached = nullptr;
    if (!cached) {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult found;
        WHT_CUDA_TRY(cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found));
        if (found != cudaDriverEntryPointSuccess || !f) return cuda_fail(cudaErrorNotSupported);
        cached = reinterpret_cast<EncodeTiled>(f);
    }
    *out = cached;
    return WHT_OK;
}

int cache_map(EncodeTiled encode, CUtensorMap* map, const void* cache, const AttnParams& p, int d, int dtype, int box_rows) {
    const unsigned elem = dtype == WHT_F32 ? 4 : 2;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(p.num_pages * p.hkv) << p.page_shift};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(d) * elem};
    const cuuint32_t box[2] = {128u / elem, static_cast<cuuint32_t>(box_rows)}, unit[2] = {1u, 1u};
    if (encode(map, dtype == WHT_F32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(cache),
               dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cuda_fail(cudaErrorInvalidValue);
    return WHT_OK;
}

}  // namespace

int cache_maps(CUtensorMap* k_map, CUtensorMap* v_map, const AttnParams& p, int d, int dtype, int box_rows) {
    EncodeTiled encode = nullptr;
    int rc = encode_function(&encode);
    if (rc == WHT_OK) rc = cache_map(encode, k_map, p.k_cache, p, d, dtype, box_rows);
    if (rc == WHT_OK) rc = cache_map(encode, v_map, p.v_cache, p, d, dtype, box_rows);
    return rc;
}

}  // namespace wht_host

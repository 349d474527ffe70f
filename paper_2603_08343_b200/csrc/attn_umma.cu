// Shared-prefix attention on the tcgen05 tensor core: tensor maps, launch geometry and instantiations.
#include "attn_umma_kernels.cuh"

#include "attn_host.h"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_umma)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attn_umma)

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

// A cache as [num_pages * Hkv * page] rows of D channels, copied in boxes of one page by 64 channels.
int cache_map(CUtensorMap* map, const void* cache, const AttnParams& p, int d) {
    EncodeTiled encode = nullptr;
    const int rc = encode_function(&encode);
    if (rc != WHT_OK) return rc;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(d), static_cast<cuuint64_t>(p.num_pages * p.hkv) << p.page_shift};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(d) * 2};
    const cuuint32_t box[2] = {64u, 1u << p.page_shift}, unit[2] = {1u, 1u};
    if (encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(cache), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return cuda_fail(cudaErrorInvalidValue);
    return WHT_OK;
}

template <int D>
int launch(const UmmaAttnParams& up, int dev, cudaStream_t s) {
    using Geo = UmmaAttnGeo<D>;
    static_assert(Geo::BYTES <= 227 * 1024 && Geo::BYTES > 116 * 1024, "one block per SM");
    static int ready[kMaxDevices] = {};
    int rc = prepare_umma(attn_umma_prefix_kernel<D>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    CUtensorMap k_map, v_map;
    rc = cache_map(&k_map, up.a.k_cache, up.a, D);
    if (rc == WHT_OK) rc = cache_map(&v_map, up.a.v_cache, up.a, D);
    if (rc != WHT_OK) return rc;
    const long long blocks = static_cast<long long>(up.splits) * up.row_blocks * up.a.hkv;
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    attn_umma_prefix_kernel<D><<<static_cast<unsigned>(blocks), kUmmaAttnThreads, Geo::BYTES, s>>>(up, k_map, v_map);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace

int launch_attn_umma_prefix(const UmmaAttnParams& up, int d, int dev, cudaStream_t s) {
    return d == 64 ? launch<64>(up, dev, s) : d == 96 ? launch<96>(up, dev, s) : launch<128>(up, dev, s);
}

}  // namespace wht_host

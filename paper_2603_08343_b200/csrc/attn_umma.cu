// Shared-prefix attention on the tcgen05 tensor core: tensor maps, launch geometry and instantiations.
#include "attn_umma_kernels.cuh"

#include "attn_host.h"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_umma)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attn_umma)

namespace {

template <int D>
int launch(const UmmaAttnParams& up, int dev, cudaStream_t s) {
    using Geo = UmmaAttnGeo<D>;
    static_assert(Geo::BYTES <= 227 * 1024 && Geo::BYTES > 116 * 1024, "one block per SM");
    static int ready[kMaxDevices] = {};
    int rc = prepare_umma(attn_umma_prefix_kernel<D>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    CUtensorMap k_map, v_map;
    rc = cache_maps(&k_map, &v_map, up.a, D, WHT_BF16, 1 << up.a.page_shift);
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

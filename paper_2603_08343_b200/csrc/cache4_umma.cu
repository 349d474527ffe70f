// Prompts over the 4-bit cache on the tcgen05 tensor core: launches.
#include "cache4_host.h"
#include "cache4_umma_kernels.cuh"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_umma4)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_umma4)

namespace {

template <int D>
int launch(const Attn4Params& p, int dev, cudaStream_t s) {
    using Geo = Umma4Geo<D>;
    static_assert(Geo::BYTES <= 227 * 1024, "shared memory");
    static_assert(kUmma4Rows == wht_plan::kUmma4Rows && kUmma4Keys == 16 << wht_plan::kUmma4Grain, "the plan's units and grains");
    static int ready[kMaxDevices] = {};
    if (!ready[dev]) {
        WHT_CUDA_TRY(cudaFuncSetAttribute(attn4_umma_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Geo::BYTES));
        WHT_CUDA_TRY(cudaFuncSetAttribute(attn4_umma_kernel<D>, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
        ready[dev] = 1;
    }
    launch_overlapped(attn4_umma_kernel<D>, dim3(static_cast<unsigned>(p.warps)), kUmma4Threads, Geo::BYTES, s, p);
    WHT_CUDA_TRY(cudaGetLastError());
    const long long rows = static_cast<long long>(p.a.T) * p.a.hq;
    launch_overlapped(attn4_join_kernel<__nv_bfloat16, D>, dim3(static_cast<unsigned>(ceil_div(rows, 4))), 128, 0, s, p, static_cast<int>(kUmma4Rows));
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace

int launch_attend4_umma(const Attn4Params& p, int d, int dev, cudaStream_t s) {
    return d == 64 ? launch<64>(p, dev, s) : d == 96 ? launch<96>(p, dev, s) : launch<128>(p, dev, s);
}

}  // namespace wht_host

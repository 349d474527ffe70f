// Eviction from the 4-bit cache: launch geometry and instantiations.
#include "cache4_evict_kernels.cuh"
#include "cache4_host.h"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_evict4)

namespace {
constexpr int kEvictThreads = 512;

template <int D>
void move(const Evict4Params& p, unsigned blocks, cudaStream_t s) {
    launch_overlapped(kv_evict4_move_kernel<D>, dim3(blocks), 32 * kMove4Warps, 0, s, p);
}
}  // namespace

int launch_evict4(const Evict4Params& p, int d, cudaStream_t s) {
    const long long rows = static_cast<long long>(p.a.B) * p.a.hkv;
    const long long blocks = ceil_div(rows * ceil_div(p.budget, kTileKeys), kMove4Warps);
    if (rows > 0x7fffffffll || blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    kv_evict4_choose_kernel<kEvictThreads><<<static_cast<unsigned>(rows), kEvictThreads, 0, s>>>(p);
    WHT_CUDA_TRY(cudaGetLastError());
    const unsigned n = static_cast<unsigned>(blocks);
    d == 64 ? move<64>(p, n, s) : d == 96 ? move<96>(p, n, s) : move<128>(p, n, s);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace wht_host

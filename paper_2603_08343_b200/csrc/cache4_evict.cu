// Eviction from the 4-bit cache: launch geometry and instantiations.
#include "cache4_evict_kernels.cuh"
#include "cache4_host.h"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_evict4)

namespace {

template <int D>
void move(const Evict4Params& p, unsigned blocks, cudaStream_t s) {
    launch_overlapped(kv_evict4_move_kernel<D>, dim3(blocks), 32 * kMove4Warps, 0, s, p);
}
}  // namespace

int launch_evict4(const Evict4Params& p, int d, cudaStream_t s) {
    const long long rows = static_cast<long long>(p.a.B) * p.a.hkv;
    const long long blocks = ceil_div(rows * ceil_div(p.budget, kTileKeys), kMove4Warps);
    if (rows > 0x7fffffffll || blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    // Blocks that have an SM each take twice the threads (us: 1 x 4096 keys, 8 heads, 8.9 against 9.8; 64 rows of up to 2500 9.1 against 10.2), more blocks
    // share SMs two by two (256 rows of up to 16384 keys 28.8 against 31.2).
    int dev = 0, sms = 0;
    const int rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    if (rows <= sms) launch_overlapped(kv_evict4_choose_kernel<1024>, dim3(static_cast<unsigned>(rows)), 1024, 0, s, p);
    else launch_overlapped(kv_evict4_choose_kernel<512>, dim3(static_cast<unsigned>(rows)), 512, 0, s, p);
    WHT_CUDA_TRY(cudaGetLastError());
    const unsigned n = static_cast<unsigned>(blocks);
    d == 64 ? move<64>(p, n, s) : d == 96 ? move<96>(p, n, s) : move<128>(p, n, s);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace wht_host

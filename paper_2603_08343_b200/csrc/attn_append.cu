// Paged-cache append: launch geometry and instantiations.
#include "attn_host.h"
#include "kv_append_kernels.cuh"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_append)

namespace {
template <typename T, bool INTERLEAVED>
void launch(const AppendParams& p, int blocks, cudaStream_t s) {
    if (p.summary)
        kv_append_kernel<T, INTERLEAVED, true><<<blocks, kAppendThreads, 0, s>>>(p);
    else
        kv_append_kernel<T, INTERLEAVED, false><<<blocks, kAppendThreads, 0, s>>>(p);
}
}  // namespace

int launch_append(AppendParams& p, int dtype, bool interleaved, int sms, cudaStream_t s) {
    (void)sms;
    p.rows = p.hq + (p.summary ? 1 : 2) * p.hkv;
    const int per_token = p.rows * (p.d / 16);
    // tokens per tile: about two items per thread and block row, so that a tile's index arithmetic stays small
    p.tile = per_token >= 2 * kAppendThreads ? 1 : 2 * kAppendThreads / per_token;
    p.flat_x = static_cast<int>(ceil_div(p.T, p.tile));
    p.flat_y = static_cast<int>(ceil_div(static_cast<long long>(p.tile) * per_token, 2 * kAppendThreads));
    long long blocks = static_cast<long long>(p.flat_x) * p.flat_y;
    if (p.summary) {
        // few tokens: every run gets a warp at once; many: fewer blocks, most of which find no run to own
        p.run_tile = p.T * p.hkv <= 8192 ? 8 : 32;
        blocks += ceil_div(p.T, p.run_tile) * p.hkv;
    }
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    if (dtype == WHT_F32)
        interleaved ? launch<float, true>(p, static_cast<int>(blocks), s) : launch<float, false>(p, static_cast<int>(blocks), s);
    else
        interleaved ? launch<__nv_bfloat16, true>(p, static_cast<int>(blocks), s)
                    : launch<__nv_bfloat16, false>(p, static_cast<int>(blocks), s);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace wht_host

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

int launch_append(AppendParams& p, int dtype, bool interleaved, cudaStream_t s) {
    const int hb = dtype == WHT_F32 ? kHeadBlock<float> : kHeadBlock<__nv_bfloat16>;
    p.q_blocks = static_cast<int>(ceil_div(p.hq, hb));
    p.kv_blocks = static_cast<int>(ceil_div(p.hkv, hb));
    const int per_token = (p.q_blocks + (p.summary ? 1 : 2) * p.kv_blocks) * (p.d / 16);
    p.tile = per_token >= kAppendThreads ? 1 : kAppendThreads / per_token;
    p.flat_x = static_cast<int>(ceil_div(p.T, p.tile));
    p.flat_y = static_cast<int>(ceil_div(static_cast<long long>(p.tile) * per_token, kAppendThreads));
    long long blocks = static_cast<long long>(p.flat_x) * p.flat_y;
    if (p.summary) {
        // A block's eight warps take the runs of a tile of tokens for eight heads: four tokens a tile in a decode step, where every
        // token is a run; more in prompts (a run per page), where most tiles of a few tokens would find none to own.
        p.run_heads = p.hkv < 8 ? p.hkv : 8;
        p.run_tile = p.T < 4 * 512 ? 4 : p.T < 32 * 512 ? static_cast<int>(p.T / 512) : 32;
        const long long page_blocks = ceil_div(p.T, p.run_tile) * ceil_div(p.hkv, p.run_heads);
        blocks += page_blocks;
        if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
        p.page_blocks = static_cast<int>(page_blocks);
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

// Append to and reading of the 4-bit cache: launch geometry and instantiations.
#include "cache4_append_kernels.cuh"
#include "cache4_host.h"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_append4)

namespace {

template <typename T, bool INTERLEAVED>
void append(const Append4Params& p, int d, unsigned blocks, cudaStream_t s) {
    if (d == 64) launch_overlapped(kv_append4_kernel<T, INTERLEAVED, 64>, dim3(blocks), kAppend4Threads, 0, s, p);
    else if (d == 96) launch_overlapped(kv_append4_kernel<T, INTERLEAVED, 96>, dim3(blocks), kAppend4Threads, 0, s, p);
    else launch_overlapped(kv_append4_kernel<T, INTERLEAVED, 128>, dim3(blocks), kAppend4Threads, 0, s, p);
}

template <typename T>
void read(const Read4Params& p, int d, unsigned blocks, cudaStream_t s) {
    if (d == 64) launch_overlapped(kv_read4_kernel<T, 64>, dim3(blocks), 256, 0, s, p);
    else if (d == 96) launch_overlapped(kv_read4_kernel<T, 96>, dim3(blocks), 256, 0, s, p);
    else launch_overlapped(kv_read4_kernel<T, 128>, dim3(blocks), 256, 0, s, p);
}

}  // namespace

int launch_append4(Append4Params& p, int dtype, bool interleaved, int d, cudaStream_t s) {
    const int hb = dtype == WHT_F32 ? kHeads4<float> : kHeads4<__nv_bfloat16>;
    p.a.q_blocks = static_cast<int>(ceil_div(p.a.hq, hb));
    p.a.kv_blocks = static_cast<int>(ceil_div(p.a.hkv, hb));
    const long long kv_grid = ceil_div(p.a.T * 2 * p.a.kv_blocks * (d == 64 ? 4 : 8), kAppend4Threads);
    const long long blocks = kv_grid + ceil_div(p.a.T * p.a.q_blocks * (d / 16), kAppend4Threads);
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    p.kv_grid = static_cast<int>(kv_grid);
    const unsigned n = static_cast<unsigned>(blocks);
    if (dtype == WHT_F32) interleaved ? append<float, true>(p, d, n, s) : append<float, false>(p, d, n, s);
    else interleaved ? append<__nv_bfloat16, true>(p, d, n, s) : append<__nv_bfloat16, false>(p, d, n, s);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

int launch_read4(const Read4Params& p, int dtype, int d, cudaStream_t s) {
    const long long blocks = ceil_div(p.n * ceil_div(p.hkv, kReadHeads4) * (d / 8), 256);
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    dtype == WHT_F32 ? read<float>(p, d, static_cast<unsigned>(blocks), s) : read<__nv_bfloat16>(p, d, static_cast<unsigned>(blocks), s);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace wht_host

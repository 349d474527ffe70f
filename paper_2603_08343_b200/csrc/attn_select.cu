// Page selection: launch geometry and instantiations.
#include "attn_host.h"
#include "select_kernels.cuh"

namespace wht_host {

using namespace wht;

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_select)

namespace {

template <typename T, int D, int TQ>
int score(SelectParams& p, cudaStream_t s) {
    p.token_tiles = static_cast<int>(ceil_div(p.a.max_q_len, TQ));
    p.chunks = static_cast<int>(ceil_div(p.a.table_width, kScoreThreads));
    const long long blocks = static_cast<long long>(p.a.B) * p.token_tiles * p.a.hkv * p.chunks;
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    attn_score_kernel<T, D, TQ><<<static_cast<unsigned>(blocks), kScoreThreads, 0, s>>>(p);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int score_tq(SelectParams& p, cudaStream_t s) {
    return p.a.max_q_len == 1 ? score<T, D, 1>(p, s) : score<T, D, 16>(p, s);
}

template <typename T>
int score_d(SelectParams& p, int d, cudaStream_t s) {
    return d == 64 ? score_tq<T, 64>(p, s) : d == 96 ? score_tq<T, 96>(p, s) : score_tq<T, 128>(p, s);
}

template <int THREADS>
int pick(const SelectParams& p, cudaStream_t s) {
    const size_t smem = static_cast<size_t>(p.a.table_width) * 4;
    if (smem > 48 * 1024)
        WHT_CUDA_TRY(cudaFuncSetAttribute(attn_pick_kernel<THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem)));
    launch_overlapped(attn_pick_kernel<THREADS>, dim3(static_cast<unsigned>(p.a.T * p.a.hkv)), THREADS, smem, s, p);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D, int TQ>
int select_one(SelectParams& p, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    p.token_tiles = static_cast<int>(ceil_div(p.a.max_q_len, TQ));
    const size_t smem = static_cast<size_t>(TQ) * p.stride * sizeof(int32_t);
    int dev = 0, sms = 0;
    const int rc = device_info(&dev, &sms);
    if (rc != WHT_OK) return rc;
    if (!ready[dev]) {
        WHT_CUDA_TRY(cudaFuncSetAttribute(attn_select_kernel<T, D, TQ>, cudaFuncAttributeMaxDynamicSharedMemorySize, 100 * 1024));
        ready[dev] = 1;
    }
    const long long blocks = static_cast<long long>(p.a.B) * p.token_tiles * p.a.hkv;
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    attn_select_kernel<T, D, TQ><<<static_cast<unsigned>(blocks), kSelectThreads, smem, s>>>(p);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T>
int select_d(SelectParams& p, int d, cudaStream_t s) {
    if (p.a.max_q_len == 1)
        return d == 64 ? select_one<T, 64, 1>(p, s) : d == 96 ? select_one<T, 96, 1>(p, s) : select_one<T, 128, 1>(p, s);
    return d == 64 ? select_one<T, 64, 16>(p, s) : d == 96 ? select_one<T, 96, 16>(p, s) : select_one<T, 128, 16>(p, s);
}

}  // namespace

int launch_select(SelectParams& p, bool one_kernel, int dtype, int d, cudaStream_t s) {
    if (one_kernel) return dtype == WHT_F32 ? select_d<float>(p, d, s) : select_d<__nv_bfloat16>(p, d, s);
    const int rc = dtype == WHT_F32 ? score_d<float>(p, d, s) : score_d<__nv_bfloat16>(p, d, s);
    if (rc != WHT_OK) return rc;
    // a thread holds a few of a row's candidates at most; long rows get a larger block
    return p.a.table_width <= 1024 ? pick<128>(p, s) : pick<512>(p, s);
}

}  // namespace wht_host

// Launches of the paged attention kernels for one storage type.
#pragma once
#include "attn_host.h"
#include "attn_kernels.cuh"

namespace wht_host {

using namespace wht;

template <typename Kernel>
int attn_prepare(Kernel kernel, int smem, int dev, int* cache) {
    if (cache[dev]) return WHT_OK;
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    cache[dev] = 1;
    return WHT_OK;
}

template <typename T, int D>
int attn_prefix_d(const AttnParams& p, int dev, bool overlapped, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = AttnRow<T, D>;
    const int rc = attn_prepare(attn_prefix_kernel<T, D>, Geo::SMEM, dev, ready);
    if (rc != WHT_OK) return rc;
    const long long prefix_units = static_cast<long long>(p.prefix_splits) * p.prefix_row_tiles * p.hkv;
    const long long own_units = static_cast<long long>(p.B) * p.hkv * p.own_row_tiles * p.own_splits;
    if (prefix_units > 0x3fffffffll || own_units > 0x3fffffffll) return WHT_ERR_BAD_T;
    const long long blocks = ceil_div(prefix_units, attn_groups(p.prefix_rw)) + ceil_div(own_units, attn_groups(p.own_rw));
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    if (overlapped) launch_overlapped(attn_prefix_kernel<T, D>, dim3(static_cast<unsigned>(blocks)), kAttnThreads, Geo::SMEM, s, p);
    else attn_prefix_kernel<T, D><<<static_cast<unsigned>(blocks), kAttnThreads, Geo::SMEM, s>>>(p);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int attn_chosen_d(const AttnParams& p, int dev, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = AttnRow<T, D>;
    const int rc = attn_prepare(attn_chosen_kernel<T, D>, Geo::SMEM, dev, ready);
    if (rc != WHT_OK) return rc;
    const long long blocks = ceil_div(static_cast<long long>(p.T) * p.hkv * p.own_row_tiles * p.own_splits, attn_groups(p.own_rw));
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    launch_overlapped(attn_chosen_kernel<T, D>, dim3(static_cast<unsigned>(blocks)), kAttnThreads, Geo::SMEM, s, p);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int attn_join_d(const AttnParams& p, cudaStream_t s) {
    const long long rows = static_cast<long long>(p.T) * p.hq;
    launch_overlapped(attn_join_kernel<T, D>, dim3(static_cast<unsigned>(ceil_div(rows, 4))), 128, 0, s, p.part_ml, p.part_o,
                      static_cast<T*>(p.out), static_cast<int64_t>(rows), p.parts);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T>
int launch_attn_prefix(const AttnParams& p, int d, int dev, bool o, cudaStream_t s) {
    return d == 64 ? attn_prefix_d<T, 64>(p, dev, o, s) : d == 96 ? attn_prefix_d<T, 96>(p, dev, o, s) : attn_prefix_d<T, 128>(p, dev, o, s);
}
template <typename T>
int launch_attn_chosen(const AttnParams& p, int d, int dev, cudaStream_t s) {
    return d == 64 ? attn_chosen_d<T, 64>(p, dev, s) : d == 96 ? attn_chosen_d<T, 96>(p, dev, s) : attn_chosen_d<T, 128>(p, dev, s);
}
template <typename T>
int launch_attn_join(const AttnParams& p, int d, cudaStream_t s) {
    return d == 64 ? attn_join_d<T, 64>(p, s) : d == 96 ? attn_join_d<T, 96>(p, s) : attn_join_d<T, 128>(p, s);
}

}  // namespace wht_host

// Launches of the paged attention kernels for one storage type.
#pragma once
#include "attn_host.h"
#include "attn_kernels.cuh"

namespace wht_host {

using namespace wht;

// (internal linkage: the statics below belong to this library alone, also where a process loads two builds of it)
namespace {

template <typename Kernel>
int attn_prepare(Kernel kernel, int smem, int dev, int* cache) {
    if (cache[dev]) return WHT_OK;
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    cache[dev] = 1;
    return WHT_OK;
}

template <typename T>
constexpr int attn_code() { return sizeof(T) == 4 ? WHT_F32 : WHT_BF16; }

template <typename T, int D, int W, int N>
int attn_prefix_w(const AttnParams& p, int dev, bool overlapped, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = AttnGeo<T, D, W, N>;
    static_assert(Geo::BYTES <= 227 * 1024, "shared memory");
    int rc = attn_prepare(attn_prefix_kernel<T, D, W, N>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    const long long prefix_units = static_cast<long long>(p.prefix_splits) * p.prefix_row_tiles * p.hkv;
    const long long own_units = static_cast<long long>(p.B) * p.hkv * p.own_row_tiles * p.own_splits;
    if (prefix_units > 0x0fffffffll || own_units > 0x0fffffffll) return WHT_ERR_BAD_T;
    const long long blocks = ceil_div(prefix_units * p.prefix_wpu, W) + ceil_div(own_units * p.own_wpu, W);
    CUtensorMap k_map, v_map;
    rc = cache_maps(&k_map, &v_map, p, D, attn_code<T>(), kChunk);
    if (rc != WHT_OK) return rc;
    if (overlapped)
        launch_overlapped(attn_prefix_kernel<T, D, W, N>, dim3(static_cast<unsigned>(blocks)), Geo::THREADS, Geo::BYTES, s, p, k_map, v_map);
    else
        attn_prefix_kernel<T, D, W, N><<<static_cast<unsigned>(blocks), Geo::THREADS, Geo::BYTES, s>>>(p, k_map, v_map);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

// Blocks of eight warps: where a unit has eight, and for fp32 as soon as there are more than four warps an SM (a block of four has
// two stages a warp, 128 KB, and an SM to itself: best for small calls, D = 64, 8 x 12 heads, 1000 keys 17.1 us against 20.5; with
// eight warps of one stage 64 sequences x 2048 keys of 8 heads, D = 128, take 240 us instead of 334).
template <typename T>
bool wide_blocks(const AttnParams& p, int64_t warps) {
    int dev = 0, sms = 0;
    return p.own_wpu == 8 || (sizeof(T) == 4 && device_info(&dev, &sms) == WHT_OK && warps > 4 * sms);
}

template <typename T, int D>
int attn_prefix_d(const AttnParams& p, int dev, bool overlapped, cudaStream_t s) {
    const bool one_tile = p.own_nr == 1 && (p.prefix_splits == 0 || p.prefix_nr == 1);
    const int64_t warps = static_cast<int64_t>(p.prefix_splits) * p.prefix_row_tiles * p.hkv * p.prefix_wpu +
                          static_cast<int64_t>(p.B) * p.hkv * p.own_row_tiles * p.own_splits * p.own_wpu;
    if (wide_blocks<T>(p, warps)) return one_tile ? attn_prefix_w<T, D, 8, 1>(p, dev, overlapped, s) : attn_prefix_w<T, D, 8, 4>(p, dev, overlapped, s);
    return one_tile ? attn_prefix_w<T, D, 4, 1>(p, dev, overlapped, s) : attn_prefix_w<T, D, 4, 4>(p, dev, overlapped, s);
}

template <typename T, int D, int W, int N>
int attn_chosen_w(const AttnParams& p, int dev, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = AttnGeo<T, D, W, N>;
    int rc = attn_prepare(attn_chosen_kernel<T, D, W, N>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    const long long units = static_cast<long long>(p.T) * p.hkv * p.own_row_tiles * p.own_splits;
    if (units > 0x0fffffffll) return WHT_ERR_BAD_T;
    CUtensorMap k_map, v_map;
    rc = cache_maps(&k_map, &v_map, p, D, attn_code<T>(), kChunk);
    if (rc != WHT_OK) return rc;
    launch_overlapped(attn_chosen_kernel<T, D, W, N>, dim3(static_cast<unsigned>(ceil_div(units * p.own_wpu, W))), Geo::THREADS, Geo::BYTES, s,
                      p, k_map, v_map);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int attn_chosen_d(const AttnParams& p, int dev, cudaStream_t s) {
    const int64_t warps = p.T * p.hkv * p.own_row_tiles * p.own_splits * p.own_wpu;
    if (wide_blocks<T>(p, warps)) return p.own_nr == 1 ? attn_chosen_w<T, D, 8, 1>(p, dev, s) : attn_chosen_w<T, D, 8, 4>(p, dev, s);
    return p.own_nr == 1 ? attn_chosen_w<T, D, 4, 1>(p, dev, s) : attn_chosen_w<T, D, 4, 4>(p, dev, s);
}

template <typename T, int D>
int attn_join_d(const AttnParams& p, cudaStream_t s) {
    const long long rows = static_cast<long long>(p.T) * p.hq;
    launch_overlapped(attn_join_kernel<T, D>, dim3(static_cast<unsigned>(ceil_div(rows, 4))), 128, 0, s, p.part_ml, p.part_o,
                      static_cast<T*>(p.out), static_cast<int64_t>(rows), p.parts, p.chosen ? nullptr : p.q_start, p.B, p.hq);
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

}  // namespace

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

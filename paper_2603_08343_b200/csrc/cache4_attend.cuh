// Launches of the attention over the 4-bit cache for one storage type of queries and outputs.
#pragma once
#include "cache4_attend_kernels.cuh"
#include "cache4_host.h"

namespace wht_host {

using namespace wht;

// (internal linkage: the statics below belong to this library alone, also where a process loads two builds of it)
namespace {

template <typename Kernel>
int prepare4(Kernel kernel, int smem, int dev, int* cache) {
    if (cache[dev]) return WHT_OK;
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    WHT_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared));
    cache[dev] = 1;
    return WHT_OK;
}

template <typename T, int D, int NR, int E>
int attend4(const Attn4Params& p, int dev, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = Attn4Geo<T, D, NR>;
    static_assert(Geo::BLOCKS == wht_plan::resident4(NR, Geo::F32), "the plan's blocks per SM");
    static_assert(Geo::BLOCKS * (Geo::BYTES + 1024) <= 228 * 1024, "shared memory");
    int rc = prepare4(attn4_kernel<T, D, NR, E>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    launch_overlapped(attn4_kernel<T, D, NR, E>, dim3(static_cast<unsigned>(p.warps)), 32, Geo::BYTES, s, p);
    WHT_CUDA_TRY(cudaGetLastError());
    const long long rows = static_cast<long long>(p.a.T) * p.a.hq;
    launch_overlapped(attn4_join_kernel<T, D>, dim3(static_cast<unsigned>(ceil_div(rows, 4))), 128, 0, s, p, static_cast<int>(Geo::ROWS));
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int attend4_d(const Attn4Params& p, int row_tiles, int dev, cudaStream_t s) {
    // (up to four rows a sequence and key head: see Rows4)
    if (row_tiles == 1) return p.part_rows <= 4 ? attend4<T, D, 1, 1>(p, dev, s) : attend4<T, D, 1, 2>(p, dev, s);
    return attend4<T, D, 2, 2>(p, dev, s);
}

template <typename T, int D, int NR>
int weigh4(const Attn4Params& p, bool after, int dev, cudaStream_t s) {
    static int ready[kMaxDevices] = {};
    using Geo = Weigh4Geo<T, D, NR>;
    int rc = prepare4(attn4_weigh_kernel<T, D, NR>, Geo::BYTES, dev, ready);
    if (rc != WHT_OK) return rc;
    const long long keys = static_cast<long long>(p.a.table_width) << p.a.page_shift;
    int device = 0, sms = 0, tiles = kWeightTiles;
    rc = device_info(&device, &sms);
    if (rc != WHT_OK) return rc;
    // (shorter chunks read the rows more often, but fill the machine.  us, chunks of 32 tiles alone and by this rule: 64 tokens of 4 rows over 4000 keys, 8 key
    // heads, 225 and 56; 8 sequences of up to 8 tokens of 16 rows over 16652, 2 key heads, 174 and 78; 512 tokens of 16 heads over 2000 431 and 95)
    while (tiles > 1 && ceil_div(keys, tiles * kTileKeys) * p.a.hkv * p.a.B < 12 * sms) tiles /= 2;
    const long long chunks = ceil_div(keys, tiles * kTileKeys), blocks = chunks * p.a.hkv * p.a.B;
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    if (blocks == 0) return WHT_OK;
    if (after)
        launch_overlapped(attn4_weigh_kernel<T, D, NR>, dim3(static_cast<unsigned>(blocks)), 32, Geo::BYTES, s, p, tiles, static_cast<int>(chunks));
    else
        attn4_weigh_kernel<T, D, NR><<<static_cast<unsigned>(blocks), 32, Geo::BYTES, s>>>(p, tiles, static_cast<int>(chunks));
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

int weigh4_scores(const Attn4Params& p, cudaStream_t s) {
    const long long keys = static_cast<long long>(p.a.table_width) << p.a.page_shift;
    const long long chunks = ceil_div(keys, 1024), blocks = chunks * p.a.hkv * p.a.B;
    if (blocks > 0x7fffffffll) return WHT_ERR_BAD_T;
    if (blocks == 0) return WHT_OK;
    launch_overlapped(attn4_weigh_scores_kernel, dim3(static_cast<unsigned>(blocks)), 256, 0, s, p, static_cast<int>(chunks));
    WHT_CUDA_TRY(cudaGetLastError());
    return WHT_OK;
}

template <typename T, int D>
int weigh4_d(const Attn4Params& p, bool few_rows, bool after, int dev, cudaStream_t s) {
    if constexpr (std::is_same<T, float>::value) return weigh4<T, D, 1>(p, after, dev, s);  // (two terms: registers for one tile)
    else return few_rows ? weigh4<T, D, 1>(p, after, dev, s) : weigh4<T, D, 2>(p, after, dev, s);
}

}  // namespace

template <typename T>
int launch_attend4(const Attn4Params& p, int row_tiles, int d, int dev, cudaStream_t s) {
    return d == 64 ? attend4_d<T, 64>(p, row_tiles, dev, s) : d == 96 ? attend4_d<T, 96>(p, row_tiles, dev, s) : attend4_d<T, 128>(p, row_tiles, dev, s);
}
template <typename T>
int launch_weigh4(const Attn4Params& p, bool few_rows, bool after, int d, int dev, cudaStream_t s) {
    if (p.scores != nullptr) return weigh4_scores(p, s);
    return d == 64 ? weigh4_d<T, 64>(p, few_rows, after, dev, s)
                   : d == 96 ? weigh4_d<T, 96>(p, few_rows, after, dev, s) : weigh4_d<T, 128>(p, few_rows, after, dev, s);
}

}  // namespace wht_host

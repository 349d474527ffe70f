// Host-side pieces shared by the serving-attention translation units: launch functions and the split of work.
#pragma once
#include <cuda.h>

#include "../../include/wht_attention.h"
#include "host_common.h"

namespace wht {
struct AppendParams;
struct AttnParams;
struct SelectParams;
struct UmmaAttnParams;
}  // namespace wht

namespace wht_host {

// attn_tma.cu: the caches as [num_pages * Hkv * page] rows of d channels, copied in boxes of box_rows rows by 128 bytes
int cache_maps(CUtensorMap* k_map, CUtensorMap* v_map, const wht::AttnParams& p, int d, int dtype, int box_rows);
// attn_append.cu
int launch_append(wht::AppendParams& p, int dtype, bool interleaved, cudaStream_t s);
// attn_paged.cuh, instantiated per storage type in attn_paged_bf16.cu and attn_paged_f32.cu
// overlapped: launched right after the tensor-core kernel of the prefix, to run next to it
template <typename T> int launch_attn_prefix(const wht::AttnParams& p, int d, int dev, bool overlapped, cudaStream_t s);
template <typename T> int launch_attn_chosen(const wht::AttnParams& p, int d, int dev, cudaStream_t s);
template <typename T> int launch_attn_join(const wht::AttnParams& p, int d, cudaStream_t s);
// attn_umma.cu
int launch_attn_umma_prefix(const wht::UmmaAttnParams& p, int d, int dev, cudaStream_t s);
// attn_select.cu; one_kernel: scores stay in shared memory, and p.scores is not used
int launch_select(wht::SelectParams& p, bool one_kernel, int dtype, int d, cudaStream_t s);

int take_attn_error_append(unsigned* flag);
int take_attn_error_paged_bf16(unsigned* flag);
int take_attn_error_paged_f32(unsigned* flag);
int take_attn_error_select(unsigned* flag);
int take_attn_error_umma(unsigned* flag);
// expired waits
int take_device_error_attn_umma(unsigned* flag);
int take_device_error_attn_paged_bf16(unsigned* flag);
int take_device_error_attn_paged_f32(unsigned* flag);

// Defines one of the readers above in the translation unit that includes the kernels.
#define WHT_DEFINE_ATTN_ERROR_READER(name)                                                            \
    int name(unsigned* flag) {                                                                        \
        unsigned v = 0;                                                                               \
        WHT_CUDA_TRY(cudaMemcpyFromSymbol(&v, ::wht::g_attn_device_error, sizeof(v)));                \
        if (v != 0) {                                                                                 \
            const unsigned zero = 0;                                                                  \
            WHT_CUDA_TRY(cudaMemcpyToSymbol(::wht::g_attn_device_error, &zero, sizeof(zero)));        \
        }                                                                                             \
        *flag = v;                                                                                    \
        return WHT_OK;                                                                                \
    }

}  // namespace wht_host

// Host-side pieces shared by the translation units of the 4-bit cache.
#pragma once
#include "attn_host.h"
#include "cache4_plan.h"

namespace wht {
struct Append4Params;
struct Read4Params;
struct Attn4Params;
struct Evict4Params;
}  // namespace wht

namespace wht_host {

// cache4_append.cu
int launch_append4(wht::Append4Params& p, int dtype, bool interleaved, int d, cudaStream_t s);
int launch_read4(const wht::Read4Params& p, int dtype, int d, cudaStream_t s);
// cache4_attend.cuh, instantiated per storage type in cache4_attend_bf16.cu and cache4_attend_f32.cu
template <typename T> int launch_attend4(const wht::Attn4Params& p, int row_tiles, int d, int dev, cudaStream_t s);
template <typename T> int launch_weigh4(const wht::Attn4Params& p, bool few_rows, bool after, int d, int dev, cudaStream_t s);
// cache4_umma.cu
int launch_attend4_umma(const wht::Attn4Params& p, int d, int dev, cudaStream_t s);
// cache4_evict.cu
int launch_evict4(const wht::Evict4Params& p, int d, cudaStream_t s);

int take_attn_error_append4(unsigned* flag);
int take_attn_error_attend4_bf16(unsigned* flag);
int take_attn_error_attend4_f32(unsigned* flag);
int take_attn_error_umma4(unsigned* flag);
int take_attn_error_evict4(unsigned* flag);
// expired waits
int take_device_error_attend4_bf16(unsigned* flag);
int take_device_error_attend4_f32(unsigned* flag);
int take_device_error_umma4(unsigned* flag);

}  // namespace wht_host

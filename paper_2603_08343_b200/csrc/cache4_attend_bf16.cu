// Attention over the 4-bit cache with bf16 queries and outputs.
#include "cache4_attend.cuh"

namespace wht_host {

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_attend4_bf16)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attend4_bf16)

template int launch_attend4<__nv_bfloat16>(const Attn4Params&, int, int, int, cudaStream_t);
template int launch_weigh4<__nv_bfloat16>(const Attn4Params&, bool, bool, int, int, cudaStream_t);

}  // namespace wht_host

// Attention over the 4-bit cache with fp32 queries and outputs.
#include "cache4_attend.cuh"

namespace wht_host {

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_attend4_f32)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attend4_f32)

template int launch_attend4<float>(const Attn4Params&, int, int, int, cudaStream_t);
template int launch_weigh4<float>(const Attn4Params&, bool, bool, int, int, cudaStream_t);

}  // namespace wht_host

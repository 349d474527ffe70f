// Paged attention on fp32 tensors.
#include "attn_paged.cuh"

namespace wht_host {

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_paged_f32)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attn_paged_f32)

template int launch_attn_prefix<float>(const AttnParams&, int, int, bool, cudaStream_t);
template int launch_attn_chosen<float>(const AttnParams&, int, int, cudaStream_t);
template int launch_attn_join<float>(const AttnParams&, int, cudaStream_t);

}  // namespace wht_host

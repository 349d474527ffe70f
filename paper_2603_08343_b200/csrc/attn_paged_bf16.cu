// Paged attention on bf16 tensors.
#include "attn_paged.cuh"

namespace wht_host {

WHT_DEFINE_ATTN_ERROR_READER(take_attn_error_paged_bf16)
WHT_DEFINE_DEVICE_ERROR_READER(take_device_error_attn_paged_bf16)

template int launch_attn_prefix<__nv_bfloat16>(const AttnParams&, int, int, bool, cudaStream_t);
template int launch_attn_chosen<__nv_bfloat16>(const AttnParams&, int, int, cudaStream_t);
template int launch_attn_join<__nv_bfloat16>(const AttnParams&, int, cudaStream_t);

}  // namespace wht_host

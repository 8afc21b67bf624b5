// str_kv4_attn for bf16 storage.
#include "kv4_attn.cuh"

namespace kv4_attn {
template int launch_type<__nv_bfloat16>(str_ctx *, const str_kv4_shape *, AttnArgs &, int, const float *, float *, cudaStream_t);
}  // namespace kv4_attn

// str_kv4_attn for f32 storage.
#include "kv4_attn.cuh"

namespace kv4_attn {
template int launch_type<float>(str_ctx *, const str_kv4_shape *, AttnArgs &, int, const float *, float *, cudaStream_t);
}  // namespace kv4_attn

// str_kv4_attn: argument checks, workspace and the choice of kernel (kernels in kv4_attn.cuh, built per storage type).
#include <cmath>

#include "kv4_attn.cuh"

using kv4_attn::AttnArgs;

namespace kv4_attn {
extern template int launch_type<__nv_bfloat16>(str_ctx *, const str_kv4_shape *, AttnArgs &, int, const float *, float *, cudaStream_t);
extern template int launch_type<float>(str_ctx *, const str_kv4_shape *, AttnArgs &, int, const float *, float *, cudaStream_t);
}  // namespace kv4_attn

extern "C" size_t str_kv4_attn_workspace_size(const str_kv4_shape *s, int Hq, int n_q, int want_weights) {
    if (kv4_check_shape(s) != STR_OK || Hq <= 0 || n_q <= 0 || Hq % s->Hkv != 0) return 0;
    return kv4_attn::ws_layout(s, Hq, n_q, kv4_attn::AT_MAX_GRID, want_weights != 0).bytes;
}

extern "C" int str_kv4_attn(str_ctx *ctx, const str_kv4_shape *s, int dtype, int Hq, int n_q, const void *q, const str_kv4_cache *cache,
                            const int32_t *lens, float softmax_scale, void *o, float *weight_out, void *workspace,
                            size_t workspace_bytes, void *stream) {
    if (!ctx || n_q < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (Hq <= 0 || Hq % s->Hkv != 0 || !kv4_pointers_ok(cache) || !lens || (weight_out && !cache->weight)) return STR_ERR_INVALID_ARG;
    // (fmaxf in the kernel would make a NaN scale a scale of zero)
    if (!std::isfinite(softmax_scale * kv4_attn::LOG2E)) return STR_ERR_INVALID_ARG;
    if (n_q == 0) return STR_OK;
    if (!q || !o || ((uintptr_t)q & 15)) return STR_ERR_INVALID_ARG;
    const size_t weight_bytes = (size_t)s->Bz * s->Hkv * s->cap * sizeof(float);
    if (weight_out && weight_out != cache->weight && kv4_overlap(weight_out, weight_bytes, cache->weight, weight_bytes)) return STR_ERR_INVALID_ARG;
    if ((long long)(Hq / s->Hkv) * n_q > 4096) return STR_ERR_UNSUPPORTED_SHAPE;      // columns of the join's shared memory
    if (!workspace || ((uintptr_t)workspace & 255)) return STR_ERR_INVALID_ARG;
    const kv4_attn::Ws w = kv4_attn::ws_layout(s, Hq, n_q, kv4_attn::AT_MAX_GRID, weight_out != nullptr);
    if (workspace_bytes < w.bytes) return STR_ERR_WORKSPACE_TOO_SMALL;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ATTN_FWD, stream);
    const int C = n_q * (Hq / s->Hkv), cols = kv4_attn::unit_columns(s, C);
    const int G = min(ctx->sm_count * (cols <= 8 ? 2 : 1), kv4_attn::AT_MAX_GRID);
    char *base = (char *)workspace;
    AttnArgs a = {s->Bz, s->cap, s->Hkv, Hq, n_q, ceil_div(C, cols), q, lens, softmax_scale * kv4_attn::LOG2E, *cache, o,
                  (float *)(base + w.part), (float2 *)(base + w.part_ml), weight_out ? (float *)(base + w.scores) : nullptr,
                  weight_out ? (float2 *)(base + w.stats) : nullptr, ctx->status_dev};
    cudaStream_t st = (cudaStream_t)stream;
    return dtype == STR_BF16 ? kv4_attn::launch_type<__nv_bfloat16>(ctx, s, a, G, cache->weight, weight_out, st)
                             : kv4_attn::launch_type<float>(ctx, s, a, G, cache->weight, weight_out, st);
}

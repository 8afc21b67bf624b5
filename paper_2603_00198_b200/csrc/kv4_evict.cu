// str_kv4_evict: keep the rows of a 4-bit cache that have drawn the most attention weight, and copy them to another cache.
//
// score_t = sum over the key heads of weight[b, h, t], taken in fp64 in head order and rounded to fp32 once, so that the
// order of rows does not hang on the order of a sum.  Rows behind the sequence score -inf and protected rows +inf; the
// selection itself is str_topk_select on the whole capacity (ties to the lower row, result in ascending order), which
// therefore returns the rows 0 .. len-1 first when the sequence is shorter than the budget.
// Then one gather: a row of codes is d / 2 bytes for keys and as many for values, moved as 16-byte vectors.
#include <float.h>

#include "kv4.cuh"

namespace {

constexpr int EV_THREADS = 256;

__global__ void __launch_bounds__(EV_THREADS)
kv4_evict_scores_kernel(int cap, int Hkv, int keep, int n_recent, const float *__restrict__ weight, const int32_t *__restrict__ lens,
                        const int32_t *__restrict__ n_evictable, float *__restrict__ scores, int *status) {
    const int b = blockIdx.y;
    const int len = kv4_len(lens, b, cap, status);
    // first protected row: the caller's rule, but never more protected rows than the budget holds (then the newest stay)
    int first = len - n_recent;
    if (n_evictable) first = min(first, n_evictable[b]);
    first = max(first, len - keep);
    const float *w = weight + (size_t)b * Hkv * cap;
    for (int t = blockIdx.x * EV_THREADS + threadIdx.x; t < cap; t += gridDim.x * EV_THREADS) {
        float s;
        if (t >= len) s = -INFINITY;
        else if (t >= first) s = INFINITY;
        else {
            double a = 0.0;
            for (int h = 0; h < Hkv; ++h) a += (double)w[(size_t)h * cap + t];
            s = (float)a;
            s = s != s ? -FLT_MAX : fminf(fmaxf(s, -FLT_MAX), FLT_MAX);
        }
        scores[(size_t)b * cap + t] = s;
    }
}

// Grid (row blocks, Hkv, Bz).  d / 16 lanes per row: the lower half moves keys, the upper half values.
__global__ void __launch_bounds__(EV_THREADS)
kv4_evict_gather_kernel(int cap, int cap_out, int d, int ngr, int keep, const int32_t *__restrict__ lens, int32_t *__restrict__ kept,
                        int32_t *__restrict__ lens_out, str_kv4_cache src, str_kv4_cache dst) {
    const int h = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
    const int len = min(max(lens[b], 0), cap), n = min(len, keep);
    const int lpr = d / 16, half = lpr / 2, l = threadIdx.x % lpr, rpb = EV_THREADS / lpr;
    const bool values = l >= half;
    const int u = values ? l - half : l;
    const long long base = (long long)b * Hkv + h;
    const uint4 *codes = (const uint4 *)(values ? src.v_codes : src.k_codes) + base * cap * half;
    uint4 *codes_out = (uint4 *)(values ? dst.v_codes : dst.k_codes) + base * cap_out * half;
    const uint32_t *words = (const uint32_t *)(values ? src.v_scales : src.k_scales) + base * cap * ngr;
    uint32_t *words_out = (uint32_t *)(values ? dst.v_scales : dst.k_scales) + base * cap_out * ngr;
    int32_t *list = kept + (size_t)b * keep;
    for (int j = blockIdx.x * rpb + threadIdx.x / lpr; j < n; j += gridDim.x * rpb) {
        const long long t = list[j];
        codes_out[(long long)j * half + u] = __ldg(codes + t * half + u);
        if (u < ngr) words_out[(long long)j * ngr + u] = __ldg(words + t * ngr + u);
        if (l == 0) {
            if (dst.weight) dst.weight[base * cap_out + j] = src.weight[base * cap + t];
            if (h == 0 && dst.pos) dst.pos[(long long)b * cap_out + j] = src.pos[(long long)b * cap + t];
        }
    }
    if (h == 0) {       // entries that name no row are -1; no block reads them as rows
        for (int j = n + blockIdx.x * EV_THREADS + threadIdx.x; j < keep; j += gridDim.x * EV_THREADS) list[j] = -1;
        if (blockIdx.x == 0 && threadIdx.x == 0) lens_out[b] = n;
    }
}

size_t scores_bytes(const str_kv4_shape *s) { return align_up((size_t)s->Bz * s->cap * sizeof(float), 256); }

}  // namespace

extern "C" size_t str_kv4_evict_workspace_size(const str_kv4_shape *s, int keep) {
    if (kv4_check_shape(s) != STR_OK) return 0;
    return scores_bytes(s) + str_topk_select_workspace_size(s->Bz, s->cap, keep);
}

extern "C" int str_kv4_evict(str_ctx *ctx, const str_kv4_shape *s, const str_kv4_cache *cache, const int32_t *lens, int keep,
                             int n_recent, const int32_t *n_evictable, int cap_out, const str_kv4_cache *out, int32_t *lens_out,
                             int32_t *kept_idx_out, void *workspace, size_t workspace_bytes, void *stream) {
    if (!ctx) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache) || !kv4_pointers_ok(out) || !cache->weight || !lens || !lens_out) return STR_ERR_INVALID_ARG;
    if ((out->pos && !cache->pos) || cache->k_codes == out->k_codes || cache->v_codes == out->v_codes ||
        cache->k_scales == out->k_scales || cache->v_scales == out->v_scales || cache->weight == out->weight ||
        (out->pos && cache->pos == out->pos) || lens == lens_out)
        return STR_ERR_INVALID_ARG;
    if (keep < 0 || keep > s->cap || keep > cap_out || n_recent < 0 || n_recent > keep) return STR_ERR_INVALID_ARG;
    if (cap_out % 16 != 0) return STR_ERR_UNSUPPORTED_SHAPE;
    if (keep > 0) {
        if (!kept_idx_out || !workspace || ((uintptr_t)workspace & 255)) return STR_ERR_INVALID_ARG;
        if (workspace_bytes < str_kv4_evict_workspace_size(s, keep)) return STR_ERR_WORKSPACE_TOO_SMALL;
    }
    cudaStream_t st = (cudaStream_t)stream;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    if (keep == 0) {
        STR_CUDA_OK(cudaMemsetAsync(lens_out, 0, (size_t)s->Bz * sizeof(int32_t), st));
        return STR_OK;
    }
    float *scores = (float *)workspace;
    {
        StrProfScope prof_scope(ctx, STR_CAT_TOPK, stream);
        const int nb = ceil_div(s->cap, EV_THREADS);
        kv4_evict_scores_kernel<<<dim3(nb < 1024 ? nb : 1024, s->Bz), EV_THREADS, 0, st>>>(s->cap, s->Hkv, keep, n_recent, cache->weight,
                                                                                          lens, n_evictable, scores, ctx->status_dev);
        const int lrc = str_launch_ok(ctx);
        if (lrc != STR_OK) return lrc;
    }
    const int src = str_topk_select(ctx, s->Bz, s->cap, keep, scores, kept_idx_out, (char *)workspace + scores_bytes(s),
                                    workspace_bytes - scores_bytes(s), stream);
    if (src != STR_OK) return src;
    StrProfScope prof_scope(ctx, STR_CAT_COMPACT, stream);
    const int nb = ceil_div(keep, EV_THREADS / (s->d / 16));
    kv4_evict_gather_kernel<<<dim3(nb < 2048 ? nb : 2048, s->Hkv, s->Bz), EV_THREADS, 0, st>>>(
        s->cap, cap_out, s->d, s->d / s->group, keep, lens, kept_idx_out, lens_out, *cache, *out);
    return str_launch_ok(ctx);
}

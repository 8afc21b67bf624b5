// str_kv4_attn: attention of a sequence's newest tokens over its 4-bit cache, optionally adding the attention weights that
// every cached row has drawn to a running sum (the quantity str_kv4_evict ranks by).
//
// Plain form: one CTA per (sequence, query head, token) writes the scores s = softmax_scale log2(e) q.k to the workspace,
// takes their maximum and sum, and forms o; the weights are a second kernel over the stored scores.
#include "kv4.cuh"

namespace {

constexpr int AT_THREADS = 256;

__device__ __forceinline__ float kv4_key(const uint32_t *codes, const uint32_t *words, int e, int ng, int group) {
    const uint32_t c = (codes[((e >> 3) & 3) * ng + (e >> 5)] >> (4 * (e & 7))) & 15u, w = words[e / group];
    return fmaf(kv4_scale(w), (float)c, kv4_zero(w));
}
__device__ __forceinline__ float kv4_value(const uint16_t *codes, const uint32_t *words, int e, int ng, int group) {
    const uint32_t c = ((uint32_t)codes[((e >> 2) & 7) * ng + (e >> 5)] >> (4 * (e & 3))) & 15u, w = words[e / group];
    return fmaf(kv4_scale(w), (float)c, kv4_zero(w));
}

template <typename T>
__global__ void __launch_bounds__(AT_THREADS)
kv4_attn_kernel(int cap, int Hkv, int d, int group, int Hq, int n_q, const T *__restrict__ q, const int32_t *__restrict__ lens,
                float scale_log2, str_kv4_cache cache, T *__restrict__ o, float *__restrict__ scores, float2 *__restrict__ stats, int *status) {
    __shared__ float red[AT_THREADS / 32], part[AT_THREADS];
    const int hq = blockIdx.x % Hq, i = blockIdx.x / Hq, b = blockIdx.y, h = hq / (Hq / Hkv);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, ng = d / 32, ngr = d / group;
    const int n = max(0, kv4_len(lens, b, cap, status) - n_q + i + 1);          // rows this token attends to
    const size_t row0 = ((size_t)b * Hkv + h) * cap;
    const uint32_t *kc = (const uint32_t *)cache.k_codes + row0 * (d / 8), *kw = (const uint32_t *)cache.k_scales + row0 * ngr;
    const uint16_t *vc = (const uint16_t *)cache.v_codes + row0 * (d / 4);
    const uint32_t *vw = (const uint32_t *)cache.v_scales + row0 * ngr;
    const size_t col = ((size_t)b * n_q + i) * Hq + hq;
    float *s = scores + col * cap;
    float top = -INFINITY;
    for (int t = warp; t < n; t += AT_THREADS / 32) {
        float a = 0.f;
        for (int e = lane; e < d; e += 32) a = fmaf(ldf(q + col * d + e), kv4_key(kc + (size_t)t * (d / 8), kw + (size_t)t * ngr, e, ng, group), a);
        a = warp_sum(a) * scale_log2;
        if (lane == 0) s[t] = a;
        top = fmaxf(top, a);
    }
    if (lane == 0) red[warp] = top;
    __syncthreads();
    for (int w = 0; w < AT_THREADS / 32; ++w) top = fmaxf(top, red[w]);
    __syncthreads();
    float sum = 0.f;
    for (int t = tid; t < n; t += AT_THREADS) sum += exp2f(s[t] - top);
    sum = warp_sum(sum);
    if (lane == 0) red[warp] = sum;
    __syncthreads();
    sum = 0.f;
    for (int w = 0; w < AT_THREADS / 32; ++w) sum += red[w];
    const int e = tid % d, per = AT_THREADS / d;
    float a = 0.f;
    for (int t = tid / d; t < n; t += per) a = fmaf(exp2f(s[t] - top), kv4_value(vc + (size_t)t * (d / 4), vw + (size_t)t * ngr, e, ng, group), a);
    part[tid] = a;
    __syncthreads();
    if (tid < d) {
        for (int w = 1; w < per; ++w) a += part[w * d + e];
        stf(o + col * d + e, n > 0 ? a / sum : 0.f);
    }
    if (tid == 0) stats[col] = make_float2(top, n > 0 ? 1.f / sum : 0.f);
}

__global__ void __launch_bounds__(AT_THREADS)
kv4_weights_kernel(int cap, int Hkv, int Hq, int n_q, const int32_t *__restrict__ lens, const float *__restrict__ scores,
                   const float2 *__restrict__ stats, const float *weight, float *weight_out) {
    const int h = blockIdx.y, b = blockIdx.z, R = Hq / Hkv, len = min(max(lens[b], 0), cap);
    for (int t = blockIdx.x * AT_THREADS + threadIdx.x; t < len; t += gridDim.x * AT_THREADS) {
        float a = 0.f;
        for (int i = 0; i < n_q; ++i) {
            if (t > len - n_q + i) continue;
            for (int r = 0; r < R; ++r) {
                const size_t col = ((size_t)b * n_q + i) * Hq + h * R + r;
                const float2 st = stats[col];
                a += exp2f(scores[col * cap + t] - st.x) * st.y;
            }
        }
        const size_t at = ((size_t)b * Hkv + h) * cap + t;
        weight_out[at] = weight[at] + a;
    }
}

size_t scores_bytes(const str_kv4_shape *s, int Hq, int n_q) { return align_up((size_t)s->Bz * n_q * Hq * s->cap * sizeof(float), 256); }

}  // namespace

extern "C" size_t str_kv4_attn_workspace_size(const str_kv4_shape *s, int Hq, int n_q, int want_weights) {
    (void)want_weights;
    if (kv4_check_shape(s) != STR_OK || Hq <= 0 || n_q <= 0) return 0;
    return scores_bytes(s, Hq, n_q) + align_up((size_t)s->Bz * n_q * Hq * sizeof(float2), 256);
}

extern "C" int str_kv4_attn(str_ctx *ctx, const str_kv4_shape *s, int dtype, int Hq, int n_q, const void *q, const str_kv4_cache *cache,
                            const int32_t *lens, float softmax_scale, void *o, float *weight_out, void *workspace,
                            size_t workspace_bytes, void *stream) {
    StrProfScope prof_scope(ctx, STR_CAT_ATTN_FWD, stream);
    if (!ctx || n_q < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (Hq <= 0 || Hq % s->Hkv != 0 || !kv4_pointers_ok(cache) || !lens || (weight_out && !cache->weight)) return STR_ERR_INVALID_ARG;
    if (n_q == 0) return STR_OK;
    if (!q || !o) return STR_ERR_INVALID_ARG;
    const size_t need = str_kv4_attn_workspace_size(s, Hq, n_q, weight_out != nullptr);
    if (need && (!workspace || ((uintptr_t)workspace & 255))) return STR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return STR_ERR_WORKSPACE_TOO_SMALL;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    float *scores = (float *)workspace;
    float2 *stats = (float2 *)((char *)workspace + scores_bytes(s, Hq, n_q));
    const float sl = softmax_scale * 1.4426950408889634f;
    const dim3 grid(Hq * n_q, s->Bz);
    if (dtype == STR_BF16)
        kv4_attn_kernel<<<grid, AT_THREADS, 0, st>>>(s->cap, s->Hkv, s->d, s->group, Hq, n_q, (const __nv_bfloat16 *)q, lens, sl, *cache,
                                                     (__nv_bfloat16 *)o, scores, stats, ctx->status_dev);
    else
        kv4_attn_kernel<<<grid, AT_THREADS, 0, st>>>(s->cap, s->Hkv, s->d, s->group, Hq, n_q, (const float *)q, lens, sl, *cache, (float *)o,
                                                     scores, stats, ctx->status_dev);
    if (weight_out) {
        const int nb = ceil_div(s->cap, AT_THREADS);
        kv4_weights_kernel<<<dim3(nb < 1024 ? nb : 1024, s->Hkv, s->Bz), AT_THREADS, 0, st>>>(s->cap, s->Hkv, Hq, n_q, lens, scores, stats,
                                                                                           cache->weight, weight_out);
    }
    return str_launch_ok(ctx, weight_out ? 2 : 1);
}

// str_kv4_evict: keep the rows of a 4-bit cache that have drawn the most attention weight, and copy them to another cache.
//
// score_t = sum over the key heads of weight[b, h, t], taken in fp64 in head order and rounded to fp32 once, so that the
// order of rows does not hang on the order of a sum.  Protected rows come before all others, NaN after all others, ties go to
// the lower row.
//
// Selection, up to 131072 rows a sequence: one cluster of up to 8 CTAs per sequence reads every weight once, keeps the scores'
// order-preserving integer images in registers and finds the keep-th largest in three radix passes of 11, 11 and 10 bits;
// per pass the CTAs' histograms meet through distributed shared memory after one cluster barrier.  Most selections need two
// passes.  It is bound by latency on the 8 SMs that a sequence has (8 x 32896 rows, 64 CTAs: of the 24 cycles between two instructions of a
// warp 7.6 are spent at barriers, 4.3 on loads): the weights, cluster barriers (0.6 us each) and the histograms' way
// between the SMs, which is why a bin is 16 bits.  (Eight copies of the first histogram against crowded bins: no gain.)  Longer rows: the
// scores go to the workspace and str_topk_select, which splits a row over many CTAs, selects (200000 rows to 50000, 8 heads: 90 us).
//
// Then one gather, set up while the selection runs: a row of codes is d / 2 bytes for keys and as many for values, moved as 16-byte
// vectors, four rows a thread in flight (eight cost 1 to 5 % of the call, two up to 3 %).  It waits for memory: 30 of 34 cycles between
// two instructions of a warp, DRAM at 73 % of its peak (66000 kept rows of 8 heads; 53 % for half as many).
#include <cooperative_groups.h>
#include <float.h>

#include "kv4.cuh"

namespace cg = cooperative_groups;

namespace {

constexpr int EV_THREADS = 256, EV_UNROLL = 4;
constexpr int SEL_THREADS = 1024, SEL_MAX_CTAS = 8, SEL_MAX_KPT = 16, SEL_BINS = 2048;
constexpr int SEL_MAX_ROWS = SEL_THREADS * SEL_MAX_CTAS * SEL_MAX_KPT;

// First protected row: the caller's rule, but never more protected rows than the budget holds (then the newest stay).
__device__ __forceinline__ int first_protected(int len, int keep, int n_recent, const int32_t *n_evictable, int b) {
    int first = len - n_recent;
    if (n_evictable) first = min(first, n_evictable[b]);
    return max(first, len - keep);
}
__device__ __forceinline__ float finite_score(double sum) {
    const float s = (float)sum;
    return s != s ? -FLT_MAX : fminf(fmaxf(s, -FLT_MAX), FLT_MAX);
}
// Unsigned integers in the order of the scores.
__device__ __forceinline__ uint32_t score_image(float s) {
    const uint32_t u = __float_as_uint(s);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Grid (CTAs of a cluster, Bz).  Every thread owns KPT consecutive rows.
template <int KPT>
__global__ void __launch_bounds__(SEL_THREADS)
kv4_evict_select_kernel(int cap, int Hkv, int keep, int n_recent, const float *__restrict__ weight, const int32_t *__restrict__ lens,
                        const int32_t *__restrict__ n_evictable, int32_t *__restrict__ kept, int32_t *__restrict__ lens_out, int *status) {
    constexpr int VEC = KPT < 4 ? KPT : 4;
    __shared__ uint32_t hist[3][SEL_BINS / 2];                                  // per pass, two 16-bit counts a word: a CTA has at most 16384 rows
    __shared__ uint32_t warp_a[32], warp_b[32], cta_total[2], found_prefix, found_need, found_all;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ncta = (int)cluster.num_blocks(), b = blockIdx.y;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int len = kv4_len(lens, b, cap, status), n = min(len, keep);
    int32_t *out = kept + (size_t)b * keep;
    for (int j = n + rank * SEL_THREADS + tid; j < keep; j += ncta * SEL_THREADS) out[j] = -1;
    if (rank == 0 && tid == 0) lens_out[b] = n;
    const int t0 = (rank * SEL_THREADS + tid) * KPT;
    if (len <= keep) {                                                          // all rows stay (the whole cluster takes this way)
#pragma unroll
        for (int j = 0; j < KPT; ++j)
            if (t0 + j < len) out[t0 + j] = t0 + j;
        return;
    }
    for (int i = tid; i < 3 * SEL_BINS / 2; i += SEL_THREADS) (&hist[0][0])[i] = 0u;
    const int first = first_protected(len, keep, n_recent, n_evictable, b);
    uint32_t key[KPT];
    {
        double sum[KPT];
#pragma unroll
        for (int j = 0; j < KPT; ++j) sum[j] = 0.0;
        const float *w = weight + (size_t)b * Hkv * cap + t0;
        if (t0 < min(first, cap)) {                                             // KPT divides the capacity: whole vectors are inside
#pragma unroll 4
            for (int h = 0; h < Hkv; ++h) {
                float v[KPT];
#pragma unroll
                for (int j = 0; j < KPT; j += VEC) {
                    if constexpr (VEC == 4) *(float4 *)(v + j) = __ldg((const float4 *)(w + (size_t)h * cap + j));
                    else if constexpr (VEC == 2) *(float2 *)(v + j) = __ldg((const float2 *)(w + (size_t)h * cap + j));
                    else v[j] = __ldg(w + (size_t)h * cap + j);
                }
#pragma unroll
                for (int j = 0; j < KPT; ++j) sum[j] += (double)v[j];
            }
        }
#pragma unroll
        for (int j = 0; j < KPT; ++j) key[j] = t0 + j >= first ? 0xFFFFFFFFu : score_image(finite_score(sum[j]));
    }
    uint32_t prefix = 0u, mask = 0u, need = (uint32_t)keep;
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        const uint32_t digit = pass == 2 ? 1023u : 2047u;
        uint32_t *hp = hist[pass];
#pragma unroll
        for (int j = 0; j < KPT; ++j)
            if (t0 + j < len && (key[j] & mask) == prefix) {
                const uint32_t bin = (key[j] >> shift) & digit;
                atomicAdd(&hp[bin >> 1], 1u << (16 * (bin & 1)));
            }
        cluster.sync();
        // bins from the top: thread i holds bins 2047 - 2i and 2046 - 2i of the whole cluster
        uint32_t c0 = 0u, c1 = 0u;
        uint32_t far[SEL_MAX_CTAS];
#pragma unroll
        for (int k = 0; k < SEL_MAX_CTAS; ++k)                                  // all under way before the first is used
            far[k] = k < ncta ? cluster.map_shared_rank(hp, k)[SEL_BINS / 2 - 1 - tid] : 0u;
#pragma unroll
        for (int k = 0; k < SEL_MAX_CTAS; ++k) {
            c0 += far[k] >> 16;
            c1 += far[k] & 0xFFFFu;
        }
        uint32_t incl = c0 + c1;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += v;
        }
        if (lane == 31) warp_a[warp] = incl;
        __syncthreads();
        uint32_t before = warp_a[lane];                                         // every warp adds up the warps before it
        before = __reduce_add_sync(0xffffffffu, lane < warp ? before : 0u) + incl - c0 - c1;
        if (before < need && need <= before + c0 + c1) {
            const bool low = need > before + c0;
            found_prefix = prefix | ((uint32_t)(SEL_BINS - 1 - 2 * tid - (low ? 1 : 0)) << shift);
            found_need = need - before - (low ? c0 : 0u);
            found_all = found_need == (low ? c1 : c0);
        }
        __syncthreads();
        prefix = found_prefix;
        need = found_need;
        mask |= digit << shift;
        if (found_all) break;                                                   // the whole bin stays: no need to look closer (the same in all CTAs)
    }
    // kept: images above the prefix, and the first `need` rows of those that share it
    uint32_t gt = 0u, eq = 0u;
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const bool in = t0 + j < len;
        gt += in && (key[j] & mask) > prefix;
        eq += in && (key[j] & mask) == prefix;
    }
    uint32_t g = gt, e = eq;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, g, o), y = __shfl_up_sync(0xffffffffu, e, o);
        if (lane >= o) { g += x; e += y; }
    }
    __syncthreads();                                                            // warp_a has been read
    if (lane == 31) { warp_a[warp] = g; warp_b[warp] = e; }
    __syncthreads();
    const uint32_t wg = warp_a[lane], we = warp_b[lane];
    uint32_t gt_before = __reduce_add_sync(0xffffffffu, lane < warp ? wg : 0u) + g - gt;
    uint32_t eq_before = __reduce_add_sync(0xffffffffu, lane < warp ? we : 0u) + e - eq;
    if (warp == 0) {
        const uint32_t a = __reduce_add_sync(0xffffffffu, wg), c = __reduce_add_sync(0xffffffffu, we);
        if (lane == 0) { cta_total[0] = a; cta_total[1] = c; }
    }
    cluster.sync();
    {
        const uint32_t *t = cluster.map_shared_rank(cta_total, lane < rank ? lane : rank);      // lane k: the CTA k before this one
        const uint32_t a = t[0], c = t[1];
        gt_before += __reduce_add_sync(0xffffffffu, lane < rank ? a : 0u);
        eq_before += __reduce_add_sync(0xffffffffu, lane < rank ? c : 0u);
    }
#pragma unroll
    for (int j = 0; j < KPT; ++j) {
        const bool in = t0 + j < len, above = in && (key[j] & mask) > prefix, same = in && (key[j] & mask) == prefix;
        if (above || (same && eq_before < need)) out[gt_before + min(eq_before, need)] = t0 + j;
        gt_before += above;
        eq_before += same;
    }
    cluster.sync();                                                             // no CTA leaves while another may read its shared memory
}

// Long rows: the scores for str_topk_select, -inf behind the sequence and +inf for protected rows.
__global__ void __launch_bounds__(EV_THREADS)
kv4_evict_scores_kernel(int cap, int Hkv, int keep, int n_recent, const float *__restrict__ weight, const int32_t *__restrict__ lens,
                        const int32_t *__restrict__ n_evictable, float *__restrict__ scores, int32_t *__restrict__ lens_out, int *status) {
    const int b = blockIdx.y, len = kv4_len(lens, b, cap, status), first = first_protected(len, keep, n_recent, n_evictable, b);
    const float *w = weight + (size_t)b * Hkv * cap;
    if (blockIdx.x == 0 && threadIdx.x == 0) lens_out[b] = min(len, keep);
    for (int t = blockIdx.x * EV_THREADS + threadIdx.x; t < cap; t += gridDim.x * EV_THREADS) {
        float s = t >= len ? -INFINITY : INFINITY;
        if (t < first) {
            double a = 0.0;
            for (int h = 0; h < Hkv; ++h) a += (double)w[(size_t)h * cap + t];
            s = finite_score(a);
        }
        scores[(size_t)b * cap + t] = s;
    }
}

// Grid (row blocks, Hkv, Bz).  D / 16 lanes per row: the lower half moves keys, the upper half values.  `fill`: the entries of
// `kept` that name no row are set to -1 here (no block reads them as rows).
template <int D>
__global__ void __launch_bounds__(EV_THREADS)
kv4_evict_gather_kernel(int cap, int cap_out, int ngr, int keep, bool fill, int32_t *__restrict__ kept, const int32_t *__restrict__ lens_out,
                        str_kv4_cache src, str_kv4_cache dst) {
    constexpr int LPR = D / 16, HALF = LPR / 2, RPB = EV_THREADS / LPR;
    const int h = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
    const int l = threadIdx.x % LPR, u = l % HALF, j0 = blockIdx.x * (RPB * EV_UNROLL) + threadIdx.x / LPR;
    const bool values = l >= HALF;
    const long long base = ((long long)b * Hkv + h) * cap, base_out = ((long long)b * Hkv + h) * cap_out;
    const uint4 *codes = (const uint4 *)(values ? src.v_codes : src.k_codes) + base * HALF + u;
    uint4 *codes_out = (uint4 *)(values ? dst.v_codes : dst.k_codes) + base_out * HALF + u;
    const uint32_t *words = (const uint32_t *)(values ? src.v_scales : src.k_scales) + base * ngr + u;
    uint32_t *words_out = (uint32_t *)(values ? dst.v_scales : dst.k_scales) + base_out * ngr + u;
    int32_t *list = kept + (size_t)b * keep;
    asm volatile("griddepcontrol.wait;" ::: "memory");                          // the selection's results are there
    const int n = lens_out[b];
    int t[EV_UNROLL];
    uint4 v[EV_UNROLL];
    uint32_t w[EV_UNROLL];
    float weight[EV_UNROLL];
#pragma unroll
    for (int i = 0; i < EV_UNROLL; ++i) t[i] = j0 + i * RPB < n ? list[j0 + i * RPB] : -1;
#pragma unroll
    for (int i = 0; i < EV_UNROLL; ++i)
        if (t[i] >= 0) {
            v[i] = __ldg(codes + (long long)t[i] * HALF);
            if (u < ngr) w[i] = __ldg(words + (long long)t[i] * ngr);
            if (l == 0 && dst.weight) weight[i] = __ldg(src.weight + base + t[i]);
        }
#pragma unroll
    for (int i = 0; i < EV_UNROLL; ++i)
        if (t[i] >= 0) {
            const long long j = j0 + i * RPB;
            codes_out[j * HALF] = v[i];
            if (u < ngr) words_out[j * ngr] = w[i];
            if (l == 0 && dst.weight) dst.weight[base_out + j] = weight[i];
        }
    if (h == 0) {                                                               // once per sequence: ids, and the list's end
        for (int j = blockIdx.x * (RPB * EV_UNROLL) + threadIdx.x; j < min((int)(blockIdx.x + 1) * (RPB * EV_UNROLL), keep); j += EV_THREADS) {
            if (j < n && dst.pos) dst.pos[(long long)b * cap_out + j] = src.pos[(long long)b * cap + list[j]];
            if (j >= n && fill) list[j] = -1;
        }
    }
}

template <int KPT>
cudaError_t launch_select(int ncta, const str_kv4_shape *s, int keep, int n_recent, const float *weight, const int32_t *lens, const int32_t *n_evictable,
                          int32_t *kept, int32_t *lens_out, int *status, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ncta, s->Bz, 1);
    cfg.blockDim = dim3(SEL_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ncta;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv4_evict_select_kernel<KPT>, s->cap, s->Hkv, keep, n_recent, weight, lens, n_evictable, kept, lens_out, status);
}

template <int D>
cudaError_t launch_gather(const str_kv4_shape *s, int cap_out, int keep, bool fill, int32_t *kept, const int32_t *lens_out, const str_kv4_cache &src,
                          const str_kv4_cache &dst, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(ceil_div(keep, EV_THREADS / (D / 16) * EV_UNROLL), s->Hkv, s->Bz);
    cfg.blockDim = dim3(EV_THREADS, 1, 1);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kv4_evict_gather_kernel<D>, s->cap, cap_out, s->d / s->group, keep, fill, kept, lens_out, src, dst);
}

// Does one of n written buffers share memory with one of m read ones or with another written one?
struct Buffer { const void *p; size_t bytes; };
bool any_shared(const Buffer *written, int n, const Buffer *read, int m) {
    for (int i = 0; i < n; ++i) {
        for (int j = 0; j < m; ++j)
            if (kv4_overlap(written[i].p, written[i].bytes, read[j].p, read[j].bytes)) return true;
        for (int j = 0; j < i; ++j)
            if (kv4_overlap(written[i].p, written[i].bytes, written[j].p, written[j].bytes)) return true;
    }
    return false;
}
bool long_rows(const str_kv4_shape *s) { return s->cap > SEL_MAX_ROWS; }
size_t scores_bytes(const str_kv4_shape *s) { return align_up((size_t)s->Bz * s->cap * sizeof(float), 256); }

}  // namespace

extern "C" size_t str_kv4_evict_workspace_size(const str_kv4_shape *s, int keep) {
    if (kv4_check_shape(s) != STR_OK || !long_rows(s)) return 0;
    return scores_bytes(s) + str_topk_select_workspace_size(s->Bz, s->cap, keep);
}

extern "C" int str_kv4_evict(str_ctx *ctx, const str_kv4_shape *s, const str_kv4_cache *cache, const int32_t *lens, int keep,
                             int n_recent, const int32_t *n_evictable, int cap_out, const str_kv4_cache *out, int32_t *lens_out,
                             int32_t *kept_idx_out, void *workspace, size_t workspace_bytes, void *stream) {
    if (!ctx) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache) || !kv4_pointers_ok(out) || !cache->weight || !lens || !lens_out) return STR_ERR_INVALID_ARG;
    if ((out->pos && !cache->pos) || cap_out <= 0) return STR_ERR_INVALID_ARG;
    // What is written shares no memory with what is read, nor with one another: rows are read, and counts looked at, while others are written.
    const size_t heads = (size_t)s->Bz * s->Hkv, rows = heads * s->cap, rows_out = heads * cap_out, words = s->d / s->group * 4;
    const size_t counts = (size_t)s->Bz * sizeof(int32_t);
    const Buffer read[] = {{cache->k_codes, rows * (s->d / 2)}, {cache->v_codes, rows * (s->d / 2)}, {cache->k_scales, rows * words},
                           {cache->v_scales, rows * words}, {cache->weight, rows * 4}, {cache->pos, counts * s->cap}, {lens, counts}, {n_evictable, counts}};
    const Buffer written[] = {{out->k_codes, rows_out * (s->d / 2)}, {out->v_codes, rows_out * (s->d / 2)}, {out->k_scales, rows_out * words},
                              {out->v_scales, rows_out * words}, {out->weight, rows_out * 4}, {out->pos, counts * cap_out}, {lens_out, counts},
                              {kept_idx_out, keep > 0 ? counts * keep : 0}};
    if (any_shared(written, 6, read, 6)) return STR_ERR_INVALID_ARG;            // the caches
    if (keep < 0 || keep > s->cap || keep > cap_out || n_recent < 0 || n_recent > keep) return STR_ERR_INVALID_ARG;
    if (cap_out % 16 != 0) return STR_ERR_UNSUPPORTED_SHAPE;
    const bool split = long_rows(s);
    if (keep > 0) {
        if (!kept_idx_out || (split && (!workspace || ((uintptr_t)workspace & 255)))) return STR_ERR_INVALID_ARG;
        if (workspace_bytes < str_kv4_evict_workspace_size(s, keep)) return STR_ERR_WORKSPACE_TOO_SMALL;
    }
    if (any_shared(written, 8, read, 8)) return STR_ERR_INVALID_ARG;            // and the counts and lists
    cudaStream_t st = (cudaStream_t)stream;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    if (keep == 0) {
        STR_CUDA_OK(cudaMemsetAsync(lens_out, 0, (size_t)s->Bz * sizeof(int32_t), st));
        return STR_OK;
    }
    if (split) {
        float *scores = (float *)workspace;
        {
            StrProfScope prof_scope(ctx, STR_CAT_TOPK, stream);
            kv4_evict_scores_kernel<<<dim3(1024, s->Bz), EV_THREADS, 0, st>>>(s->cap, s->Hkv, keep, n_recent, cache->weight, lens, n_evictable,
                                                                             scores, lens_out, ctx->status_dev);
            const int lrc = str_launch_ok(ctx);
            if (lrc != STR_OK) return lrc;
        }
        const int src = str_topk_select(ctx, s->Bz, s->cap, keep, scores, kept_idx_out, (char *)workspace + scores_bytes(s),
                                        workspace_bytes - scores_bytes(s), stream);
        if (src != STR_OK) return src;
    } else {
        StrProfScope prof_scope(ctx, STR_CAT_TOPK, stream);
        // Smallest cluster (power of two, at most 8 CTAs) in which a thread has `run` rows: one where all clusters fit the card at
        // once (one sequence of 4096 rows 9.5 us against 11.8 with runs of four), else four (32 sequences of 8448 rows 80 against 83).
        const int run = s->Bz * SEL_MAX_CTAS <= ctx->sm_count ? 1 : 4;
        int ncta = 1;
        while (ncta < SEL_MAX_CTAS && ncta * SEL_THREADS * run < s->cap) ncta *= 2;
        const int per_thread = ceil_div(s->cap, ncta * SEL_THREADS);
        auto launch = per_thread <= 1 ? launch_select<1> : per_thread <= 2 ? launch_select<2> : per_thread <= 4 ? launch_select<4>
                    : per_thread <= 8 ? launch_select<8> : launch_select<16>;
        if (launch(ncta, s, keep, n_recent, cache->weight, lens, n_evictable, kept_idx_out, lens_out, ctx->status_dev, st) != cudaSuccess)
            return STR_ERR_CUDA;
        ctx->launches += 1;
    }
    StrProfScope prof_scope(ctx, STR_CAT_COMPACT, stream);
    auto gather = s->d == 64 ? launch_gather<64> : launch_gather<128>;
    if (gather(s, cap_out, keep, split, kept_idx_out, lens_out, *cache, *out, st) != cudaSuccess) return STR_ERR_CUDA;
    ctx->launches += 1;
    return STR_OK;
}

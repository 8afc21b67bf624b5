// str_attn_prefill_packed: causal attention with grouped heads over packed sequences; query i of a sequence with lq queries and lk keys
// sees its keys 0 .. lk - lq + i.  The entry point, and the kernel in fp32 arithmetic: every type, head sizes up to 128.
//
// One pass over the keys with the running maximum and sum of the softmax.  The BR rows of a block are (query, head) pairs: the queries of a
// key head's group lie in one block, so that its keys and values are fetched once for all of them.  Bound by fp32 arithmetic: both products
// are formed two elements an instruction, from 16-byte pieces of shared memory (4000 rows, 12 / 4 heads of 128: 1.31 ms, 38 TFLOP/s, half of what the
// FMA pipes do; half of shared memory's bandwidth goes with it).  Unrolled so far that reads run ahead of the products (by 2 and 2: 1.36 ms).
#include <math.h>

#include "dispatch.cuh"
#include "packed.cuh"

namespace {

constexpr int MAX_ROWS = 128, BC = 64, LDP = BC + 4;

// Four columns of a row, the first `in` of which exist.
__device__ __forceinline__ float4 raw4(const float *p) { return __ldg((const float4 *)p); }
__device__ __forceinline__ float4 raw4(const __nv_bfloat16 *p) {
    const uint2 w = __ldg((const uint2 *)p);
    return make_float4(__uint_as_float(w.x << 16), __uint_as_float(w.x & 0xFFFF0000u), __uint_as_float(w.y << 16), __uint_as_float(w.y & 0xFFFF0000u));
}
template <typename T>
__device__ __forceinline__ float4 load4(const T *p, int in, bool vec) {
    if (vec && in >= 4) return raw4(p);
    return make_float4(in > 0 ? ldf(p) : 0.f, in > 1 ? ldf(p + 1) : 0.f, in > 2 ? ldf(p + 2) : 0.f, in > 3 ? ldf(p + 3) : 0.f);
}

// DP: head size padded to 64 or 128.  Thread (ty, tx) of BR/8 x 16: rows ty + BR/8 a (a < 8), keys tx + 16 j (j < 4), columns 4 tx + 64 c ...
template <typename T, int DP, int BR>
__global__ void __launch_bounds__(2 * BR)
attn_packed_simt_kernel(int n_seq, int rows_q, int rows_k, int Hq, int Hkv, int d, float scale_log2, const PackedBlockSize per, const int32_t *__restrict__ q_start,
                        const int32_t *__restrict__ k_start, const T *__restrict__ q, const T *__restrict__ k, const T *__restrict__ v, T *__restrict__ o,
                        int *status) {
    constexpr int LD = DP + 4, DC = DP / 64, THREADS = 2 * BR, RS = BR / 8;
    extern __shared__ float4 smem4[];
    float *Qs = (float *)smem4, *Ks = Qs + BR * LD, *Vs = Ks + BC * LD, *Ps = Vs + BC * DP;
    __shared__ PackedBlock blk;
    const int tid = threadIdx.x, ty = tid / 16, tx = tid % 16;
    const int kv = blockIdx.x % Hkv, group = Hq / Hkv;                   // `per` queries a block
    if (blockIdx.x == 0) {
        packed_check(q_start, n_seq, rows_q, status);
        packed_check(k_start, n_seq, rows_k, status);
    }
    if (tid < 32) {
        const PackedBlock b = packed_block(q_start, k_start, n_seq, rows_q, rows_k, per, BC, blockIdx.x / Hkv);
        if (tid == 0) blk = b;
    }
    __syncthreads();
    const PackedBlock b = blk;
    if (b.n <= 0) return;
    const int first_limit = b.lk - b.lq + b.first;                       // last key that the block's first query sees
    const int seen = max(first_limit + b.n, 0);                          // keys that its last query sees
    // Rows whose columns come in fours are read so.
    const bool vec = d % 4 == 0 && (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v) & 15) == 0;
    for (int e = tid; e < BR * (DP / 4); e += THREADS) {
        const int r = e / (DP / 4), c = e % (DP / 4) * 4, t = r / group;
        *(float4 *)(Qs + r * LD + c) = load4(q + ((size_t)(b.q0 + b.first + t) * Hq + kv * group + r % group) * d + c, t < b.n ? d - c : 0, vec);
    }
    int limit[8];
    float mx[8], sm[8];
    float2 acc[8][DC * 2];
#pragma unroll
    for (int a = 0; a < 8; ++a) {
        limit[a] = first_limit + min((ty + RS * a) / group, b.n - 1);
        mx[a] = -INFINITY;
        sm[a] = 0.f;
#pragma unroll
        for (int c = 0; c < DC * 2; ++c) acc[a][c] = make_float2(0.f, 0.f);
    }
    // fp32 rows travel to shared memory in the background, the next keys during the softmax and the second product, the next values during the first.
    const bool ahead = sizeof(T) == 4 && vec;
    auto fetch = [&](const T *from, float *to, int ld, int c0) {
#pragma unroll 4
        for (int e = tid; e < BC * (DP / 4); e += THREADS) {
            const int r = e / (DP / 4), c = e % (DP / 4) * 4;
            const bool in = c0 + r < seen && c < d;                      // the rest is filled with zeros
            const T *at = in ? from + ((size_t)(b.k0 + c0 + r) * Hkv + kv) * d + c : from;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(to + r * ld + c)), "l"(at), "r"(in ? 16 : 0) : "memory");
        }
    };
    auto sent = [&]() { asm volatile("cp.async.commit_group;" ::: "memory"); };
    auto all_but_last_here = [&]() { asm volatile("cp.async.wait_group 1;" ::: "memory"); };
    auto odd4 = [&](const float4 &x) { return !(isfinite(x.x) && isfinite(x.y) && isfinite(x.z) && isfinite(x.w)); };
    if (ahead && seen > 0) {
        fetch(k, Ks, LD, 0);
        sent();
        fetch(v, Vs, DP, 0);
        sent();
    }
    for (int c0 = 0; c0 < seen; c0 += BC) {
        // Weights of hidden keys are zero, and zero times a value that is not finite is not: a tile that some rows see in part only, with such a
        // value in it, takes the sum that leaves hidden keys out.
        const bool hides = c0 + BC - 1 > first_limit;
        bool careful = false;
        if (ahead) {
            all_but_last_here();
            __syncthreads();
        } else {
            __syncthreads();
            bool odd = false;                                            // a value that is not finite
#pragma unroll 4
            for (int e = tid; e < BC * (DP / 4); e += THREADS) {
                const int r = e / (DP / 4), c = e % (DP / 4) * 4;
                const size_t at = ((size_t)(b.k0 + c0 + r) * Hkv + kv) * d + c;
                const int in = c0 + r < seen ? d - c : 0;                // columns from c on
                const float4 kk = load4(k + at, in, vec), vv = load4(v + at, in, vec);
                *(float4 *)(Ks + r * LD + c) = kk;
                *(float4 *)(Vs + r * DP + c) = vv;
                odd |= odd4(vv);
            }
            careful = __syncthreads_or(odd && hides);
        }
        float2 s2[8][4];                                                 // even and odd columns' sums
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[a][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < DP; c += 4) {
            float4 kk[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) kk[j] = *(const float4 *)(Ks + (tx + 16 * j) * LD + c);
#pragma unroll
            for (int a = 0; a < 8; ++a) {
                const float4 qq = *(const float4 *)(Qs + (ty + RS * a) * LD + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s2[a][j] = __ffma2_rn(make_float2(qq.x, qq.y), make_float2(kk[j].x, kk[j].y), s2[a][j]);
                    s2[a][j] = __ffma2_rn(make_float2(qq.z, qq.w), make_float2(kk[j].z, kk[j].w), s2[a][j]);
                }
            }
        }
        if (ahead) {
            __syncthreads();
            if (c0 + BC < seen) fetch(k, Ks, LD, c0 + BC);
            sent();
        }
        float s[8][4];
#pragma unroll
        for (int a = 0; a < 8; ++a)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[a][j] = s2[a][j].x + s2[a][j].y;
#pragma unroll
        for (int a = 0; a < 8; ++a) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[a][j] = c0 + tx + 16 * j <= limit[a] ? s[a][j] * scale_log2 : -INFINITY;
                top = fmaxf(top, s[a][j]);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
            const float nm = fmaxf(mx[a], top), at = nm == -INFINITY ? 0.f : nm;
            const float f = exp2f(mx[a] - at);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = exp2f(s[a][j] - at);
                Ps[(ty + RS * a) * LDP + tx + 16 * j] = p;
                sum += p;
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
            sm[a] = fmaf(sm[a], f, sum);
            mx[a] = nm;
#pragma unroll
            for (int c = 0; c < DC * 2; ++c) acc[a][c] = __fmul2_rn(acc[a][c], make_float2(f, f));
        }
        __syncwarp();                                                    // a row's weights are written and read by the same half warp
        if (ahead) {
            all_but_last_here();
            bool odd = false;
            if (hides)
                for (int e = tid; e < BC * (DP / 4); e += THREADS) odd |= odd4(*(const float4 *)(Vs + 4 * e));
            careful = __syncthreads_or(odd);
        }
        if (!careful) {
#pragma unroll 8
            for (int j = 0; j < BC; j += 4) {
                float4 vv[4][DC];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < DC; ++c) vv[i][c] = *(const float4 *)(Vs + (j + i) * DP + 4 * tx + 64 * c);
#pragma unroll
                for (int a = 0; a < 8; ++a) {
                    const float4 p4 = *(const float4 *)(Ps + (ty + RS * a) * LDP + j);
                    const float p[4] = {p4.x, p4.y, p4.z, p4.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int c = 0; c < DC; ++c) {
                            acc[a][2 * c] = __ffma2_rn(make_float2(p[i], p[i]), make_float2(vv[i][c].x, vv[i][c].y), acc[a][2 * c]);
                            acc[a][2 * c + 1] = __ffma2_rn(make_float2(p[i], p[i]), make_float2(vv[i][c].z, vv[i][c].w), acc[a][2 * c + 1]);
                        }
                }
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < BC; ++j)
#pragma unroll
                for (int a = 0; a < 8; ++a)
                    if (c0 + j <= limit[a]) {
                        const float p = Ps[(ty + RS * a) * LDP + j];
#pragma unroll
                        for (int c = 0; c < DC * 2; ++c) {
                            const float *vv = Vs + j * DP + 4 * tx + 64 * (c / 2) + 2 * (c % 2);
                            acc[a][c] = __ffma2_rn(make_float2(p, p), make_float2(vv[0], vv[1]), acc[a][c]);
                        }
                    }
        }
        if (ahead) {
            __syncthreads();
            if (c0 + BC < seen) fetch(v, Vs, DP, c0 + BC);
            sent();
        }
    }
#pragma unroll
    for (int a = 0; a < 8; ++a) {
        const int r = ty + RS * a, t = r / group;
        if (t >= b.n) continue;
        const float inv = limit[a] >= 0 ? 1.0f / sm[a] : 0.f;
        T *dst = o + ((size_t)(b.q0 + b.first + t) * Hq + kv * group + r % group) * d;
#pragma unroll
        for (int c = 0; c < DC * 4; ++c) {
            const int col = 4 * tx + 64 * (c / 4) + c % 4;
            if (col < d) stf(dst + col, limit[a] >= 0 ? (c % 2 ? acc[a][c / 2].y : acc[a][c / 2].x) * inv : 0.f);
        }
    }
}

template <typename T, int DP, int BR>
int launch(str_ctx *ctx, const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const int32_t *q_start, const int32_t *k_start,
           float scale, void *o, cudaStream_t st) {
    constexpr size_t smem = sizeof(float) * ((size_t)(BR + BC) * (DP + 4) + BC * DP + BR * LDP);
    STR_CUDA_OK(cudaFuncSetAttribute(attn_packed_simt_kernel<T, DP, BR>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    const int per = BR / (s->Hq / s->Hkv);
    attn_packed_simt_kernel<T, DP, BR><<<(s->rows_q / per + s->n_seq) * s->Hkv, 2 * BR, smem, st>>>(
        s->n_seq, s->rows_q, s->rows_k, s->Hq, s->Hkv, s->d, scale * 1.4426950408889634f, PackedBlockSize(per), q_start, k_start, (const T *)q, (const T *)k, (const T *)v,
        (T *)o, ctx->status_dev);
    return str_launch_ok(ctx);
}

// Small heads: blocks of 64 rows, three of which fit an SM; blocks of 128 where a group needs them or the head is wide (one block fits, and has to
// bring its warps along), but 64 for wide heads too where blocks of 128 would not reach every SM (4 / 4 heads of 128: 1000 rows 148 us against 231,
// 4000 rows of 12 / 4 heads, 380 blocks of 128, 1466 against 1306).
template <typename T>
int dispatch(str_ctx *ctx, const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const int32_t *q_start, const int32_t *k_start,
             float scale, void *o, cudaStream_t st) {
    const int group = s->Hq / s->Hkv;
    const bool few = group <= 64 && ((long long)s->rows_q / (128 / group) + s->n_seq) * s->Hkv <= ctx->sm_count;
    if (s->d > 64 && few) return launch<T, 128, 64>(ctx, s, q, k, v, q_start, k_start, scale, o, st);
    if (s->d > 64) return launch<T, 128, 128>(ctx, s, q, k, v, q_start, k_start, scale, o, st);
    if (group > 64) return launch<T, 64, 128>(ctx, s, q, k, v, q_start, k_start, scale, o, st);
    return launch<T, 64, 64>(ctx, s, q, k, v, q_start, k_start, scale, o, st);
}

}  // namespace

extern "C" size_t str_attn_prefill_packed_workspace_size(const str_attn_packed_shape *s) {
    if (!s || s->n_seq <= 0 || s->rows_q <= 0 || s->rows_k <= 0 || s->Hq <= 0 || s->Hkv <= 0 || s->Hq % s->Hkv != 0 || s->d <= 0) return 0;
    return str_attn_packed_tc_workspace(s);
}

extern "C" int str_attn_prefill_packed(str_ctx *ctx, const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const int32_t *q_start,
                                       const int32_t *k_start, float softmax_scale, void *o, void *workspace, size_t workspace_bytes, void *stream) {
    if (!ctx || !s || !q_start) return STR_ERR_INVALID_ARG;
    if (s->n_seq <= 0 || s->rows_q < 0 || s->rows_k < 0 || s->Hq <= 0 || s->Hkv <= 0 || s->Hq % s->Hkv != 0 || s->d <= 0 ||
        (s->dtype != STR_F32 && s->dtype != STR_BF16) || !(softmax_scale > 0.f) || !isfinite(softmax_scale * 1.4426950408889634f))
        return STR_ERR_INVALID_ARG;
    if (!k_start) {
        if (s->rows_q != s->rows_k) return STR_ERR_INVALID_ARG;
        k_start = q_start;
    }
    if (s->rows_q == 0) return STR_OK;
    if (!q || !o || (s->rows_k > 0 && (!k || !v))) return STR_ERR_INVALID_ARG;
    const int group = s->Hq / s->Hkv;
    if (s->d > 128 || group > MAX_ROWS || s->n_seq > 32768 || s->rows_q > (1 << 30) || s->rows_k > (1 << 30) ||
        ((long long)s->rows_q * group + s->n_seq) * s->Hkv > INT32_MAX)
        return STR_ERR_UNSUPPORTED_SHAPE;
    const size_t es = dtype_size(s->dtype), qb = es * s->rows_q * s->Hq * s->d, kb = es * s->rows_k * s->Hkv * s->d;
    const size_t need = str_attn_prefill_packed_workspace_size(s), sb = ((size_t)s->n_seq + 1) * sizeof(int32_t);
    const struct { const void *at; size_t bytes; } in[] = {{q, qb}, {k, kb}, {v, kb}, {q_start, sb}, {k_start, sb}};
    for (const auto &i : in)
        if (kv4_overlap(i.at, i.bytes, o, qb)) return STR_ERR_INVALID_ARG;
    if (workspace_bytes < need) return STR_ERR_WORKSPACE_TOO_SMALL;
    if (need && (!workspace || ((uintptr_t)workspace & 255) != 0 || kv4_overlap(workspace, need, o, qb))) return STR_ERR_INVALID_ARG;
    for (const auto &i : in)
        if (kv4_overlap(i.at, i.bytes, workspace, need)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ATTN_FWD, stream);
    cudaStream_t st = (cudaStream_t)stream;
    if (!str_force_simt() && str_attn_packed_tc_supported(s, q, k, v, o))
        return ++ctx->tc_calls, str_attn_packed_tc(ctx, s, q, k, v, q_start, k_start, softmax_scale, o, workspace, st);
    ++ctx->fallback_calls;
    return s->dtype == STR_BF16 ? dispatch<__nv_bfloat16>(ctx, s, q, k, v, q_start, k_start, softmax_scale, o, st)
                                : dispatch<float>(ctx, s, q, k, v, q_start, k_start, softmax_scale, o, st);
}

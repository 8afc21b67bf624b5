// The 4-bit key/value cache: rows in (str_kv4_append) and rows back out (str_kv4_read).
//
// Per group of `group` elements x of a row: zero = the largest bf16 value <= min x (exact for bf16 rows), scale =
// bf16((max x - zero) / 15), code = clamp(rint((x - zero) / scale), 0, 15).  zero is rounded down so that no element lies
// below it; scale is rounded to nearest (off by at most 2^-9: the top code moves by 0.03 of a step).  Both bounds of what
// the work costs are memory: every row is read once and written once.
//
// One thread takes 8 consecutive elements of a row: 16 or 32 bytes in, one 32-bit word of codes out, the group's extremes
// by shuffles among its 4, 8 or 16 neighbours.  d / 8 neighbouring lanes share a row, so loads are whole rows.
#include "kv4.cuh"

namespace {

constexpr int KV4_THREADS = 256;

__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *(const uint32_t *)&h;
    }
    *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    ((float4 *)p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    ((float4 *)p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}

// Codes of this thread's 8 elements (nibble j = element j) and the group's word.  All lanes of the warp take part.
template <int GROUP>
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], uint32_t &word) {
    float lo = x[0], hi = x[0], poison = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
        poison += x[j] * 0.f;                       // NaN where an element is not finite: the extremes alone drop NaN
    }
#pragma unroll
    for (int o = 1; o < GROUP / 8; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        poison += __shfl_xor_sync(0xffffffffu, poison, o);
    }
    const float zero = __bfloat162float(__float2bfloat16_rd(lo));
    const float scale = __bfloat162float(__float2bfloat16_rn((hi - zero) / 15.0f));
    if (!(poison == 0.f) || !(scale <= 3.4e38f)) {  // a NaN or infinity in the group, or extremes too far apart
        word = 0x7FFF0000u;                         // NaN scale: the whole group reads back as NaN
        return 0u;
    }
    word = (__float_as_uint(scale) & 0xFFFF0000u) | (__float_as_uint(zero) >> 16);
    uint32_t codes = 0u;
    if (scale > 0.f) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            codes |= (uint32_t)fminf(fmaxf(rintf((x[j] - zero) / scale), 0.f), 15.f) << (4 * j);
    }
    return codes;
}

// Where this thread's 8 elements sit in a row: lane `l` of the row's D / 8 covers elements 8 l .. 8 l + 7 (g = l / 4, c = l % 4).
// Keys: they are word c * NG + g.  Values: they are the 16-bit words r = 2c and 2c + 1 of run g; the row's lanes exchange
// halves so that each ends up with one whole 32-bit word of the stored order.
template <int D>
__device__ __forceinline__ uint32_t value_word(uint32_t codes, int l) {
    constexpr int NG = D / 32;
    const int p0 = 2 * l, p1 = p0 + 1;                                  // 16-bit words of stored word l
    const int r0 = p0 / NG, g0 = p0 % NG, r1 = p1 / NG, g1 = p1 % NG;
    const uint32_t a = __shfl_sync(0xffffffffu, codes, g0 * 4 + (r0 >> 1), D / 8);
    const uint32_t b = __shfl_sync(0xffffffffu, codes, g1 * 4 + (r1 >> 1), D / 8);
    return ((a >> (16 * (r0 & 1))) & 0xFFFFu) | ((b >> (16 * (r1 & 1))) << 16);
}

template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_append_kernel(int Bz, int cap, int Hkv, int T_new, const T *__restrict__ k, const T *__restrict__ v,
                  const int32_t *__restrict__ positions, const int32_t *__restrict__ row_start, const int32_t *__restrict__ n_new,
                  str_kv4_cache cache, int *status) {
    constexpr int LPR = D / 8, RPW = 32 / LPR, NG = D / 32;
    const int lane = threadIdx.x & 31, l = lane % LPR, g = l >> 2, c = l & 3;
    const long long rows = (long long)Bz * T_new * Hkv;
    const long long warps = (long long)gridDim.x * (KV4_THREADS / 32);
    // the loop bound is the same for all lanes of a warp: shuffles below need all of them
    for (long long r0 = ((long long)blockIdx.x * (KV4_THREADS / 32) + (threadIdx.x >> 5)) * RPW; r0 < rows; r0 += warps * RPW) {
        const long long r = r0 + lane / LPR;
        bool live = r < rows;
        const int h = live ? (int)(r % Hkv) : 0;
        const long long bt = live ? r / Hkv : 0;
        const int b = (int)(bt / T_new), t = (int)(bt % T_new);
        if (live && n_new) live = t < n_new[b];
        const long long row = live ? (long long)row_start[b] + t : 0;
        if (live && (row < 0 || row >= cap)) {
            atomicCAS(status, 0, STR_ERR_INVALID_ARG);
            live = false;
        }
        float xk[8], xv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) xk[j] = xv[j] = 0.f;
        if (live) {
            kv4_load8(k + r * D + 8 * l, xk);
            kv4_load8(v + r * D + 8 * l, xv);
        }
        uint32_t wk, wv;
        const uint32_t ck = quantise8<GROUP>(xk, wk);
        const uint32_t cv = value_word<D>(quantise8<GROUP>(xv, wv), l);
        if (!live) continue;
        const long long at = ((long long)b * Hkv + h) * cap + row;
        ((uint32_t *)cache.k_codes)[at * LPR + c * NG + g] = ck;
        ((uint32_t *)cache.v_codes)[at * LPR + l] = cv;
        if (l % (GROUP / 8) == 0) {
            ((uint32_t *)cache.k_scales)[at * (D / GROUP) + l / (GROUP / 8)] = wk;
            ((uint32_t *)cache.v_scales)[at * (D / GROUP) + l / (GROUP / 8)] = wv;
        }
        if (l == 0) {
            if (cache.weight) cache.weight[at] = 0.f;
            if (h == 0 && cache.pos && positions) cache.pos[(long long)b * cap + row] = positions[bt];
        }
    }
}

template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(int Bz, int cap, int Hkv, int n_out, const int32_t *__restrict__ row_start, const int32_t *__restrict__ n_rows,
                str_kv4_cache cache, T *__restrict__ k_out, T *__restrict__ v_out, int *status) {
    constexpr int LPR = D / 8, NG = D / 32;
    const long long items = (long long)Bz * n_out * Hkv * LPR;
    for (long long i = (long long)blockIdx.x * KV4_THREADS + threadIdx.x; i < items; i += (long long)gridDim.x * KV4_THREADS) {
        const int l = (int)(i % LPR), g = l >> 2, c = l & 3;
        const long long r = i / LPR, bt = r / Hkv;
        const int h = (int)(r % Hkv), b = (int)(bt / n_out), t = (int)(bt % n_out);
        float xk[8], xv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) xk[j] = xv[j] = 0.f;
        if (!n_rows || t < n_rows[b]) {
            const long long row = (long long)row_start[b] + t;
            if (row < 0 || row >= cap) {
                atomicCAS(status, 0, STR_ERR_INVALID_ARG);
            } else {
                const long long at = ((long long)b * Hkv + h) * cap + row;
                const uint32_t ck = __ldg((const uint32_t *)cache.k_codes + at * LPR + c * NG + g);
                const uint16_t *hv = (const uint16_t *)cache.v_codes + at * (2 * LPR);
                const uint32_t cv = (uint32_t)__ldg(hv + 2 * c * NG + g) | ((uint32_t)__ldg(hv + (2 * c + 1) * NG + g) << 16);
                const uint32_t wk = __ldg((const uint32_t *)cache.k_scales + at * (D / GROUP) + l / (GROUP / 8));
                const uint32_t wv = __ldg((const uint32_t *)cache.v_scales + at * (D / GROUP) + l / (GROUP / 8));
#pragma unroll
                for (int j = 0; j < 8; ++j) {       // one rounding in fp32, then the storage type's
                    xk[j] = fmaf(kv4_scale(wk), (float)((ck >> (4 * j)) & 15u), kv4_zero(wk));
                    xv[j] = fmaf(kv4_scale(wv), (float)((cv >> (4 * j)) & 15u), kv4_zero(wv));
                }
            }
        }
        store8(k_out + i * 8, xk);
        store8(v_out + i * 8, xv);
    }
}

int grid_for(const str_ctx *ctx, long long threads) {
    const long long want = (threads + KV4_THREADS - 1) / KV4_THREADS, most = (long long)ctx->sm_count * 8;
    return (int)(want < 1 ? 1 : want < most ? want : most);
}

// Calls f(type tag, d, group) as template arguments; the shape has been checked.
#define KV4_DISPATCH(dtype, s, CALL)                                                     \
    do {                                                                                 \
        if ((dtype) == STR_BF16) { KV4_DISPATCH_SHAPE(__nv_bfloat16, s, CALL); }         \
        else { KV4_DISPATCH_SHAPE(float, s, CALL); }                                     \
    } while (0)
#define KV4_DISPATCH_SHAPE(T, s, CALL)                                                   \
    do {                                                                                 \
        if ((s)->d == 64 && (s)->group == 32) CALL(T, 64, 32);                           \
        else if ((s)->d == 64) CALL(T, 64, 64);                                          \
        else if ((s)->group == 32) CALL(T, 128, 32);                                     \
        else if ((s)->group == 64) CALL(T, 128, 64);                                     \
        else CALL(T, 128, 128);                                                          \
    } while (0)

}  // namespace

extern "C" int str_kv4_append(str_ctx *ctx, const str_kv4_shape *s, int dtype, int T_new, const void *k, const void *v,
                              const int32_t *positions, const int32_t *row_start, const int32_t *n_new,
                              const str_kv4_cache *cache, void *stream) {
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    if (!ctx || T_new < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache)) return STR_ERR_INVALID_ARG;
    if (T_new == 0) return STR_OK;
    if (!k || !v || !row_start || (((uintptr_t)k | (uintptr_t)v) & 15)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    const int grid = grid_for(ctx, (long long)s->Bz * T_new * s->Hkv * (s->d / 8));
#define KV4_CALL(T, D, G)                                                                                              \
    kv4_append_kernel<T, D, G><<<grid, KV4_THREADS, 0, (cudaStream_t)stream>>>(s->Bz, s->cap, s->Hkv, T_new, (const T *)k, \
                                                                               (const T *)v, positions, row_start, n_new, *cache, ctx->status_dev)
    KV4_DISPATCH(dtype, s, KV4_CALL);
#undef KV4_CALL
    return str_launch_ok(ctx);
}

extern "C" int str_kv4_read(str_ctx *ctx, const str_kv4_shape *s, int dtype, int n_out, const int32_t *row_start,
                            const int32_t *n_rows, const str_kv4_cache *cache, void *k_out, void *v_out, void *stream) {
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    if (!ctx || n_out < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache)) return STR_ERR_INVALID_ARG;
    if (n_out == 0) return STR_OK;
    if (!k_out || !v_out || !row_start || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    const int grid = grid_for(ctx, (long long)s->Bz * n_out * s->Hkv * (s->d / 8));
#define KV4_CALL(T, D, G)                                                                                              \
    kv4_read_kernel<T, D, G><<<grid, KV4_THREADS, 0, (cudaStream_t)stream>>>(s->Bz, s->cap, s->Hkv, n_out, row_start, n_rows, \
                                                                             *cache, (T *)k_out, (T *)v_out, ctx->status_dev)
    KV4_DISPATCH(dtype, s, KV4_CALL);
#undef KV4_CALL
    return str_launch_ok(ctx);
}

// The 4-bit key/value cache: rows in (str_kv4_append) and rows back out (str_kv4_read).
//
// Per group of `group` elements x of a row: zero = the largest bf16 value <= min x (exact for bf16 rows), scale =
// bf16((max x - zero) * (1/15)), code = clamp(rint((x - zero) / scale), 0, 15).  zero is rounded down so that no element lies
// below it; scale is rounded to nearest (off by at most 2^-9: the top code moves by 0.03 of a step).  Both bounds of what
// the work costs are memory: every row is read once and written once.
//
// One thread takes 8 consecutive elements of a row: 16 or 32 bytes in, one 32-bit word of codes out, the group's extremes
// by shuffles among its 4, 8 or 16 neighbours; d / 8 neighbouring lanes share a row.  A block works on consecutive tokens of one
// head, so that the cache's rows, which lie head by head, are written and read as whole lines, and every thread has all the
// loads of its KV4_UNROLL tokens in flight before it uses the first.
#include "kv4.cuh"

namespace {

constexpr int KV4_THREADS = 128, KV4_UNROLL = 4;

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

__device__ __forceinline__ uint64_t both(float lo, float hi) { return (uint64_t)__float_as_uint(hi) << 32 | __float_as_uint(lo); }
__device__ __forceinline__ uint64_t twice(float v) { return both(v, v); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

// Extremes of a group, whose elements lie on GROUP / 8 neighbouring lanes, and whether all of them are finite (NaN or infinity
// would otherwise be lost among the extremes).  bf16 is compared two at a time: (max of -x, max of x) in one register.
template <int GROUP>
__device__ __forceinline__ void group_extremes(const Kv4Raw8<__nv_bfloat16> &raw, float &lo, float &hi, bool &finite) {
    const uint32_t w[4] = {raw.u.x, raw.u.y, raw.u.z, raw.u.w};
    const __nv_bfloat162 *p = (const __nv_bfloat162 *)w;
    const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(p[0], p[1]), __hmin2_nan(p[2], p[3]));
    const __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
    __nv_bfloat162 both = __halves2bfloat162(__hneg(__hmin_nan(__low2bfloat16(mn), __high2bfloat16(mn))),
                                             __hmax_nan(__low2bfloat16(mx), __high2bfloat16(mx)));
#pragma unroll
    for (int o = 1; o < GROUP / 8; o <<= 1) {
        const uint32_t other = __shfl_xor_sync(0xffffffffu, *(const uint32_t *)&both, o);
        both = __hmax2_nan(both, *(const __nv_bfloat162 *)&other);
    }
    lo = -__low2float(both);
    hi = __high2float(both);
    finite = lo > -INFINITY && hi < INFINITY;       // NaN has gone into both
}
template <int GROUP>
__device__ __forceinline__ void group_extremes(const Kv4Raw8<float> &raw, float &lo, float &hi, bool &finite) {
    float x[8], poison = 0.f;
    kv4_widen8(raw, x);
    lo = hi = x[0];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        lo = fminf(lo, x[j]);
        hi = fmaxf(hi, x[j]);
        poison = fmaf(x[j], 0.f, poison);           // NaN where an element is not finite
    }
#pragma unroll
    for (int o = 1; o < GROUP / 8; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
        poison += __shfl_xor_sync(0xffffffffu, poison, o);
    }
    finite = poison == 0.f;
}

// Codes of this thread's 8 elements (nibble j = element j) and the group's word.  All lanes of the warp take part.
//
// The quotient (x - zero) / scale is Markstein's: with y the correctly rounded reciprocal, q0 = t y and q = q0 + (t - q0 scale) y,
// both fused, is the correctly rounded quotient (P. Markstein, IBM J. Res. Dev. 34, 1990); adding 1.5 2^23 then rounds it to an
// integer, ties to even, in the low bits.  Scales so small or large that the reciprocal is not normal, and those so small that
// their own rounding is coarse, are divided by; both ways give the same codes.
template <int GROUP, typename T>
__device__ __forceinline__ uint32_t quantise8(const Kv4Raw8<T> &raw, uint32_t &word) {
    float lo, hi, x[8];
    bool finite;
    group_extremes<GROUP>(raw, lo, hi, finite);
    kv4_widen8(raw, x);
    const float zero = __bfloat162float(__float2bfloat16_rd(lo));
    const float scale = __bfloat162float(__float2bfloat16_rn((hi - zero) * (1.f / 15.f)));
    if (!finite || !(scale <= 3.4e38f)) {  // a NaN or infinity in the group, or extremes too far apart
        word = 0x7FFF0000u;                         // NaN scale: the whole group reads back as NaN
        return 0u;
    }
    word = (__float_as_uint(scale) & 0xFFFF0000u) | (__float_as_uint(zero) >> 16);
    uint32_t codes = 0u;
    const float inv = 1.f / scale;
    const uint64_t inv2 = twice(inv), scale2 = twice(-scale), zero2 = twice(-zero), magic2 = twice(12582912.f);
#pragma unroll
    for (int j = 6; j >= 0; j -= 2) {               // two at a time in the packed fp32 instructions
        const uint64_t t = add2(both(x[j], x[j + 1]), zero2), q0 = mul2(t, inv2);
        const uint64_t v = add2(fma2(fma2(q0, scale2, t), inv2, q0), magic2);   // 0x4B400000 + code: the constant is taken off below
        codes = codes * 256u + (uint32_t)(v >> 32) * 16u + (uint32_t)v;
    }
    codes -= 0x3F400000u;                           // sum over j of 0x4B400000 16^j, modulo 2^32
    if (!(scale > 1e-30f && scale < 1e37f)) {
        codes = 0u;
        if (scale > 0.f) {
#pragma unroll 1
            for (int j = 0; j < 8; ++j) {
                float t = x[0];
#pragma unroll
                for (int k = 1; k < 8; ++k) t = j == k ? x[k] : t;
                codes |= (uint32_t)fminf(fmaxf(rintf((t - zero) / scale), 0.f), 15.f) << (4 * j);
            }
        }
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

// Grid (token blocks, Hkv, Bz).
template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_append_kernel(int cap, int T_new, const T *__restrict__ k, const T *__restrict__ v, const int32_t *__restrict__ positions,
                  const int32_t *__restrict__ row_start, const int32_t *__restrict__ n_new, str_kv4_cache cache, int *status) {
    constexpr int LPR = D / 8, NG = D / 32, ROWS = KV4_THREADS / LPR;
    const int h = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
    const int l = threadIdx.x % LPR, g = l >> 2, c = l & 3;
    const int n = n_new ? min(n_new[b], T_new) : T_new, start = row_start[b];
    const long long src = ((long long)b * T_new * Hkv + h) * D + 8 * l, dst = ((long long)b * Hkv + h) * cap;
    const int t0 = blockIdx.x * (ROWS * KV4_UNROLL) + threadIdx.x / LPR;
    Kv4Raw8<T> rk[KV4_UNROLL], rv[KV4_UNROLL];                                  // as stored: widened only when their turn comes
    bool live[KV4_UNROLL];
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        const int t = t0 + i * ROWS;
        live[i] = t < n;
        if (live[i] && ((long long)start + t < 0 || (long long)start + t >= cap)) {
            kv4_report(status);
            live[i] = false;
        }
        rk[i] = rv[i] = {};
        if (live[i]) {
            rk[i] = kv4_raw8(k + src + (long long)t * Hkv * D);
            rv[i] = kv4_raw8(v + src + (long long)t * Hkv * D);
        }
    }
    const long long at = dst + start + t0;                                      // the first token's row; only live ones are stored
    uint32_t *kc = (uint32_t *)cache.k_codes + at * LPR + c * NG + g, *vc = (uint32_t *)cache.v_codes + at * LPR + l;
    uint32_t *ks = (uint32_t *)cache.k_scales + at * (D / GROUP) + l / (GROUP / 8), *vs = (uint32_t *)cache.v_scales + at * (D / GROUP) + l / (GROUP / 8);
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        if (!__any_sync(0xffffffffu, live[i])) continue;                        // the lanes of a warp stay together: shuffles
        uint32_t wk, wv;
        const uint32_t ck = quantise8<GROUP>(rk[i], wk);
        const uint32_t cv = value_word<D>(quantise8<GROUP>(rv[i], wv), l);
        if (!live[i]) continue;
        const int t = t0 + i * ROWS;
        kc[i * (ROWS * LPR)] = ck;
        vc[i * (ROWS * LPR)] = cv;
        if (l % (GROUP / 8) == 0) {
            ks[i * (ROWS * (D / GROUP))] = wk;
            vs[i * (ROWS * (D / GROUP))] = wv;
        }
        if (l == 0) {
            if (cache.weight) cache.weight[at + i * ROWS] = 0.f;
            if (h == 0 && cache.pos && positions) cache.pos[(long long)b * cap + start + t] = positions[(long long)b * T_new + t];
        }
    }
}

// Grid (token blocks, Hkv, Bz).
template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(int cap, int n_out, const int32_t *__restrict__ row_start, const int32_t *__restrict__ n_rows, str_kv4_cache cache,
                T *__restrict__ k_out, T *__restrict__ v_out, int *status) {
    constexpr int LPR = D / 8, NG = D / 32, ROWS = KV4_THREADS / LPR;
    const int h = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
    const int l = threadIdx.x % LPR, g = l >> 2, c = l & 3;
    const int n = n_rows ? n_rows[b] : n_out, start = row_start[b];
    const long long base = ((long long)b * Hkv + h) * cap, out = ((long long)b * n_out * Hkv + h) * D + 8 * l;
    const int t0 = blockIdx.x * (ROWS * KV4_UNROLL) + threadIdx.x / LPR;
    uint32_t ck[KV4_UNROLL], cv[KV4_UNROLL], wk[KV4_UNROLL], wv[KV4_UNROLL];
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        const int t = t0 + i * ROWS;
        const long long row = (long long)start + t;
        ck[i] = cv[i] = wk[i] = wv[i] = 0u;                                     // reads as zero
        if (t >= n_out || t >= n) continue;
        if (row < 0 || row >= cap) {
            kv4_report(status);
            continue;
        }
        const long long at = base + row;
        const uint16_t *hv = (const uint16_t *)cache.v_codes + at * (2 * LPR);
        ck[i] = __ldg((const uint32_t *)cache.k_codes + at * LPR + c * NG + g);
        cv[i] = (uint32_t)__ldg(hv + 2 * c * NG + g) | ((uint32_t)__ldg(hv + (2 * c + 1) * NG + g) << 16);
        wk[i] = __ldg((const uint32_t *)cache.k_scales + at * (D / GROUP) + l / (GROUP / 8));
        wv[i] = __ldg((const uint32_t *)cache.v_scales + at * (D / GROUP) + l / (GROUP / 8));
    }
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        const int t = t0 + i * ROWS;
        if (t >= n_out) break;
        float xk[8], xv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {               // a code as the low bits of 2^23, less 2^23; one rounding in fp32, then the storage type's
            const float yk = __uint_as_float(((ck[i] >> (4 * j)) & 15u) | 0x4B000000u) - 8388608.f;
            const float yv = __uint_as_float(((cv[i] >> (4 * j)) & 15u) | 0x4B000000u) - 8388608.f;
            xk[j] = fmaf(kv4_scale(wk[i]), yk, kv4_zero(wk[i]));
            xv[j] = fmaf(kv4_scale(wv[i]), yv, kv4_zero(wv[i]));
        }
        store8(k_out + out + (long long)t * Hkv * D, xk);
        store8(v_out + out + (long long)t * Hkv * D, xv);
    }
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
    const dim3 grid(ceil_div(T_new, KV4_THREADS / (s->d / 8) * KV4_UNROLL), s->Hkv, s->Bz);
#define KV4_CALL(T, D, G)                                                                                              \
    kv4_append_kernel<T, D, G><<<grid, KV4_THREADS, 0, (cudaStream_t)stream>>>(s->cap, T_new, (const T *)k, (const T *)v, positions, \
                                                                               row_start, n_new, *cache, ctx->status_dev)
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
    const dim3 grid(ceil_div(n_out, KV4_THREADS / (s->d / 8) * KV4_UNROLL), s->Hkv, s->Bz);
#define KV4_CALL(T, D, G)                                                                                              \
    kv4_read_kernel<T, D, G><<<grid, KV4_THREADS, 0, (cudaStream_t)stream>>>(s->cap, n_out, row_start, n_rows, *cache, \
                                                                             (T *)k_out, (T *)v_out, ctx->status_dev)
    KV4_DISPATCH(dtype, s, KV4_CALL);
#undef KV4_CALL
    return str_launch_ok(ctx);
}

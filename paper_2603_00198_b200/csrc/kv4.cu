// The 4-bit key/value cache: rows in (str_kv4_append) and rows back out (str_kv4_read).
//
// Per group of `group` elements x of a row: zero = the largest bf16 value <= min x (exact for bf16 rows), scale =
// bf16((max x - zero) * (1/15)), code = clamp(rint((x - zero) / scale), 0, 15).  zero is rounded down so that no element lies
// below it; scale is rounded to nearest (off by at most 2^-9: the top code moves by 0.03 of a step).
//
// One thread takes 8 consecutive elements of a row: 16 or 32 bytes in, one 32-bit word of codes out, the group's extremes
// from its 4, 8 or 16 neighbours; d / 8 neighbouring lanes share a row.  A block works on consecutive tokens of one
// head, so that the cache's rows, which lie head by head, are written and read as whole lines, and every thread has all the
// loads of its KV4_UNROLL tokens in flight before it uses the first.
//
// Every row is read once and written once, so memory is the floor; the bf16 forms are held up by instruction issue (74 and 70 % of the
// slots busy, DRAM at 35 and 22 % of its peak, the rest in L2).  16512 rows, 8 heads of 128, group 32, back to back: append of
// bf16 20.9 us (4.2 TB/s), of fp32 26.0 (6.0); read as bf16 15.3 (5.8), as fp32 29.5 (5.3).  Two tokens a thread, for more warps an
// SM: with four, 25.0 and 34.4, 19.0 and 39.2 in the steps' first form; with one, 30.5 and 32.9.
#include "kv4.cuh"

namespace {

constexpr int KV4_THREADS = 128, KV4_UNROLL = 2;

__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float (&x)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *(const uint32_t *)&h;
    }
    *(uint4 *)p = make_uint4(w[0], w[1], w[2], w[3]);
}
// 32 bytes a lane in one store where the address allows it: a warp then writes whole lines (29 us for the fp32 read above; two
// 16-byte stores, each half of every 32-byte sector, 37).
__device__ __forceinline__ void store8(float *p, const float (&x)[8]) {
    if (((uintptr_t)p & 31) == 0) {
        asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]),
                     "f"(x[6]), "f"(x[7])
                     : "memory");
        return;
    }
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

// Extremes of some elements: the maxima of -x and of x, so that both are found with one operation.  NaN among the elements goes
// into both (fmaxf would lose it).  For bf16 rows the pair is one register: (max of -x, max of x).
template <typename T> struct Extremes;
template <> struct Extremes<__nv_bfloat16> {
    __nv_bfloat162 e;
    __device__ __forceinline__ static Extremes of(const Kv4Raw8<__nv_bfloat16> &raw) {
        const uint32_t w[4] = {raw.u.x, raw.u.y, raw.u.z, raw.u.w};
        const __nv_bfloat162 *p = (const __nv_bfloat162 *)w;
        const __nv_bfloat162 mn = __hmin2_nan(__hmin2_nan(p[0], p[1]), __hmin2_nan(p[2], p[3]));
        const __nv_bfloat162 mx = __hmax2_nan(__hmax2_nan(p[0], p[1]), __hmax2_nan(p[2], p[3]));
        return {__halves2bfloat162(__hneg(__hmin_nan(__low2bfloat16(mn), __high2bfloat16(mn))), __hmax_nan(__low2bfloat16(mx), __high2bfloat16(mx)))};
    }
    __device__ __forceinline__ Extremes from_lane(int o) const {                // what lane ^ o holds here
        const uint32_t other = __shfl_xor_sync(0xffffffffu, *(const uint32_t *)&e, o);
        return {*(const __nv_bfloat162 *)&other};
    }
    __device__ __forceinline__ Extremes merged(const Extremes &x) const { return {__hmax2_nan(e, x.e)}; }
    __device__ __forceinline__ float lo() const { return -__low2float(e); }
    __device__ __forceinline__ float hi() const { return __high2float(e); }
};
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <> struct Extremes<float> {
    float neg, pos;
    __device__ __forceinline__ static Extremes of(const Kv4Raw8<float> &raw) {
        float x[8];
        kv4_widen8(raw, x);
        Extremes r = {-x[0], x[0]};
#pragma unroll
        for (int j = 1; j < 8; ++j) r = r.merged({-x[j], x[j]});
        return r;
    }
    __device__ __forceinline__ Extremes from_lane(int o) const {
        return {__shfl_xor_sync(0xffffffffu, neg, o), __shfl_xor_sync(0xffffffffu, pos, o)};
    }
    __device__ __forceinline__ Extremes merged(const Extremes &x) const { return {max_nan(neg, x.neg), max_nan(pos, x.pos)}; }
    __device__ __forceinline__ float lo() const { return -neg; }
    __device__ __forceinline__ float hi() const { return pos; }
};

// The groups of the N pieces (8 elements each) that every thread holds; piece j of L = GROUP / 8 neighbouring lanes is one group.
// The extremes are reduced and scattered: in step s the lanes with bit s set keep the odd pieces and the others the even ones, so
// that lane m ends up with group m % N, after three shuffles instead of eight (L = 4), and works the word out for that one
// alone; the lanes then ask one another for the word and the reciprocal scale of a piece.  Against every lane doing so for every
// group: 1 to 5 % of the append's time for bf16, 5 to 9 % for fp32.
template <int GROUP>
struct Groups {
    static constexpr int N = 2 * KV4_UNROLL, L = GROUP / 8;
    static_assert(N == 4 && L >= N, "two steps leave one group a lane");
    uint32_t mine;
    float mine_inv;
    // of piece j, which all lanes ask for together
    __device__ __forceinline__ uint32_t word(int j) const { return __shfl_sync(0xffffffffu, mine, j, L); }
    __device__ __forceinline__ float inv(int j) const { return __shfl_sync(0xffffffffu, mine_inv, j, L); }

    template <typename T>
    __device__ __forceinline__ explicit Groups(const Kv4Raw8<T> (&raw)[N]) {
        Extremes<T> e[N];
#pragma unroll
        for (int j = 0; j < N; ++j) e[j] = Extremes<T>::of(raw[j]);
#pragma unroll
        for (int o = 1, n = N / 2; n >= 1; o <<= 1, n /= 2) {
            const bool odd = threadIdx.x & o;
#pragma unroll
            for (int j = 0; j < n; ++j) {
                const Extremes<T> keep = odd ? e[2 * j + 1] : e[2 * j], send = odd ? e[2 * j] : e[2 * j + 1];
                e[j] = keep.merged(send.from_lane(o));
            }
        }
#pragma unroll
        for (int o = N; o < L; o <<= 1) e[0] = e[0].merged(e[0].from_lane(o));  // L = 8, 16: two, four lanes hold each group
        const float lo = e[0].lo(), hi = e[0].hi();
        const float zero = __bfloat162float(__float2bfloat16_rd(lo));
        const float scale = __bfloat162float(__float2bfloat16_rn((hi - zero) * (1.f / 15.f)));
        // a NaN or infinity in the group, or extremes too far apart: NaN scale, the whole group reads back as NaN
        const bool ok = lo > -INFINITY && hi < INFINITY && scale <= 3.4e38f;
        mine = ok ? (__float_as_uint(scale) & 0xFFFF0000u) | (__float_as_uint(zero) >> 16) : 0x7FFF0000u;
        mine_inv = 1.f / scale;
    }
};

// Codes of this thread's 8 elements (nibble j = element j), with the group's word and the reciprocal of its scale.
//
// The quotient (x - zero) / scale is Markstein's: with y the correctly rounded reciprocal, q0 = t y and q = q0 + (t - q0 scale) y,
// both fused, is the correctly rounded quotient (P. Markstein, IBM J. Res. Dev. 34, 1990); adding 1.5 2^23 then rounds it to an
// integer, ties to even, in the low bits.  Scales so small or large that the reciprocal is not normal, and those so small that
// their own rounding is coarse, are divided by; both ways give the same codes.
template <typename T>
__device__ __forceinline__ uint32_t quantise8(const Kv4Raw8<T> &raw, uint32_t word, float inv) {
    float x[8];
    kv4_widen8(raw, x);
    const float zero = kv4_zero(word), scale = kv4_scale(word);
    uint32_t codes = 0u;
    if (scale > 1e-30f && scale < 1e37f) {
        const uint64_t inv2 = twice(inv), scale2 = twice(-scale), zero2 = twice(-zero), magic2 = twice(12582912.f);
#pragma unroll
        for (int j = 6; j >= 0; j -= 2) {           // two at a time in the packed fp32 instructions
            const uint64_t t = add2(both(x[j], x[j + 1]), zero2), q0 = mul2(t, inv2);
            const uint64_t v = add2(fma2(fma2(q0, scale2, t), inv2, q0), magic2);       // 0x4B400000 + code: the constant is taken off below
            codes = codes * 256u + (uint32_t)(v >> 32) * 16u + (uint32_t)v;
        }
        codes -= 0x3F400000u;                       // sum over j of 0x4B400000 16^j, modulo 2^32
    } else if (scale > 0.f) {                       // zero (all elements alike) and NaN scales leave the codes at zero
#pragma unroll 1
        for (int j = 0; j < 8; ++j) {
            float t = x[0];
#pragma unroll
            for (int k = 1; k < 8; ++k) t = j == k ? x[k] : t;
            codes |= (uint32_t)fminf(fmaxf(rintf((t - zero) / scale), 0.f), 15.f) << (4 * j);
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
    Kv4Raw8<T> raw[2 * KV4_UNROLL];                                             // k, v, k, v .. as stored: widened only when their turn comes
    bool live[KV4_UNROLL], any = false;
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        const int t = t0 + i * ROWS;
        live[i] = t < n;
        if (live[i] && ((long long)start + t < 0 || (long long)start + t >= cap)) {
            kv4_report(status);
            live[i] = false;
        }
        raw[2 * i] = raw[2 * i + 1] = {};
        if (live[i]) {
            raw[2 * i] = kv4_raw8(k + src + (long long)t * Hkv * D);
            raw[2 * i + 1] = kv4_raw8(v + src + (long long)t * Hkv * D);
        }
        any |= live[i];
    }
    if (n_new && blockIdx.x == 0 && h == 0 && threadIdx.x == 0 && (n_new[b] < 0 || n_new[b] > T_new)) kv4_report(status);       // behind the loads: in front 3 %
    static_assert(ROWS * KV4_UNROLL <= KV4_THREADS, "one thread a token");
    if (threadIdx.x < ROWS * KV4_UNROLL) {  // weights and positions: one store for all tokens of the block (one a token: +8 %)
        const int t = blockIdx.x * (ROWS * KV4_UNROLL) + threadIdx.x;
        const long long row = (long long)start + t;
        if (t < n && row >= 0 && row < cap) {
            if (cache.weight) cache.weight[dst + row] = 0.f;
            if (h == 0 && cache.pos && positions) cache.pos[(long long)b * cap + row] = positions[(long long)b * T_new + t];
        }
    }
    if (!__any_sync(0xffffffffu, any)) return;                                  // the lanes of a warp stay together: shuffles
    const Groups<GROUP> groups(raw);
    const long long at = dst + start + t0;                                      // the first token's row; only live ones are stored
    uint32_t *kc = (uint32_t *)cache.k_codes + at * LPR + c * NG + g, *vc = (uint32_t *)cache.v_codes + at * LPR + l;
    uint32_t *ks = (uint32_t *)cache.k_scales + at * (D / GROUP) + l / (GROUP / 8), *vs = (uint32_t *)cache.v_scales + at * (D / GROUP) + l / (GROUP / 8);
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        if (!__any_sync(0xffffffffu, live[i])) continue;
        const uint32_t wk = groups.word(2 * i), wv = groups.word(2 * i + 1);
        const uint32_t ck = quantise8(raw[2 * i], wk, groups.inv(2 * i));
        const uint32_t cv = value_word<D>(quantise8(raw[2 * i + 1], wv, groups.inv(2 * i + 1)), l);
        if (!live[i]) continue;
        kc[i * (ROWS * LPR)] = ck;
        vc[i * (ROWS * LPR)] = cv;
        if (l % (GROUP / 8) == 0) {
            ks[i * (ROWS * (D / GROUP))] = wk;
            vs[i * (ROWS * (D / GROUP))] = wv;
        }
    }
}

// Tokens of a sequence: what the caller says (NULL: all `most`), held to [0, most]; a value outside is recorded by its first block.
__device__ __forceinline__ int tokens(const int32_t *counts, int b, int most, int *status) {
    if (!counts) return most;
    const int n = counts[b];
    if ((n < 0 || n > most) && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) kv4_report(status);
    return min(max(n, 0), most);
}

// Grid (token blocks, Hkv, Bz).
template <typename T, int D, int GROUP>
__global__ void __launch_bounds__(KV4_THREADS)
kv4_read_kernel(int cap, int n_out, const int32_t *__restrict__ row_start, const int32_t *__restrict__ n_rows, str_kv4_cache cache,
                T *__restrict__ k_out, T *__restrict__ v_out, int *status) {
    constexpr int LPR = D / 8, NG = D / 32, ROWS = KV4_THREADS / LPR;
    const int h = blockIdx.y, b = blockIdx.z, Hkv = gridDim.y;
    const int l = threadIdx.x % LPR, g = l >> 2, c = l & 3;
    const int n = tokens(n_rows, b, n_out, status), start = row_start[b];
    const long long base = ((long long)b * Hkv + h) * cap, out = ((long long)b * n_out * Hkv + h) * D + 8 * l;
    const int t0 = blockIdx.x * (ROWS * KV4_UNROLL) + threadIdx.x / LPR;
    uint32_t ck[KV4_UNROLL], cv[KV4_UNROLL], wk[KV4_UNROLL], wv[KV4_UNROLL];
#pragma unroll
    for (int i = 0; i < KV4_UNROLL; ++i) {
        const int t = t0 + i * ROWS;
        const long long row = (long long)start + t;
        ck[i] = cv[i] = wk[i] = wv[i] = 0u;                                     // reads as zero
        if (t >= n) continue;
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
    if (!ctx || T_new < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache)) return STR_ERR_INVALID_ARG;
    if (T_new == 0) return STR_OK;
    if (!k || !v || !row_start || (((uintptr_t)k | (uintptr_t)v) & 15)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
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
    if (!ctx || n_out < 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    const int rc = kv4_check_shape(s);
    if (rc != STR_OK) return rc;
    if (!kv4_pointers_ok(cache)) return STR_ERR_INVALID_ARG;
    if (n_out == 0) return STR_OK;
    if (!k_out || !v_out || !row_start || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    const dim3 grid(ceil_div(n_out, KV4_THREADS / (s->d / 8) * KV4_UNROLL), s->Hkv, s->Bz);
#define KV4_CALL(T, D, G)                                                                                              \
    kv4_read_kernel<T, D, G><<<grid, KV4_THREADS, 0, (cudaStream_t)stream>>>(s->cap, n_out, row_start, n_rows, *cache, \
                                                                             (T *)k_out, (T *)v_out, ctx->status_dev)
    KV4_DISPATCH(dtype, s, KV4_CALL);
#undef KV4_CALL
    return str_launch_ok(ctx);
}

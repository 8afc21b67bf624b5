// str_rope_split_ex: the columns [q heads | k heads | v heads] of a projection go to three tensors, the first rot_dim elements of every q
// and k head turned pair by pair,
//   (a, b) <- amplitude (a cos - b sin, b cos + a sin),   angle = position * f_i,
// with pairs (i, i + rot_dim / 2) or (2 i, 2 i + 1), and frequencies f_i stretched for contexts longer than the trained one.
//
// The host forms f_i in 64 bits and hands the kernel turns per position, f_i / 2 pi.  A position times that is still 64 bits; quarter turns are
// taken off before the rest is rounded to fp32.  Frequency and product are each right to 2^-53: with f_i = 1 a position of 2^31 is 2^30.4 quarter turns, and its
// angle right to 2^-21 of one, in proportion less for smaller positions and frequencies, down to the 2^-26 of the rounding.
//
// Bound by memory: every column in once and out once (16512 rows of 32 / 8 heads of 128, bf16: 70 us = 5.8 TB/s in both layouts, interleaved down to 66).
#include <math.h>

#include "packed.cuh"

namespace {

constexpr int THREADS = 256, MAX_PAIRS = 128;
constexpr double MAX_TURNS = 1 << 20;                     // a position: quarter turns stay below 2^53, where the last whole one is still known

struct RopeTable {
    double turns[MAX_PAIRS];                              // per position
    float amplitude;
};

__device__ __forceinline__ float2 rotation(const RopeTable &tab, int32_t pos, int i) {
    const double quarters = 4.0 * ((double)pos * tab.turns[i]);
    const double whole = rint(quarters);
    float sn, cs;
    sincospif(0.5f * (float)(quarters - whole), &sn, &cs);
    const int k = (int)((long long)whole & 3);
    const float c = k == 0 ? cs : k == 1 ? -sn : k == 2 ? -cs : sn;
    const float s = k == 0 ? sn : k == 1 ? cs : k == 2 ? -sn : -cs;
    return make_float2(tab.amplitude * c, tab.amplitude * s);
}

// Written out, so that every variant rounds alike.
__device__ __forceinline__ float turn_a(float2 w, float a, float b) { return fmaf(a, w.x, -__fmul_rn(b, w.y)); }
__device__ __forceinline__ float turn_b(float2 w, float a, float b) { return fmaf(b, w.x, __fmul_rn(a, w.y)); }

// One 16-byte access, or VEC accesses of one element.
template <typename T, int VEC> struct alignas(VEC * sizeof(T) == 16 ? 16 : sizeof(T)) Pack { T v[VEC]; };

// ROWS rows a block, their rotations in shared memory.  A unit is VEC pairs (HALF: a vector of first elements and one of second ones;
// interleaved: one vector, VEC / 2 pairs) or a vector that is copied; a thread takes one unit of all the rows at a time.
template <typename T, int VEC, bool HALF, int ROWS>
__global__ void __launch_bounds__(THREADS)
rope_split_ex_kernel(const __grid_constant__ RopeTable tab, int rows, int Hq, int Hkv, int d, int rot, const int32_t *__restrict__ positions,
                     const T *__restrict__ qkv, T *__restrict__ q_out, T *__restrict__ k_out, T *__restrict__ v_out) {
    extern __shared__ float2 turn[];                      // [ROWS][rot / 2]
    typedef Pack<T, VEC> V;
    const int pairs = rot / 2, row0 = blockIdx.x * ROWS, ld = (Hq + 2 * Hkv) * d;
    for (int e = threadIdx.x; e < ROWS * pairs; e += THREADS) {
        const int r = e / pairs, i = e - r * pairs;
        if (row0 + r < rows) turn[e] = rotation(tab, __ldg(positions + row0 + r), i);
    }
    __syncthreads();
    const int turned = HALF ? pairs / VEC : rot / VEC, per_head = turned + (d - rot) / VEC;
    const int heads = (Hq + Hkv) * per_head, units = heads + Hkv * d / VEC;
    for (int e = threadIdx.x; e < units; e += blockDim.x) {
        int head = 0, u = turned, at;                     // at: column of the unit's (first) vector
        T *dst;
        int width;                                        // elements of a row of dst
        if (e < heads) {
            head = e / per_head;
            u = e - head * per_head;
            const int c = u < turned ? u * VEC : rot + (u - turned) * VEC;
            at = head * d + c;
            dst = head < Hq ? q_out + at : k_out + (at - Hq * d);
            width = head < Hq ? Hq * d : Hkv * d;
        } else {
            at = (Hq + Hkv) * d + (e - heads) * VEC;
            dst = v_out + (e - heads) * VEC;
            width = Hkv * d;
        }
        V a[ROWS], b[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (row0 + r < rows) {
                const T *src = qkv + (size_t)(row0 + r) * ld + at;
                a[r] = *(const V *)src;
                if (HALF && u < turned) b[r] = *(const V *)(src + pairs);
            }
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (row0 + r < rows) {
                T *to = dst + (size_t)(row0 + r) * width;
                if (u < turned) {
                    const float2 *t = turn + r * pairs + (HALF ? u * VEC : u * (VEC / 2));
                    if (HALF) {
#pragma unroll
                        for (int i = 0; i < VEC; ++i) {
                            const float2 w = t[i];
                            const float x = ldf(&a[r].v[i]), y = ldf(&b[r].v[i]);
                            stf(&a[r].v[i], turn_a(w, x, y));
                            stf(&b[r].v[i], turn_b(w, x, y));
                        }
                        *(V *)(to + pairs) = b[r];
                    } else {
#pragma unroll
                        for (int i = 0; i < VEC / 2; ++i) {
                            const float2 w = t[i];
                            const float x = ldf(&a[r].v[2 * i]), y = ldf(&a[r].v[2 * i + 1]);
                            stf(&a[r].v[2 * i], turn_a(w, x, y));
                            stf(&a[r].v[2 * i + 1], turn_b(w, x, y));
                        }
                    }
                }
                *(V *)to = a[r];
            }
    }
}

template <typename T, int VEC, bool HALF, int ROWS>
void launch_rows(const RopeTable &tab, int rows, int Hq, int Hkv, int d, int rot, const int32_t *pos, const void *qkv, void *q, void *k, void *v,
                 cudaStream_t st) {
    rope_split_ex_kernel<T, VEC, HALF, ROWS><<<ceil_div(rows, ROWS), THREADS, (size_t)ROWS * (rot / 2) * sizeof(float2), st>>>(
        tab, rows, Hq, Hkv, d, rot, pos, (const T *)qkv, (T *)q, (T *)k, (T *)v);
}
template <typename T, int VEC, bool HALF>
void launch(const RopeTable &tab, int rows, int Hq, int Hkv, int d, int rot, int sms, const int32_t *pos, const void *qkv, void *q, void *k, void *v,
            cudaStream_t st) {
    // Four rows a block where a block has one vector of each in flight and there are enough rows (16512 rows, interleaved: 66 us against 75); one where it has
    // two, whose registers leave too few warps (half layout: 70 us against 131).
    if (!HALF && rows >= 16 * sms) launch_rows<T, VEC, HALF, 4>(tab, rows, Hq, Hkv, d, rot, pos, qkv, q, k, v, st);
    else launch_rows<T, VEC, HALF, 1>(tab, rows, Hq, Hkv, d, rot, pos, qkv, q, k, v, st);
}
// 16-byte vectors where they stay within a head's turned part (its halves) and its rest and the pointers allow it; else single elements (half
// layout) or pairs.
template <typename T>
void dispatch(const RopeTable &tab, bool half, int rows, int Hq, int Hkv, int d, int rot, int sms, const int32_t *pos, const void *qkv, void *q, void *k,
              void *v, cudaStream_t st) {
    constexpr int VEC = 16 / sizeof(T);
    const bool aligned = (((uintptr_t)qkv | (uintptr_t)q | (uintptr_t)k | (uintptr_t)v) & 15) == 0 && d % VEC == 0;
    if (half) {
        if (aligned && rot % (2 * VEC) == 0) launch<T, VEC, true>(tab, rows, Hq, Hkv, d, rot, sms, pos, qkv, q, k, v, st);
        else launch<T, 1, true>(tab, rows, Hq, Hkv, d, rot, sms, pos, qkv, q, k, v, st);
    } else {
        if (aligned && rot % VEC == 0) launch<T, VEC, false>(tab, rows, Hq, Hkv, d, rot, sms, pos, qkv, q, k, v, st);
        else launch<T, 2, false>(tab, rows, Hq, Hkv, d, rot, sms, pos, qkv, q, k, v, st);
    }
}

}  // namespace

extern "C" int str_rope_split_ex(str_ctx *ctx, const str_rope_desc *r, int dtype, int rows, int Hq, int Hkv, int d, const int32_t *positions, const void *qkv,
                                 void *q_out, void *k_out, void *v_out, void *stream) {
    if (!ctx || !r || rows < 0 || Hq <= 0 || Hkv <= 0 || d <= 0 || (dtype != STR_F32 && dtype != STR_BF16)) return STR_ERR_INVALID_ARG;
    if (r->rot_dim <= 0 || r->rot_dim > d || r->rot_dim % 2 != 0 || !(r->theta > 0.0) || !isfinite(r->theta) || !isfinite((float)r->amplitude) ||
        (r->layout != STR_ROPE_HALF && r->layout != STR_ROPE_INTERLEAVED))
        return STR_ERR_INVALID_ARG;
    if (r->scaling != STR_ROPE_NONE && r->scaling != STR_ROPE_LINEAR && r->scaling != STR_ROPE_BANDED) return STR_ERR_INVALID_ARG;
    if (r->scaling != STR_ROPE_NONE && !(r->factor > 0.0 && isfinite(r->factor))) return STR_ERR_INVALID_ARG;
    if (r->scaling == STR_ROPE_BANDED && (r->trained_len <= 0 || !(r->turns_low >= 0.0) || !(r->turns_high > r->turns_low) || !isfinite(r->turns_high)))
        return STR_ERR_INVALID_ARG;
    if (rows == 0) return STR_OK;
    if (!positions || !qkv || !q_out || !k_out || !v_out) return STR_ERR_INVALID_ARG;
    if (r->rot_dim > 2 * MAX_PAIRS || rows > (1 << 30) || ((long long)Hq + 2LL * Hkv) * d > (1 << 28)) return STR_ERR_UNSUPPORTED_SHAPE;
    if (d % 2 != 0 && r->layout == STR_ROPE_INTERLEAVED) return STR_ERR_UNSUPPORTED_SHAPE;
    const size_t row = dtype_size(dtype) * d, in = row * (Hq + 2 * Hkv) * rows;
    const struct { const void *at; size_t bytes; } out[] = {{q_out, row * Hq * rows}, {k_out, row * Hkv * rows}, {v_out, row * Hkv * rows}};
    for (int i = 0; i < 3; ++i)
        if (kv4_overlap(qkv, in, out[i].at, out[i].bytes) || kv4_overlap(positions, sizeof(int32_t) * rows, out[i].at, out[i].bytes) ||
            kv4_overlap(out[i].at, out[i].bytes, out[(i + 1) % 3].at, out[(i + 1) % 3].bytes))
            return STR_ERR_INVALID_ARG;
    RopeTable tab = {};
    for (int i = 0; i < r->rot_dim / 2; ++i) {
        double f = pow(r->theta, -2.0 * i / r->rot_dim) / 6.283185307179586476925;
        if (r->scaling == STR_ROPE_LINEAR) f /= r->factor;
        if (r->scaling == STR_ROPE_BANDED) {
            double keep = (r->trained_len * f - r->turns_low) / (r->turns_high - r->turns_low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f = f * keep + f / r->factor * (1.0 - keep);
        }
        if (!(f < MAX_TURNS)) return STR_ERR_INVALID_ARG;
        tab.turns[i] = f;
    }
    tab.amplitude = (float)r->amplitude;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    const bool half = r->layout == STR_ROPE_HALF;
    if (dtype == STR_BF16)
        dispatch<__nv_bfloat16>(tab, half, rows, Hq, Hkv, d, r->rot_dim, ctx->sm_count, positions, qkv, q_out, k_out, v_out, (cudaStream_t)stream);
    else
        dispatch<float>(tab, half, rows, Hq, Hkv, d, r->rot_dim, ctx->sm_count, positions, qkv, q_out, k_out, v_out, (cudaStream_t)stream);
    return str_launch_ok(ctx);
}

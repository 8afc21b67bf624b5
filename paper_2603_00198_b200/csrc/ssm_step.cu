// str_mamba2_step: the Mamba-2 recurrence for a few tokens, one after the other, from a state in memory:
//   S <- exp(dt A_h) S + (dt x) b^T,   y = S c (+ D_h x)
// which is linear attention with a decay per head in its recurrent form (q = c, k = dt b, v = x, decay = exp(dt A)).
//
// The state is p x n fp32 per head, read once and written once whatever the number of tokens: it stays in registers while
// the tokens go by.  A row of the state (one of p) lies across a group of lanes, each holding vectors of VEC consecutive
// columns, so that both the loads and the sum over n in y are along the lanes; a warp works on RPT rows per group at once,
// all their loads in flight together.  All arithmetic is fp32; y is rounded to the storage type once.
//
// Bound by memory.  64 sequences of the 8B-class layer (537 MB of state in and out): 83.0 us = 6.50 TB/s, 0.99 of the measured
// copy bandwidth, in a CUDA graph; one call after the other 88.4 us, 0.93.  Streaming loads and stores (neither alone does it) and blocks of 128 threads are what it takes: 99.8 us with 256
// threads and plain accesses, 93.5 with 128 threads.  From 1 to 32 sequences they are never slower, with the states in L2 or
// not (one sequence 3.2 us either way).
#include "kv4.cuh"

namespace {

constexpr int STEP_THREADS = 128;

template <int VEC> struct Vec;
template <> struct Vec<4> { typedef float4 type; };
template <> struct Vec<1> { typedef float type; };

// LPR lanes per row, NV vectors of VEC columns per lane (columns (v * LPR + lane) * VEC ..), RPT rows per lane group.
template <typename T, int VEC, int LPR, int NV, int RPT>
__global__ void __launch_bounds__(STEP_THREADS)
mamba2_step_kernel(int T_new, int H, int p, int n, int G, const T *__restrict__ x, const float *__restrict__ dt, const float *__restrict__ A,
                   const T *__restrict__ B, const T *__restrict__ C, const float *__restrict__ Dskip, const float *state, float *state_out,
                   T *__restrict__ y) {
    typedef typename Vec<VEC>::type V;
    constexpr int GPW = 32 / LPR;                                       // row groups per warp
    const int h = blockIdx.y, b = blockIdx.z, g = h / (H / G);
    const int lane = threadIdx.x & 31, l = lane % LPR;
    const int group = blockIdx.x * (STEP_THREADS / LPR) + (threadIdx.x >> 5) * GPW + lane / LPR;
    const int row0 = group * RPT;
    const long long sbase = ((long long)b * H + h) * p * n;
    alignas(16) float S[RPT][NV][VEC];
#pragma unroll
    for (int r = 0; r < RPT; ++r)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * LPR + l) * VEC;
            V val = {};
            if (row0 + r < p && col < n) val = __ldcs((const V *)(state + sbase + (long long)(row0 + r) * n + col));
            *(V *)S[r][v] = val;
        }
    const float Ah = A[h], Dh = Dskip ? Dskip[h] : 0.f;
    for (int t = 0; t < T_new; ++t) {
        const long long bt = (long long)b * T_new + t;
        const float dtv = dt[bt * H + h], decay = expf(dtv * Ah);
        float xv[RPT], acc[RPT];
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
            xv[r] = row0 + r < p ? ldf(x + (bt * H + h) * p + row0 + r) : 0.f;
            acc[r] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * LPR + l) * VEC;
            float bv[VEC], cv[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                bv[i] = col < n ? ldf(B + (bt * G + g) * n + col + i) : 0.f;
                cv[i] = col < n ? ldf(C + (bt * G + g) * n + col + i) : 0.f;
            }
#pragma unroll
            for (int r = 0; r < RPT; ++r) {
                const float dx = dtv * xv[r];
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    S[r][v][i] = fmaf(decay, S[r][v][i], dx * bv[i]);
                    acc[r] = fmaf(S[r][v][i], cv[i], acc[r]);
                }
            }
        }
#pragma unroll
        for (int r = 0; r < RPT; ++r) {
#pragma unroll
            for (int o = LPR / 2; o > 0; o >>= 1) acc[r] += __shfl_xor_sync(0xffffffffu, acc[r], o);
            if (l == 0 && row0 + r < p) stf(y + (bt * H + h) * p + row0 + r, fmaf(Dh, xv[r], acc[r]));
        }
    }
#pragma unroll
    for (int r = 0; r < RPT; ++r)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * LPR + l) * VEC;
            if (row0 + r < p && col < n) __stcs((V *)(state_out + sbase + (long long)(row0 + r) * n + col), *(V *)S[r][v]);
        }
}

template <typename T, int VEC, int LPR, int NV, int RPT>
void launch_step(const str_ssd_shape *s, const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D,
                 const float *state, float *state_out, void *y, cudaStream_t st) {
    const int rows_per_cta = STEP_THREADS / LPR * RPT;
    mamba2_step_kernel<T, VEC, LPR, NV, RPT><<<dim3(ceil_div(s->p, rows_per_cta), s->H, s->Bz), STEP_THREADS, 0, st>>>(
        s->T, s->H, s->p, s->n, s->G, (const T *)x, dt, A, (const T *)B, (const T *)C, D, state, state_out, (T *)y);
}

template <typename T>
void dispatch_step(const str_ssd_shape *s, const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D,
                   const float *state, float *state_out, void *y, cudaStream_t st) {
    const bool vec = s->n % 4 == 0 && (((uintptr_t)state | (uintptr_t)state_out) & 15) == 0;
#define STEP(VEC, LPR, NV, RPT) launch_step<T, VEC, LPR, NV, RPT>(s, x, dt, A, B, C, D, state, state_out, y, st)
    if (vec) {
        if (s->n <= 16) STEP(4, 4, 1, 4);
        else if (s->n <= 32) STEP(4, 8, 1, 4);
        else if (s->n <= 64) STEP(4, 16, 1, 8);
        else if (s->n <= 128) STEP(4, 32, 1, 8);
        else if (s->n <= 256) STEP(4, 32, 2, 4);
        else STEP(4, 32, 4, 2);
    } else {
        if (s->n <= 32) STEP(1, 32, 1, 8);
        else if (s->n <= 128) STEP(1, 32, 4, 4);
        else STEP(1, 32, 16, 2);
    }
#undef STEP
}

}  // namespace

extern "C" int str_mamba2_step(str_ctx *ctx, const str_ssd_shape *s, const void *x, const float *dt, const float *A, const void *B,
                               const void *C, const float *D, const float *state, void *y, float *state_out, void *stream) {
    if (!ctx || !s || !x || !dt || !A || !B || !C || !state || !y || !state_out) return STR_ERR_INVALID_ARG;
    if (s->Bz <= 0 || s->T <= 0 || s->H <= 0 || s->p <= 0 || s->n <= 0 || s->G <= 0 || s->H % s->G != 0 ||
        (s->dtype != STR_F32 && s->dtype != STR_BF16))
        return STR_ERR_INVALID_ARG;
    const size_t state_bytes = (size_t)s->Bz * s->H * s->p * s->n * sizeof(float);
    if (state_out != state && kv4_overlap(state, state_bytes, state_out, state_bytes)) return STR_ERR_INVALID_ARG;
    if (s->n > 512 || s->Bz > 65535 || s->H > 65535) return STR_ERR_UNSUPPORTED_SHAPE;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_SSD, stream);
    if (s->dtype == STR_BF16) dispatch_step<__nv_bfloat16>(s, x, dt, A, B, C, D, state, state_out, y, (cudaStream_t)stream);
    else dispatch_step<float>(s, x, dt, A, B, C, D, state, state_out, y, (cudaStream_t)stream);
    return str_launch_ok(ctx);
}

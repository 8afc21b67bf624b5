// str_mamba2_prefill_packed: the Mamba-2 recurrence over packed sequences, each from a state of its own,
//   S <- exp(dt A_h) S + (dt x) b^T,   y = S c + D_h x.
// The entry point, and the kernel that runs the recurrence token by token in fp32: every type and shape.
//
// A row of the state (one of p) lies across four lanes, NV vectors of four columns each; a block holds the rows of one head of one
// sequence in registers from the first token to the last.  Tokens come through shared memory TB at a time; the next ones are already on their way to
// registers.  A lane leaves its part of y in shared memory, and the four parts are added when the tokens' outputs are written: no shuffles between
// tokens, whose chain is then one fused operation a token.  Per token and head that is p n (one multiplication and two fused ones): as many
// operations as the chunked form in fp32 needs, without its two roundings more, and a state that never leaves the registers.
//
// Bound by the chain of tokens where sequences are few (five turns of 1237 rows, 24 heads of 32 x 20: 67 us, 120 ns a token of the longest), by fp32
// arithmetic and the reading of b and c from shared memory where there are many (5000 rows, 128 heads of 64 x 128: 1.88 ms, 17 TFLOP/s).
#include "dispatch.cuh"
#include "packed.cuh"

namespace {

constexpr int LPR = 4;                                    // lanes per row
// Tokens per turn: as many as their b, c and outputs leave registers for.
template <int NV> constexpr int TOKENS = NV <= 4 ? 32 : 16;

template <typename T, int NV, int WARPS>
__global__ void __launch_bounds__(32 * WARPS)
scan_packed_kernel(int n_seq, int rows, int H, int p, int n, int G, const T *__restrict__ x, const float *__restrict__ dt, const float *__restrict__ A,
                   const T *__restrict__ B, const T *__restrict__ C, const float *__restrict__ Dskip, const int32_t *__restrict__ start,
                   const float *state, T *__restrict__ y, float *final_state, int *status) {
    constexpr int NP = NV * 4 * LPR, TB = TOKENS<NV>;     // columns, padded; tokens per turn
    constexpr int threads = 32 * WARPS, R = threads / LPR; // rows of the state per block
    extern __shared__ float4 smem4[];
    float *bs = (float *)smem4, *cs = bs + TB * NP, *xs = cs + TB * NP;
    float *ys = xs + TB * R, *dts = ys + TB * R * LPR, *decay = dts + TB;
    const int h = blockIdx.y, s = blockIdx.z, g = h / (H / G);
    const int tid = threadIdx.x, i0 = blockIdx.x * R, r = tid / LPR, l = tid % LPR;
    if (blockIdx.x == 0 && h == 0 && s == 0) packed_check(start, n_seq, rows, status);
    const int t0 = packed_start(start, s, rows), t1 = packed_start(start, s + 1, rows);
    if (t1 <= t0 && (!final_state || (state == final_state))) return;
    const size_t base = (((size_t)s * H + h) * p + i0 + r) * n;
    // Four columns at a time where a row has whole vectors of them.
    const bool vec = n % 4 == 0 && (((uintptr_t)state | (uintptr_t)final_state) & 15) == 0;
    alignas(16) float S[NV][4];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * LPR + l) * 4;
#pragma unroll
        for (int i = 0; i < 4; ++i) S[v][i] = 0.f;
        if (state && i0 + r < p && col < n) {
            if (vec) *(float4 *)S[v] = *(const float4 *)(state + base + col);
            else
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (col + i < n) S[v][i] = state[base + col + i];
        }
    }
    const float Ah = A[h], Dh = Dskip ? Dskip[h] : 0.f;
    // What the thread carries of the next TB tokens: elements tid + k threads of [TB][NP] and of [TB][R].
    constexpr int PER = TB * NP / threads;
    T bq[PER], cq[PER], xq[TB / LPR];
    float dq = 0.f;
    auto fetch = [&](int tb) {
        const int m = min(TB, t1 - tb);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int e = tid + k * threads, t = e / NP, col = e % NP;
            stf(&bq[k], 0.f);
            stf(&cq[k], 0.f);
            if (t < m && col < n) {
                const size_t at = ((size_t)(tb + t) * G + g) * n + col;
                bq[k] = B[at];
                cq[k] = C[at];
            }
        }
#pragma unroll
        for (int k = 0; k < TB / LPR; ++k) {
            const int e = tid + k * threads, t = e / R, i = e % R;
            stf(&xq[k], 0.f);
            if (t < m && i0 + i < p) xq[k] = x[((size_t)(tb + t) * H + h) * p + i0 + i];
        }
        if (tid < m) dq = dt[(size_t)(tb + tid) * H + h];
    };
    if (t0 < t1) fetch(t0);
    for (int tb = t0; tb < t1; tb += TB) {
        const int m = min(TB, t1 - tb);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            bs[tid + k * threads] = ldf(&bq[k]);
            cs[tid + k * threads] = ldf(&cq[k]);
        }
#pragma unroll
        for (int k = 0; k < TB / LPR; ++k) xs[tid + k * threads] = ldf(&xq[k]);
        if (tid < m) {
            dts[tid] = dq;
            decay[tid] = expf(dq * Ah);
        }
        __syncthreads();
        if (tb + TB < t1) fetch(tb + TB);
#pragma unroll (NV >= 8 ? 2 : 4)
        for (int t = 0; t < m; ++t) {
            const float dx = dts[t] * xs[t * R + r], a = decay[t];
            float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const float4 b = *(const float4 *)(bs + t * NP + (v * LPR + l) * 4), c = *(const float4 *)(cs + t * NP + (v * LPR + l) * 4);
                S[v][0] = fmaf(a, S[v][0], dx * b.x); acc[0] = fmaf(S[v][0], c.x, acc[0]);
                S[v][1] = fmaf(a, S[v][1], dx * b.y); acc[1] = fmaf(S[v][1], c.y, acc[1]);
                S[v][2] = fmaf(a, S[v][2], dx * b.z); acc[2] = fmaf(S[v][2], c.z, acc[2]);
                S[v][3] = fmaf(a, S[v][3], dx * b.w); acc[3] = fmaf(S[v][3], c.w, acc[3]);
            }
            ys[t * threads + tid] = (acc[0] + acc[1]) + (acc[2] + acc[3]);
        }
        __syncthreads();
        for (int e = tid; e < m * R; e += threads) {
            const int t = e / R, i = e % R;
            const float4 part = *(const float4 *)(ys + e * LPR);
            if (i0 + i < p) stf(y + ((size_t)(tb + t) * H + h) * p + i0 + i, fmaf(Dh, xs[e], (part.x + part.y) + (part.z + part.w)));
        }
        __syncthreads();
    }
    if (!final_state || i0 + r >= p) return;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = (v * LPR + l) * 4;
        if (vec && col < n) *(float4 *)(final_state + base + col) = *(const float4 *)S[v];
        if (!vec)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (col + i < n) final_state[base + col + i] = S[v][i];
    }
}

template <typename T, int NV, int WARPS>
int launch(str_ctx *ctx, const str_ssd_packed_shape *s, const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D,
           const int32_t *start, const float *state, void *y, float *final_state, cudaStream_t st) {
    constexpr int TB = TOKENS<NV>, threads = 32 * WARPS, R = threads / LPR;
    constexpr size_t smem = sizeof(float) * ((size_t)TB * (2 * NV * 4 * LPR + R + threads) + 2 * TB);
    if (smem > 48 * 1024) STR_CUDA_OK(cudaFuncSetAttribute(scan_packed_kernel<T, NV, WARPS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    scan_packed_kernel<T, NV, WARPS><<<dim3(ceil_div(s->p, R), s->H, s->n_seq), threads, smem, st>>>(
        s->n_seq, s->rows, s->H, s->p, s->n, s->G, (const T *)x, dt, A, (const T *)B, (const T *)C, D, start, state, (T *)y, final_state, ctx->status_dev);
    return str_launch_ok(ctx);
}
// Four warps hold 32 rows of a head, eight 64.
template <typename T>
int dispatch(str_ctx *ctx, const str_ssd_packed_shape *s, const void *x, const float *dt, const float *A, const void *B, const void *C, const float *D,
             const int32_t *start, const float *state, void *y, float *final_state, cudaStream_t st) {
    const int need = ceil_div(s->n, 4 * LPR);
#define SCAN(NV)                                                                                              \
    (s->p <= 32 && NV < 16 ? launch<T, NV, 4>(ctx, s, x, dt, A, B, C, D, start, state, y, final_state, st) \
                           : launch<T, NV, 8>(ctx, s, x, dt, A, B, C, D, start, state, y, final_state, st))
    return need <= 1 ? SCAN(1) : need <= 2 ? SCAN(2) : need <= 4 ? SCAN(4) : need <= 8 ? SCAN(8) : SCAN(16);
#undef SCAN
}

}  // namespace

extern "C" size_t str_mamba2_prefill_packed_workspace_size(const str_ssd_packed_shape *) { return 0; }

extern "C" int str_mamba2_prefill_packed(str_ctx *ctx, const str_ssd_packed_shape *s, const void *x, const float *dt, const float *A, const void *B,
                                         const void *C, const float *D, const int32_t *seq_start, const float *init_state, void *y,
                                         float *final_state, void *workspace, size_t workspace_bytes, void *stream) {
    (void)workspace;
    if (!ctx || !s || !A || !seq_start) return STR_ERR_INVALID_ARG;
    if (s->n_seq <= 0 || s->rows < 0 || s->H <= 0 || s->p <= 0 || s->n <= 0 || s->G <= 0 || s->H % s->G != 0 ||
        (s->dtype != STR_F32 && s->dtype != STR_BF16))
        return STR_ERR_INVALID_ARG;
    if (s->rows > 0 && (!x || !dt || !B || !C || !y)) return STR_ERR_INVALID_ARG;
    if (s->n > 256 || s->n_seq > 65535 || s->H > 65535 || s->rows > (1 << 30) || s->p > (1 << 20)) return STR_ERR_UNSUPPORTED_SHAPE;
    const size_t state_bytes = (size_t)s->n_seq * s->H * s->p * s->n * sizeof(float), es = dtype_size(s->dtype);
    const size_t xb = (size_t)s->rows * s->H * s->p * es, bb = (size_t)s->rows * s->G * s->n * es;
    if (final_state != init_state && kv4_overlap(init_state, state_bytes, final_state, state_bytes)) return STR_ERR_INVALID_ARG;
    if (kv4_overlap(x, xb, y, xb) || kv4_overlap(B, bb, y, xb) || kv4_overlap(C, bb, y, xb)) return STR_ERR_INVALID_ARG;
    if (workspace_bytes < str_mamba2_prefill_packed_workspace_size(s)) return STR_ERR_WORKSPACE_TOO_SMALL;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_SSD, stream);
    cudaStream_t st = (cudaStream_t)stream;
    // The chunked kernel's CTAs cost what a chunk of 128 rows costs however few there are.  Sequences of 16 rows on average are where the two meet (one
    // sequence, 128 heads of 64 x 128: 8 rows 6.6 us token by token against 9.0, 16 rows 9.5 against 9.0; 33 sequences, 24 heads: 16 rows 15 against 49).
    if (!str_force_simt() && s->rows > 16LL * s->n_seq && str_scan_packed_tc_supported(s, x, B, C, y))
        return ++ctx->tc_calls, str_scan_packed_tc(ctx, s, x, dt, A, B, C, D, seq_start, init_state, y, final_state, st);
    ++ctx->fallback_calls;
    if (s->dtype == STR_BF16) return dispatch<__nv_bfloat16>(ctx, s, x, dt, A, B, C, D, seq_start, init_state, y, final_state, st);
    return dispatch<float>(ctx, s, x, dt, A, B, C, D, seq_start, init_state, y, final_state, st);
}

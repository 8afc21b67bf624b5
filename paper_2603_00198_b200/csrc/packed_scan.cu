// str_mamba2_prefill_packed: the Mamba-2 recurrence over packed sequences, each from a state of its own,
//   S <- exp(dt A_h) S + (dt x) b^T,   y = S c + D_h x.
// The entry point, and the kernel that runs the recurrence token by token in fp32: every type and shape.
//
// Two rows of the state (of p) lie across four or eight lanes, NV vectors of four columns each; a block holds the rows of one head of one
// sequence in registers from the first token to the last.  Tokens come through shared memory TB at a time; the next ones are already on their way to
// registers.  A lane leaves its part of y in shared memory, half of a row's lanes after one exchange with the other half's, and the parts are added when
// the tokens' outputs are written; the chain from token to token is one fused operation.  Per token and head that is p n (one multiplication and two
// fused ones, two elements an instruction): as many operations as the chunked form in fp32 needs, without its two roundings more, and a state that never
// leaves the registers.
//
// Bound by the reading of b and c from shared memory: two rows a lane, so that a vector read serves eight fused operations (one row a lane: 1.88 ms where
// two take 1.22, 25.8 TFLOP/s, 5000 rows, 128 heads of 64 x 128), and several tokens' reads before the first one's output is stored.  Few sequences are
// bound by the chain of tokens, 77 ns each, whence the segments below (five turns of 1237 rows, the longest 547, 24 heads of 32 x 20: 31 to 34 us, whole 45).
#include <algorithm>

#include "dispatch.cuh"
#include "packed.cuh"

namespace {

// Tokens per turn: as many as their b, c and outputs leave registers for.  Tokens at a time, whose outputs are kept until all are formed: a store
// between two tokens would hold up the second one's reads.
template <int NV> constexpr int TOKENS = NV <= 2 ? 32 : 16;
template <int NV> constexpr int TOGETHER = NV <= 1 ? 8 : NV <= 2 ? 4 : 2;

// Y: outputs are wanted; else the final state and the sum of dt A (in powers of two) of every sequence are.
template <typename T, int NV, int LPR, int WARPS, bool Y>
__global__ void __launch_bounds__(32 * WARPS)
scan_packed_kernel(int n_seq, int rows, int H, int p, int n, int G, const T *__restrict__ x, const float *__restrict__ dt, const float *__restrict__ A,
                   const T *__restrict__ B, const T *__restrict__ C, const float *__restrict__ Dskip, const int32_t *__restrict__ start,
                   const float *state, T *__restrict__ y, float *final_state, float *__restrict__ faded, int *status) {
    constexpr int NP = NV * 4 * LPR, TB = TOKENS<NV>, TG = TOGETHER<NV>;  // columns, padded; tokens per turn, at a time
    constexpr int threads = 32 * WARPS, R = threads / LPR * 2, PARTS = LPR / 2; // rows of the state per block; what a row's sums come in
    extern __shared__ float4 smem4[];
    float *bs = (float *)smem4, *cs = bs + TB * NP, *ys = cs + TB * NP, *xs = ys + TB * threads;
    float2 *rate = (float2 *)(xs + TB * R);               // dt, exp(dt A)
    const int h = blockIdx.y, s = blockIdx.z, g = h / (H / G);
    const int tid = threadIdx.x, i0 = blockIdx.x * R, r = tid / LPR * 2, l = tid % LPR;
    if (blockIdx.x == 0 && h == 0 && s == 0) packed_check(start, n_seq, rows, status);
    const int t0 = packed_start(start, s, rows), t1 = packed_start(start, s + 1, rows);
    if (t1 <= t0 && (Y ? !final_state || state == final_state : false)) return;
    const size_t base = (((size_t)s * H + h) * p + i0 + r) * n;
    // Four columns at a time where a row has whole vectors of them.
    const bool vec = n % 4 == 0 && (((uintptr_t)state | (uintptr_t)final_state) & 15) == 0;
    alignas(16) float2 S[2][NV][2];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * LPR + l) * 4;
            const float *from = state + base + (size_t)j * n + col;
            S[j][v][0] = S[j][v][1] = make_float2(0.f, 0.f);
            if (state && i0 + r + j < p && col < n) {
                if (vec) *(float4 *)S[j][v] = *(const float4 *)from;
                else {
                    S[j][v][0].x = from[0];
                    if (col + 1 < n) S[j][v][0].y = from[1];
                    if (col + 2 < n) S[j][v][1].x = from[2];
                    if (col + 3 < n) S[j][v][1].y = from[3];
                }
            }
        }
    const float Ah = A[h], Dh = Dskip ? Dskip[h] : 0.f;
    // What the thread carries of the next TB tokens: elements tid + k threads of [TB][NP] and of [TB][R].
    constexpr int PER = TB * NP / threads, PER_X = TB * R / threads;
    T bq[PER], cq[PER], xq[PER_X];
    float dq = 0.f, fade = 0.f;
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
                if (Y) cq[k] = C[at];
            }
        }
#pragma unroll
        for (int k = 0; k < PER_X; ++k) {
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
            if (Y) cs[tid + k * threads] = ldf(&cq[k]);
        }
#pragma unroll
        for (int k = 0; k < PER_X; ++k) xs[tid + k * threads] = ldf(&xq[k]);
        if (tid < m) {
            rate[tid] = make_float2(dq, expf(dq * Ah));
            if (!Y) fade = fmaf(dq, Ah * 1.4426950408889634f, fade);
        }
        __syncthreads();
        if (tb + TB < t1) fetch(tb + TB);
        auto token = [&](int t) -> float {                // one token; its output's part that this thread leaves
            const float2 da = rate[t], xv = *(const float2 *)(xs + t * R + r), a = make_float2(da.y, da.y);
            const float2 dx[2] = {make_float2(da.x * xv.x, da.x * xv.x), make_float2(da.x * xv.y, da.x * xv.y)};
            float2 acc[2][2];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                const float4 b = *(const float4 *)(bs + t * NP + (v * LPR + l) * 4);
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    S[j][v][0] = __ffma2_rn(a, S[j][v][0], __fmul2_rn(dx[j], make_float2(b.x, b.y)));
                    S[j][v][1] = __ffma2_rn(a, S[j][v][1], __fmul2_rn(dx[j], make_float2(b.z, b.w)));
                }
                if (Y) {
                    const float4 c = *(const float4 *)(cs + t * NP + (v * LPR + l) * 4);
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        acc[j][0] = v == 0 ? __fmul2_rn(S[j][v][0], make_float2(c.x, c.y)) : __ffma2_rn(S[j][v][0], make_float2(c.x, c.y), acc[j][0]);
                        acc[j][1] = v == 0 ? __fmul2_rn(S[j][v][1], make_float2(c.z, c.w)) : __ffma2_rn(S[j][v][1], make_float2(c.z, c.w), acc[j][1]);
                    }
                }
            }
            if (Y) {                                  // of two neighbours one keeps the first row's sum of both, the other the second's
                const float2 s0 = __fadd2_rn(acc[0][0], acc[0][1]), s1 = __fadd2_rn(acc[1][0], acc[1][1]);
                const float o0 = s0.x + s0.y, o1 = s1.x + s1.y;
                return (l & 1 ? o1 : o0) + __shfl_xor_sync(0xffffffffu, l & 1 ? o0 : o1, 1);
            }
            return 0.f;
        };
        auto part = [&](int t) -> float & { return ys[(t * R + r + (l & 1)) * PARTS + (l >> 1)]; };
        int tg = 0;
#pragma unroll 1
        for (; tg + TG <= m; tg += TG) {
            float out[TG];
#pragma unroll
            for (int u = 0; u < TG; ++u) out[u] = token(tg + u);
            if (Y)
#pragma unroll
                for (int u = 0; u < TG; ++u) part(tg + u) = out[u];
        }
#pragma unroll 1
        for (; tg < m; ++tg) {
            const float out = token(tg);
            if (Y) part(tg) = out;
        }
        __syncthreads();
        if (Y) {
#pragma unroll
            for (int k = 0; k < PER_X; ++k) {
                const int e = tid + k * threads, t = e / R, i = e % R;
                float sum;
                if constexpr (PARTS == 4) {
                    const float4 part = *(const float4 *)(ys + e * PARTS);
                    sum = (part.x + part.y) + (part.z + part.w);
                } else {
                    const float2 part = *(const float2 *)(ys + e * PARTS);
                    sum = part.x + part.y;
                }
                if (t < m && i0 + i < p) stf(y + ((size_t)(tb + t) * H + h) * p + i0 + i, Dskip ? fmaf(Dh, xs[e], sum) : sum);
            }
            __syncthreads();
        }
    }
    if (!Y && i0 == 0 && tid < 32) {
        fade = warp_sum(fade);
        if (tid == 0) faded[(size_t)s * H + h] = fade;
    }
    if (!final_state) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int col = (v * LPR + l) * 4;
            float *to = final_state + base + (size_t)j * n + col;
            if (i0 + r + j >= p || col >= n) continue;
            if (vec) *(float4 *)to = *(const float4 *)S[j][v];
            else {
                to[0] = S[j][v][0].x;
                if (col + 1 < n) to[1] = S[j][v][0].y;
                if (col + 2 < n) to[2] = S[j][v][1].x;
                if (col + 3 < n) to[3] = S[j][v][1].y;
            }
        }
}

// Arguments of a call, or of one of its two passes.
struct ScanCall {
    const str_ssd_packed_shape *s;                        // of the call; the pass has n_seq sequences
    int n_seq;
    const void *x, *B, *C;
    const float *dt, *A, *D;
    const int32_t *start;
    const float *state;
    void *y;
    float *final_state, *faded;
};
template <typename T, int NV, int LPR, int WARPS>
int launch(str_ctx *ctx, const ScanCall &k, cudaStream_t st) {
    const str_ssd_packed_shape *s = k.s;
    constexpr int TB = TOKENS<NV>, threads = 32 * WARPS, R = threads / LPR * 2;
    constexpr size_t smem = sizeof(float) * ((size_t)TB * (2 * NV * 4 * LPR + R + threads) + 2 * TB);
    auto *kernel = k.y ? scan_packed_kernel<T, NV, LPR, WARPS, true> : scan_packed_kernel<T, NV, LPR, WARPS, false>;
    if (smem > 48 * 1024) STR_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    kernel<<<dim3(ceil_div(s->p, R), s->H, k.n_seq), threads, smem, st>>>(k.n_seq, s->rows, s->H, s->p, s->n, s->G, (const T *)k.x, k.dt, k.A, (const T *)k.B, (const T *)k.C, k.D,
                                                                         k.start, k.state, (T *)k.y, k.final_state, k.faded, ctx->status_dev);
    return str_launch_ok(ctx);
}
// Blocks of 32 rows of a head, or of 64: four warps or eight, half of that where four lanes hold a row.
template <typename T>
int dispatch(str_ctx *ctx, const ScanCall &k, cudaStream_t st) {
    const int n = k.s->n;
#define SCAN(NV, LPR) (k.s->p <= 32 && NV < 8 ? launch<T, NV, LPR, LPR / 2>(ctx, k, st) : launch<T, NV, LPR, LPR>(ctx, k, st))
    return n <= 16 ? SCAN(1, 4) : n <= 32 ? SCAN(1, 8) : n <= 64 ? SCAN(2, 8) : n <= 128 ? SCAN(4, 8) : SCAN(8, 8);
#undef SCAN
}
int pass(str_ctx *ctx, const ScanCall &k, bool tc, cudaStream_t st) {
    if (tc) {
        str_ssd_packed_shape s = *k.s;
        s.n_seq = k.n_seq;
        return str_scan_packed_tc(ctx, &s, k.x, k.dt, k.A, k.B, k.C, k.D, k.start, k.state, k.y, k.final_state, k.faded, st);
    }
    return k.s->dtype == STR_BF16 ? dispatch<__nv_bfloat16>(ctx, k, st) : dispatch<float>(ctx, k, st);
}

// ---- long sequences of few heads ----------------------------------------------------------------
// A sequence is a chain of tokens, and few chains leave most SMs without work.  Then sequences are cut into segments of equal length: one pass forms every
// segment's state from zero, S <- 2^(sum of dt A) S + (that state) from segment to segment gives the states they start from, and a second pass
// forms the outputs.  Twice the work, in as many chains as there are segments.  How many is decided from the shape alone (the lengths are on the
// device), so that the workspace is known beforehand.
struct Segments {
    int len, n;                  // rows of one, number of them at most; len 0: sequences are walked whole
};
constexpr int SMS = 148;
Segments segments_of(const str_ssd_packed_shape *s) {
    const bool tc = str_scan_packed_tc_shape(s);
    // Blocks that run at a time, those of one sequence, and the shortest segment that is worth a pass (token by token 64 rows, 5 us: 24 heads of 32 x 20, one
    // sequence of 256 rows 18.8 us in fours, 21.9 whole; chunked 512 rows, of which a CTA's start and end are a third).
    const int rows_at_a_time = s->p <= 32 && s->n <= 128 ? 32 : 64;
    const long long room = tc ? SMS : s->n > 128 ? SMS : s->p > 32 ? 2 * SMS : 4 * SMS, least = tc ? 512 : 64;
    const long long per = (long long)s->H * (tc ? 1 : ceil_div(s->p, rows_at_a_time));
    const long long more = room / per - s->n_seq;         // segments beside the one that every sequence ends with
    if (more < 1) return {0, 0};
    const long long len = align_up((size_t)std::max<long long>((s->rows + more - 1) / more, least), tc ? 128 : 4);
    // Two passes over a segment against one over the sequence: two and a half segments are where they meet (chunked, 24 heads: one sequence of 2000 rows in 4
    // 44 us, whole 60).  Several sequences are seldom of one length, and the longest is what is waited for: there somewhat fewer on average will do (16 heads,
    // sequences of 20000, 3000 and 1000 rows 158 us, whole 365; two of 5000, 24 heads, 121, whole 101).
    if (s->n_seq == 1 ? 2LL * s->rows < 5 * len : 8LL * s->rows < 15 * len * s->n_seq) return {0, 0};
    return {(int)len, (int)(s->rows / len + s->n_seq)};
}
struct Workspace {
    float *states, *faded;       // [n][H][p][n], [n][H]
    int32_t *start, *first;      // [n + 1]: the segments' rows; [n_seq + 1]: the sequences' segments
    size_t bytes;
    Workspace(const str_ssd_packed_shape *s, const Segments &g, void *at) {
        const size_t states_bytes = (size_t)g.n * s->H * s->p * s->n * sizeof(float), faded_bytes = (size_t)g.n * s->H * sizeof(float);
        states = (float *)at;
        faded = (float *)((uint8_t *)at + states_bytes);
        start = (int32_t *)((uint8_t *)at + states_bytes + faded_bytes);
        first = start + g.n + 1;
        bytes = align_up(states_bytes + faded_bytes + sizeof(int32_t) * ((size_t)g.n + 1 + s->n_seq + 1), 256);
    }
};

// One block: the segments of all sequences, in their order.  (n_seq < 4 * SMS.)
__global__ void __launch_bounds__(1024) segments_kernel(int n_seq, int rows, Segments g, const int32_t *__restrict__ start, int32_t *__restrict__ seg_start,
                                                        int32_t *__restrict__ first, int *status) {
    __shared__ int upto[1024];
    packed_check(start, n_seq, rows, status);
    const int s = threadIdx.x;
    const int r0 = s < n_seq ? packed_start(start, s, rows) : 0, len = s < n_seq ? max(packed_start(start, s + 1, rows) - r0, 0) : 0;
    const int mine = min((len + g.len - 1) / g.len, g.n); // (fewer than g.n in all, unless the starts are wrong)
    upto[s] = mine;
    __syncthreads();
    for (int o = 1; o < 1024; o <<= 1) {
        const int v = s >= o ? upto[s - o] : 0;
        __syncthreads();
        upto[s] += v;
        __syncthreads();
    }
    const int all = min(upto[1023], g.n), at = upto[s] - mine, end = packed_start(start, n_seq, rows);
    if (s < n_seq) {
        first[s] = min(at, g.n);
        for (int j = 0; j < mine && at + j < g.n; ++j) seg_start[at + j] = r0 + j * g.len;
    }
    if (s == 0) first[n_seq] = all;
    for (int v = all + s; v <= g.n; v += 1024) seg_start[v] = end;
}

// The states that a sequence's segments start from, over those that they arrive at from zero; a thread VEC elements of one head's state.
template <int VEC>
__global__ void __launch_bounds__(256) segment_states_kernel(int H, int elements, const int32_t *__restrict__ first, const float *__restrict__ faded, const float *init_state,
                                                             float *__restrict__ states, float *final_state) {
    constexpr int AHEAD = 8;
    const int e = (blockIdx.x * 256 + threadIdx.x) * VEC, h = blockIdx.y, s = blockIdx.z;
    if (e >= elements) return;
    const int v0 = first[s], v1 = first[s + 1];
    const size_t at = ((size_t)s * H + h) * elements + e;
    alignas(16) float S[VEC], W[AHEAD][VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) S[i] = init_state ? init_state[at + i] : 0.f;
    for (int v = v0; v < v1; v += AHEAD) {
        float f[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (v + k < v1) {
                const float *w = states + ((size_t)(v + k) * H + h) * elements + e;
                if constexpr (VEC == 4) *(float4 *)W[k] = *(const float4 *)w;
                else W[k][0] = w[0];
                f[k] = exp2f(faded[(size_t)(v + k) * H + h]);
            }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k)
            if (v + k < v1) {
                float *w = states + ((size_t)(v + k) * H + h) * elements + e;
                if constexpr (VEC == 4) *(float4 *)w = *(const float4 *)S;
                else w[0] = S[0];
#pragma unroll
                for (int i = 0; i < VEC; ++i) S[i] = fmaf(f[k], S[i], W[k][i]);
            }
    }
    if (final_state)
#pragma unroll
        for (int i = 0; i < VEC; ++i) final_state[at + i] = S[i];
}

int in_segments(str_ctx *ctx, const ScanCall &k, const Segments &g, void *workspace, bool tc, cudaStream_t st) {
    const str_ssd_packed_shape *s = k.s;
    const Workspace w(s, g, workspace);
    segments_kernel<<<1, 1024, 0, st>>>(s->n_seq, s->rows, g, k.start, w.start, w.first, ctx->status_dev);
    int rc = str_launch_ok(ctx);
    ScanCall states = k, outputs = k;
    states.n_seq = outputs.n_seq = g.n;
    states.start = outputs.start = w.start;
    states.state = nullptr, states.final_state = w.states, states.faded = w.faded, states.y = nullptr;
    outputs.state = w.states, outputs.final_state = nullptr;
    if (rc == STR_OK) rc = pass(ctx, states, tc, st);
    if (rc != STR_OK) return rc;
    const int elements = s->p * s->n;
    if (elements % 4 == 0)
        segment_states_kernel<4><<<dim3(ceil_div(elements, 1024), s->H, s->n_seq), 256, 0, st>>>(s->H, elements, w.first, w.faded, k.state, w.states, k.final_state);
    else
        segment_states_kernel<1><<<dim3(ceil_div(elements, 256), s->H, s->n_seq), 256, 0, st>>>(s->H, elements, w.first, w.faded, k.state, w.states, k.final_state);
    rc = str_launch_ok(ctx);
    return rc == STR_OK ? pass(ctx, outputs, tc, st) : rc;
}

}  // namespace

extern "C" size_t str_mamba2_prefill_packed_workspace_size(const str_ssd_packed_shape *s) {
    if (!s || s->n_seq <= 0 || s->rows <= 0 || s->H <= 0 || s->p <= 0 || s->n <= 0 || s->n > 256 || s->p > (1 << 20)) return 0;
    const Segments g = segments_of(s);
    return g.len ? Workspace(s, g, nullptr).bytes : 0;
}

extern "C" int str_mamba2_prefill_packed(str_ctx *ctx, const str_ssd_packed_shape *s, const void *x, const float *dt, const float *A, const void *B,
                                         const void *C, const float *D, const int32_t *seq_start, const float *init_state, void *y,
                                         float *final_state, void *workspace, size_t workspace_bytes, void *stream) {
    if (!ctx || !s || !A || !seq_start) return STR_ERR_INVALID_ARG;
    if (s->n_seq <= 0 || s->rows < 0 || s->H <= 0 || s->p <= 0 || s->n <= 0 || s->G <= 0 || s->H % s->G != 0 ||
        (s->dtype != STR_F32 && s->dtype != STR_BF16))
        return STR_ERR_INVALID_ARG;
    if (s->rows > 0 && (!x || !dt || !B || !C || !y)) return STR_ERR_INVALID_ARG;
    if (s->n > 256 || s->n_seq > 65535 || s->H > 65535 || s->rows > (1 << 30) || s->p > (1 << 20)) return STR_ERR_UNSUPPORTED_SHAPE;
    const size_t state_bytes = (size_t)s->n_seq * s->H * s->p * s->n * sizeof(float), es = dtype_size(s->dtype);
    const size_t xb = (size_t)s->rows * s->H * s->p * es, bb = (size_t)s->rows * s->G * s->n * es;
    const size_t need = str_mamba2_prefill_packed_workspace_size(s), db = (size_t)s->rows * s->H * sizeof(float), hb = s->H * sizeof(float);
    if (workspace_bytes < need) return STR_ERR_WORKSPACE_TOO_SMALL;
    if (need && (!workspace || ((uintptr_t)workspace & 255) != 0)) return STR_ERR_INVALID_ARG;
    // What is written against what is read, and against one another; a state may be updated where it lies.
    const struct { const void *at; size_t bytes; } in[] = {{x, xb}, {dt, db}, {A, hb}, {B, bb}, {C, bb}, {D, hb}, {seq_start, ((size_t)s->n_seq + 1) * sizeof(int32_t)},
                                                           {init_state, state_bytes}},
        out[] = {{y, xb}, {final_state, state_bytes}, {workspace, need}};
    for (const auto &o : out)
        for (const auto &i : in)
            if (kv4_overlap(i.at, i.bytes, o.at, o.bytes) && !(&i == in + 7 && &o == out + 1 && init_state == final_state)) return STR_ERR_INVALID_ARG;
    for (int i = 0; i < 3; ++i)
        if (kv4_overlap(out[i].at, out[i].bytes, out[(i + 1) % 3].at, out[(i + 1) % 3].bytes)) return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_SSD, stream);
    cudaStream_t st = (cudaStream_t)stream;
    // The chunked kernel's CTAs cost what a chunk of 128 rows costs however few there are.  Sequences of 32 rows on average are where the two meet (128 heads of
    // 64 x 128: one sequence of 32 rows 10.3 us token by token, 10.4 chunked, of 64 rows 17.9 and 10.6; 33 sequences of 32 rows 204 and 276, of 64 rows 387 and
    // 277; 24 heads of 32 x 64: one of 32 rows 5.5 and 9.2).
    const bool tc = !str_force_simt() && s->rows > 32LL * s->n_seq && str_scan_packed_tc_supported(s, x, B, C, y);
    ++(tc ? ctx->tc_calls : ctx->fallback_calls);
    const ScanCall call = {s, s->n_seq, x, B, C, dt, A, D, seq_start, init_state, y, final_state, nullptr};
    return need ? in_segments(ctx, call, segments_of(s), workspace, tc, st) : pass(ctx, call, tc, st);
}

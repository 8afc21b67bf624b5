// The scan over packed sequences on tcgen05 tensor cores (bf16 in, fp32 accumulate): head dim p <= 64, state dim n <= 128, both multiples of 8 and
// padded with zeros by the tensor maps.  The chunked form of ssd_tc.cu, in which the decomposition, its decay factors (each formed from a
// difference of cumulative sums that is <= 0) and the pipeline are described; what is different here:
//   sequences   One CTA per (sequence, head) walks its own rows; longer sequences start first.  Rows behind the sequence in its last chunk belong to
//               others: their dt counts as zero and their rows of X and B are zeroed in shared memory, as zero times what stands there need not be zero.
//   states      The state starts from init_state; its bf16 copy is written before the first chunk, so Y_inter exists for every chunk.
//   D skip      D_h is added to the diagonal of W: Y_intra = (W + D_h I) X.
//   accuracy    The final state is an fp32 result.  Xs_j = exp(l_end - l_j) dt_j x_j is formed to 16 bits and enters the tensor pipe as two bf16
//               pieces, Xs + Xs', relative error 2^-16 instead of 2^-8, and l_end - l_j as a sum from the end of the chunk, not as a difference.
//               A third piece brings it to 2^-24 in the last chunk and in those that the rest of the sequence fades by less than 2^-4; what
//               lies further back is faded with its error.
//               y is bf16 itself: W and the state's copy are narrowed once, relative error 2^-8 of each term at most, random in sign.
//               Xs' has no buffer of its own: it takes the X slot of the chunk before, once that chunk's Y_intra is complete and until the
//               chunk after next is loaded there.
//   not finite  W is zero above the diagonal, and zero times infinity or NaN is NaN: an x that is not finite would reach the up to 127 tokens
//               before it.  It also makes the state infinite or NaN, to the end: a CTA whose state ends so runs its sequence anew token by token
//               (scan_rows).
// Warp roles: 0-3, 14, 15 W; 4-7 Xs, Xs' and the state; 8-11 epilogue; 12 decay vectors and TMA producer; 13 MMA issuer; iteration c
// issues CB_c, Y_intra_{c-1}, Y_inter_c, dS_c in halves of 64 tokens, as soon as these are there, and dS'_c.  The chain from chunk to chunk is
// dS -> state (and its copy) -> Xs -> dS; the state warps, who wait for dS anyhow, form Xs, so that no other role's work lies on it (formed by
// the epilogue's warps, in front of each epilogue, it took 4400 clocks a chunk).
//
// Measured: eight sequences of 24576 rows, 128 heads: 451 us, 2.2 TB/s, 0.33 of the measured copy bandwidth (497 to 508 with inputs that change from call to call); one sequence of 32896
// rows 606 us, 2.36 us (4300 clocks) a chunk; a turn of 300 rows 16 us.  With decays so slow that every chunk takes the third piece 689 and 1020 us.  Bound by shared memory: of a chunk's clocks its 128 bytes a clock are busy for about 3500 (operands of
// the products 1750, tiles coming in 640, the warps' own accesses 1130), and the stores of y, 32 rows a warp, hold the load/store units for 800 more.
// The two pieces of x cost 0.5 us a chunk over one.  The loops are rolled wherever registers allow: with the pieces of W unrolled the instruction cache
// no longer held the roles, and the same work took 527 us.
// All mbarrier waits are bounded; a give-up records STR_ERR_TIMEOUT and tears the CTA down.
#include "dispatch.cuh"
#include "packed.cuh"
#include "tc_common.cuh"

namespace {

constexpr int Q = 128, P = 64, NS = 128;
constexpr int TILE_16K = 16384;
constexpr int X_SLOTS = 3, DEC_DEPTH = 4, DEC_FLOATS = 928;
constexpr int OFF_X = 0;                                  // 3 x 16 KB
constexpr int OFF_B = OFF_X + X_SLOTS * TILE_16K;         // 2 x 32 KB
constexpr int OFF_C = OFF_B + 4 * TILE_16K;               // 2 x 32 KB
constexpr int OFF_XS = OFF_C + 4 * TILE_16K;              // 16 KB
constexpr int OFF_SB = OFF_XS + TILE_16K;                 // 16 KB
constexpr int OFF_DEC = OFF_SB + TILE_16K;                // 4 x 3712 B
constexpr int OFF_MASK = OFF_DEC + DEC_DEPTH * DEC_FLOATS * 4;   // 2 KB: which pairs of columns of a 32 x 32 block lie on or below its diagonal
constexpr int OFF_BARS = OFF_MASK + 2048;
// decay vectors of one chunk (floats): log2-domain cumulative decay l_j, log2(dt_j) - l_j, column / state / row factors
constexpr int D_LS = 0, D_NLC = 128, D_COLF = 256, D_XW = 384, D_ROWF = 640, D_EROW = 768, D_BLK = 896, D_EEND = 912;
enum {
    B_XF = 0, B_BCF = 3, B_DECF = 5, B_DECE = 9, B_CBF = 13, B_WF = 15, B_XSF = 17, B_DSF = 19, B_DSE = 21,
    B_SF, B_YF, B_YE, B_XLF, B_HIF, B_X3F, B_FINE, B_COUNT
};
constexpr size_t SMEM_BYTES = (size_t)OFF_BARS + B_COUNT * 8 + 40;
constexpr int NUM_WARPS = 16, NUM_THREADS = NUM_WARPS * 32;
constexpr int W_WARPS = 6;
constexpr int DEC_READERS = W_WARPS + 4 + 4;              // warps that read a chunk's decay vectors
constexpr uint32_t TM_CB = 0, TM_YO = 256, TM_YI = 384, TM_DS = 448;
constexpr float LOG2E = 1.4426950408889634f;
constexpr float FADED = 4.0f;                             // a chunk takes the third piece unless what is behind it fades it by this many powers of two

// Sixteen fp32 values of a row as bf16: one 32-byte store where the row has room and its address allows it.
__device__ __forceinline__ void store16(__nv_bfloat16 *to, const uint32_t *v, int room, bool wide) {
    uint32_t w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = tc::pack_bf16x2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
    if (wide && room >= 16) {
        asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
                     : "memory");
    } else {
        if (room >= 8) *(uint4 *)to = make_uint4(w[0], w[1], w[2], w[3]);
        if (room >= 16) *(uint4 *)(to + 8) = make_uint4(w[4], w[5], w[6], w[7]);
    }
}
__device__ __forceinline__ void warp_arrive(uint64_t *bar, int lane) {
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar);
}

// The state warps among themselves.
__device__ __forceinline__ void state_warps_sync() { asm volatile("barrier.sync 1, 128;" ::: "memory"); }

// Descriptor arithmetic: the 14-bit start-address field holds (shared address >> 4); every operand of
// this kernel lies below 256 KB, so adding a byte offset >> 4 to the descriptor never carries out of it.
__device__ __forceinline__ uint64_t desc_add(uint64_t d, uint32_t bytes) { return d + (uint64_t)(bytes >> 4); }
// Half (64 tokens) of Xs and Xs' of one chunk (same swizzled layout as the X tile), 128 threads, four 16-byte units each.  The factor comes as two
// bf16 pieces, w = w1 + w2 to 2^-17; hi = bf16(w1 x), whose rounding error w1 x - hi is itself a bf16 number, and lo = bf16(w2 x + that error): hi + lo is
// w x to 2^-16, in three packed instructions a pair.  lo stays in registers until its place is free.  A token's factor: w1 and w2 in the halves of one
// word, w itself in the next.  Rows from `valid` on are another sequence's: zeroed, in the X tile too.
__device__ __forceinline__ void split_x(uint8_t *x_tile, uint8_t *hi_tile, uint4 (&lo)[4], const float *dec_xw, int tid_g, int half, int valid) {
    uint4 v[4];
    uint2 w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int u = tid_g + 128 * (4 * half + i);
        v[i] = ((const uint4 *)x_tile)[u];
        w[i] = ((const uint2 *)dec_xw)[u >> 3];
    }
    if (valid < Q)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int u = tid_g + 128 * (4 * half + i);
            if ((u >> 3) >= valid) ((uint4 *)x_tile)[u] = v[i] = make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int u = tid_g + 128 * (4 * half + i);
        const uint32_t w11 = __byte_perm(w[i].x, 0, 0x1010), w22 = __byte_perm(w[i].x, 0, 0x3232);
        const __nv_bfloat162 w1 = *reinterpret_cast<const __nv_bfloat162 *>(&w11), w2 = *reinterpret_cast<const __nv_bfloat162 *>(&w22);
        __nv_bfloat162 *x = reinterpret_cast<__nv_bfloat162 *>(&v[i]);
        __nv_bfloat162 *l = reinterpret_cast<__nv_bfloat162 *>(&lo[i]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __hmul2(x[j], w1);
            l[j] = __hfma2(x[j], w2, __hfma2(x[j], w1, __hneg2(h)));
            x[j] = h;
        }
        ((uint4 *)hi_tile)[u] = v[i];
    }
}

// The third piece, bf16(w x - hi - lo) with the product in fp32, over hi once its product is through: w x to 2^-24.
__device__ __forceinline__ void third_x(const uint8_t *x_tile, uint8_t *hi_tile, const float *dec_xw, int tid_g) {
#pragma unroll 1
    for (int i = 0; i < 8; ++i) {
        const int u = tid_g + 128 * i;
        const uint4 v = ((const uint4 *)x_tile)[u];
        const uint2 w = ((const uint2 *)dec_xw)[u >> 3];
        const uint32_t w11 = __byte_perm(w.x, 0, 0x1010), w22 = __byte_perm(w.x, 0, 0x3232);
        const __nv_bfloat162 w1 = *reinterpret_cast<const __nv_bfloat162 *>(&w11), w2 = *reinterpret_cast<const __nv_bfloat162 *>(&w22);
        const __nv_bfloat162 *x = reinterpret_cast<const __nv_bfloat162 *>(&v);
        uint32_t r[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const __nv_bfloat162 h = __hmul2(x[j], w1), l = __hfma2(x[j], w2, __hfma2(x[j], w1, __hneg2(h)));
            const float wf = __uint_as_float(w.y);
            r[j] = tc::pack_bf16x2(fmaf(__low2float(x[j]), wf, -__low2float(h)) - __low2float(l), fmaf(__high2float(x[j]), wf, -__high2float(h)) - __high2float(l));
        }
        ((uint4 *)hi_tile)[u] = make_uint4(r[0], r[1], r[2], r[3]);
    }
}

// One 16-column piece of W = CB o decay for this thread's token row: fp32 CB values in, eight packed bf16 pairs out.
// Diagonal 32x32 block: one exponential per element, exp2(l_t + (log2 dt_j - l_j)).  Above the diagonal anything may come of it (infinities, and NaN where B
// is not finite): those elements are cleared as bits.  D is added to the pair that holds this row's diagonal element.
__device__ __forceinline__ void w_piece_diag(const uint32_t (&v)[16], uint32_t (&packed)[8], const float *dec, const uint4 *mask, int col0, int lane, float l_t, float2 skip) {
    const float2 lt2 = make_float2(l_t, l_t);
    const int pair0 = (col0 & 31) >> 1;
#pragma unroll
    for (int i4 = 0; i4 < 2; ++i4) {
        const uint4 m4 = mask[(pair0 / 4 + i4) * 32 + lane];
        const uint32_t m[4] = {m4.x, m4.y, m4.z, m4.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i2 = 4 * i4 + k;
            const float2 a = __fadd2_rn(lt2, *(const float2 *)(dec + D_NLC + col0 + 2 * i2));
            float2 w = __fmul2_rn(make_float2(__uint_as_float(v[2 * i2]), __uint_as_float(v[2 * i2 + 1])), make_float2(tc::ex2(a.x), tc::ex2(a.y)));
            if ((lane >> 1) == pair0 + i2) w = __fadd2_rn(w, skip);
            packed[i2] = tc::pack_bf16x2(w.x, w.y) & m[k];
        }
    }
}
// Block below the diagonal: exp(l_t - l_j) dt_j = f (row part times block-pair scalar) * column part, each <= 1.
__device__ __forceinline__ void w_piece_below(const uint32_t (&v)[16], uint32_t (&packed)[8], const float *dec, int col0, float f) {
    const float2 ff = make_float2(f, f);
#pragma unroll
    for (int i4 = 0; i4 < 4; ++i4) {
        const float4 cf = *(const float4 *)(dec + D_COLF + col0 + 4 * i4);
        const float2 r01 = __fmul2_rn(make_float2(__uint_as_float(v[4 * i4]), __uint_as_float(v[4 * i4 + 1])), __fmul2_rn(ff, make_float2(cf.x, cf.y)));
        const float2 r23 = __fmul2_rn(make_float2(__uint_as_float(v[4 * i4 + 2]), __uint_as_float(v[4 * i4 + 3])), __fmul2_rn(ff, make_float2(cf.z, cf.w)));
        packed[2 * i4] = tc::pack_bf16x2(r01.x, r01.y);
        packed[2 * i4 + 1] = tc::pack_bf16x2(r23.x, r23.y);
    }
}

// The recurrence of one head of one sequence token by token, in fp32, by the whole CTA: eight lanes a row of the state (one of p).
__device__ __noinline__ void scan_rows(const __nv_bfloat16 *x, const float *dt, float A, const __nv_bfloat16 *B, const __nv_bfloat16 *C, const float *D, const float *init,
                                       __nv_bfloat16 *y, float *fin, int T, int H, int G, int p, int n) {
    const int r = threadIdx.x / 8, l = threadIdx.x % 8;
    float S[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) S[i] = init && r < p && l + 8 * i < n ? init[(size_t)r * n + l + 8 * i] : 0.f;
    for (int t = 0; t < T; ++t) {
        const float d = dt[(size_t)t * H], a = expf(d * A), xv = r < p ? ldf(x + (size_t)t * H * p + r) : 0.f;
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (l + 8 * i < n) {
                S[i] = fmaf(a, S[i], d * xv * ldf(B + (size_t)t * G * n + l + 8 * i));
                sum = fmaf(S[i], ldf(C + (size_t)t * G * n + l + 8 * i), sum);
            }
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
        if (y && l == 0 && r < p) stf(y + (size_t)t * H * p + r, D ? fmaf(*D, xv, sum) : sum);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (fin && r < p && l + 8 * i < n) fin[(size_t)r * n + l + 8 * i] = S[i];
}

// Sequence whose length is number `rank` in descending order (equal lengths by index), found by counting; the whole CTA.  Beyond RANKED sequences
// the counting would cost more than the order gives: then they are taken as they come.
constexpr int RANKED = NUM_THREADS;
__device__ __forceinline__ int packed_by_length(const int32_t *start, int n_seq, int rows, int rank, int *slot) {
    if (n_seq > RANKED) return rank;
    const int s = threadIdx.x;
    if (s < n_seq) {
        const int len = max(packed_start(start, s + 1, rows) - packed_start(start, s, rows), 0);
        int before = 0;
        for (int i = 0; i < n_seq; ++i) {
            const int li = max(packed_start(start, i + 1, rows) - packed_start(start, i, rows), 0);
            before += li > len || (li == len && i < s);
        }
        if (before == rank) *slot = s;
    }
    __syncthreads();
    return *slot;
}

__global__ void __launch_bounds__(NUM_THREADS, 1)
scan_packed_tc_kernel(const __grid_constant__ CUtensorMap tmap_x, const __grid_constant__ CUtensorMap tmap_b,
                      const __grid_constant__ CUtensorMap tmap_c, int n_seq, int rows, int H, int p, int n, int G, const float *__restrict__ dt,
                      const float *__restrict__ A, const float *__restrict__ Dskip, const int32_t *__restrict__ start, const __nv_bfloat16 *__restrict__ x,
                      const __nv_bfloat16 *__restrict__ B, const __nv_bfloat16 *__restrict__ C, const float *init_state, __nv_bfloat16 *__restrict__ y,
                      float *final_state, float *__restrict__ faded, int *status) {
    extern __shared__ __align__(1024) uint8_t smem[];
    float *decs = (float *)(smem + OFF_DEC);
    uint64_t *bars = (uint64_t *)(smem + OFF_BARS);
    uint32_t *tmem_slot = (uint32_t *)(bars + B_COUNT);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);       // [2]
    volatile int *found = abort_flag + 2;                             // the state is not finite
    volatile int *fine_from = (volatile int *)(tmem_slot + 5);        // the chunks from here on take the third piece

    // Role numbers (the `warp` used below) are decoupled from hardware warp numbers: when several warps of a
    // scheduler are ready it favours the lower-numbered one, so the MMA issuer and the decay warp, which need
    // few issue slots but need them promptly, take hardware warps 0 and 1 and the instruction-heavy W roles
    // the highest numbers.  Roles that touch tensor memory keep role % 4 == hardware warp % 4 (lane quadrant).
    const int hw_warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int warp = hw_warp < 2 ? 13 - hw_warp : hw_warp < 4 ? hw_warp + 12 : hw_warp < 12 ? hw_warp : hw_warp - 12;
    const int h = blockIdx.x % H, g = h / (H / G);

    if ((tc::smem_u32(smem) & 1023u) != 0) {          // swizzled tiles need a 1024-byte aligned base
        if (threadIdx.x == 0) atomicCAS(status, 0, STR_ERR_CUDA);
        return;
    }
    if (tc::cta_should_leave(status)) return;     // an earlier CTA failed: the whole CTA leaves at once
    if (blockIdx.x == 0) packed_check(start, n_seq, rows, status);
    const int b = packed_by_length(start, n_seq, rows, blockIdx.x / H, (int *)(tmem_slot + 4));
    const int row0 = packed_start(start, b, rows), Tlen = max(packed_start(start, b + 1, rows) - row0, 0);
    const int nchunks = (Tlen + Q - 1) / Q;
    const float *init = init_state ? init_state + ((size_t)b * H + h) * p * n : nullptr;
    float *fin = final_state ? final_state + ((size_t)b * H + h) * p * n : nullptr;
    if (nchunks == 0) {
        if (faded && threadIdx.x == 0) faded[(size_t)b * H + h] = 0.f;
        if (fin && fin != init)
            for (int e = threadIdx.x; e < p * n; e += NUM_THREADS) fin[e] = init ? init[e] : 0.f;
        return;
    }
    const float skip = Dskip ? Dskip[h] : 0.f;
    if (threadIdx.x == 0) {
        for (int i = 0; i < X_SLOTS; ++i) tc::mbar_init(bars + B_XF + i, 1);
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(bars + B_BCF + i, 1);
            tc::mbar_init(bars + B_CBF + i, 1); tc::mbar_init(bars + B_WF + i, W_WARPS);
        }
        for (int i = 0; i < DEC_DEPTH; ++i) { tc::mbar_init(bars + B_DECF + i, 1); tc::mbar_init(bars + B_DECE + i, DEC_READERS); }
        tc::mbar_init(bars + B_XSF, 4); tc::mbar_init(bars + B_XSF + 1, 4); tc::mbar_init(bars + B_DSF, 1); tc::mbar_init(bars + B_DSF + 1, 1); tc::mbar_init(bars + B_DSE, 4);
        tc::mbar_init(bars + B_SF, 4); tc::mbar_init(bars + B_YF, 1); tc::mbar_init(bars + B_YE, 4); tc::mbar_init(bars + B_XLF, 4);
        tc::mbar_init(bars + B_HIF, 1); tc::mbar_init(bars + B_X3F, 4); tc::mbar_init(bars + B_FINE, 1);
        abort_flag[0] = 0; abort_flag[1] = 0; found[0] = 0;
        tc::fence_mbar_init();
        tc::prefetch_tmap(&tmap_x); tc::prefetch_tmap(&tmap_b); tc::prefetch_tmap(&tmap_c);
    }
    {
        const int k = threadIdx.x >> 5;               // pair of columns 2k, 2k + 1 of a block, against row `lane`
        ((uint32_t *)(smem + OFF_MASK))[((k >> 2) * 32 + lane) * 4 + (k & 3)] = (2 * k <= lane ? 0xFFFFu : 0u) | (2 * k + 1 <= lane ? 0xFFFF0000u : 0u);
    }
    if (warp == 13) { tc::tmem_alloc(tmem_slot, 512); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp == 12) {
        // ------------------------------------------------------------------ decay vectors
        const float Ah2 = A[h] * LOG2E;
        // A token that fades what lies before it by 2^-256 leaves nothing of it, and counts as no more: the chunk's sums stay above -2^15, so that their
        // differences are right to 2^-9 however fast the decay (at -2^21 the weight of a token's own x would be 6 % off).
        const float longest = Ah2 < 0.f ? -256.f / Ah2 : INFINITY;
        const float *dtb = dt + (size_t)row0 * H + h;
        bool ok = true;
        // Lane 0 is the TMA producer too.  The operands of chunk c go into the slots of chunk c-2 (B, C: ring of 2) and chunk c-3 (X: ring of 3)
        // once dS_{c-2} is seen complete: the tensor pipe runs in order, so CB_{c-2}, Y_inter_{c-2}, Y_intra_{c-3} and both products with the
        // pieces of chunk c-2, one of which lay in that X slot, are complete too.  No slot-release barriers are needed.  (Two barriers for dS in turn: the next arrival on the one
        // waited for is that of chunk c itself, so it cannot be passed over.)
        int n_loaded = 0;
        auto load_chunk = [&](int c) {
            const int t0 = row0 + c * Q, s = c & 1, sx = c % X_SLOTS;
            uint64_t *fb = bars + B_BCF + s;
            tc::mbar_arrive_expect_tx(fb, 4 * TILE_16K);
            tc::tma_load_3d(smem + OFF_B + (s * 2) * TILE_16K, &tmap_b, fb, 0, g, t0);
            tc::tma_load_3d(smem + OFF_B + (s * 2 + 1) * TILE_16K, &tmap_b, fb, 64, g, t0);
            tc::tma_load_3d(smem + OFF_C + (s * 2) * TILE_16K, &tmap_c, fb, 0, g, t0);
            tc::tma_load_3d(smem + OFF_C + (s * 2 + 1) * TILE_16K, &tmap_c, fb, 64, g, t0);
            tc::mbar_arrive_expect_tx(bars + B_XF + sx, TILE_16K);
            tc::tma_load_3d(smem + OFF_X + sx * TILE_16K, &tmap_x, bars + B_XF + sx, 0, h, t0);
            ++n_loaded;
        };
        if (lane == 0) {
            load_chunk(0);
            if (nchunks > 1) load_chunk(1);
        }
        __syncwarp();
        float dv[4], dn[4], fade = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) dn[i] = (4 * lane + i < Tlen) ? __ldg(dtb + (size_t)(4 * lane + i) * H) : 0.f;
#pragma unroll 1
        for (int c = 0; c < nchunks; ++c) {
            const int d = c & (DEC_DEPTH - 1);
#pragma unroll
            for (int i = 0; i < 4; ++i) {             // this chunk's dt was fetched one iteration ago
                dv[i] = dn[i];
                const int t = (c + 1) * Q + 4 * lane + i;
                dn[i] = t < Tlen ? __ldg(dtb + (size_t)t * H) : 0.f;
            }
            if (!tc::mbar_wait(bars + B_DECE + d, ((c >> 2) & 1) ^ 1, abort_flag)) { ok = false; break; }
            float l[4], dl[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) dl[i] = dv[i] > longest ? longest : dv[i];          // (NaN stays)
            l[0] = dl[0] * Ah2;
#pragma unroll
            for (int i = 1; i < 4; ++i) l[i] = fmaf(dl[i], Ah2, l[i - 1]);
            float incl = l[3];
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const float excl = incl - l[3];
            const float l_start = __shfl_sync(0xffffffffu, excl, lane & ~7);     // start of this 32-token block
            const float l_endb = __shfl_sync(0xffffffffu, incl, lane | 7);       // end of this 32-token block
            const float l_end = __shfl_sync(0xffffffffu, incl, 31);
            fade += l_end;
            // sums over what comes behind a token: what l_end - l_j is, without the difference of two large numbers
            float tail[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 2; i >= 0; --i) tail[i] = fmaf(dl[i + 1], Ah2, tail[i + 1]);
            float rev = fmaf(dl[0], Ah2, tail[0]);                    // the lane's four tokens together
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const float v = __shfl_down_sync(0xffffffffu, rev, o);
                if (lane + o < 32) rev += v;
            }
            const float next = __shfl_down_sync(0xffffffffu, rev, 1), behind = lane == 31 ? 0.f : next;
            // blk[bt][bj] = exp(l_start(bt) - l_endblock(bj)), bj < bt; lanes 0..15 hold (bt, bj) = (lane/4, lane%4)
            const float bs = __shfl_sync(0xffffffffu, excl, ((lane >> 2) & 3) * 8);
            const float be = __shfl_sync(0xffffffffu, incl, (lane & 3) * 8 + 7);
            float *dec = decs + d * DEC_FLOATS;
            float o_ls[4], o_nlc[4], o_colf[4], o_rowf[4], o_erow[4];
            uint32_t o_xw[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float li = excl + l[i];
                o_ls[i] = li;
                o_nlc[i] = tc::lg2(dv[i]) - li;          // exp2(l_t + nlc_j) = exp(l_t - l_j) dt_j; a padded token (dt = 0) gives -inf
                o_colf[i] = tc::ex2(l_endb - li) * dv[i];
                const float xw = tc::ex2(behind + tail[i]) * dv[i];
                const float w1 = __bfloat162float(__float2bfloat16_rn(xw));
                o_xw[2 * i] = tc::pack_bf16x2(xw, xw - w1);
                o_xw[2 * i + 1] = __float_as_uint(xw);
                o_rowf[i] = tc::ex2(li - l_start);
                o_erow[i] = tc::ex2(li);
            }
            *(float4 *)(dec + D_LS + 4 * lane) = make_float4(o_ls[0], o_ls[1], o_ls[2], o_ls[3]);
            *(float4 *)(dec + D_NLC + 4 * lane) = make_float4(o_nlc[0], o_nlc[1], o_nlc[2], o_nlc[3]);
            *(float4 *)(dec + D_COLF + 4 * lane) = make_float4(o_colf[0], o_colf[1], o_colf[2], o_colf[3]);
            *(uint4 *)(dec + D_XW + 8 * lane) = make_uint4(o_xw[0], o_xw[1], o_xw[2], o_xw[3]);
            *(uint4 *)(dec + D_XW + 8 * lane + 4) = make_uint4(o_xw[4], o_xw[5], o_xw[6], o_xw[7]);
            *(float4 *)(dec + D_ROWF + 4 * lane) = make_float4(o_rowf[0], o_rowf[1], o_rowf[2], o_rowf[3]);
            *(float4 *)(dec + D_EROW + 4 * lane) = make_float4(o_erow[0], o_erow[1], o_erow[2], o_erow[3]);
            if (lane < 16) dec[D_BLK + lane] = ((lane & 3) < (lane >> 2)) ? tc::ex2(bs - be) : 0.f;
            if (lane == 0) dec[D_EEND] = tc::ex2(l_end);
            warp_arrive(bars + B_DECF + d, lane);
            if (c >= 2) {
                if (!tc::mbar_wait(bars + B_DSF + (c & 1), ((c - 2) >> 1) & 1, abort_flag)) { ok = false; break; }
                if (lane == 0) load_chunk(c);
                __syncwarp();
            }
        }
        if (faded && lane == 0) faded[(size_t)b * H + h] = fade;
        if (!ok && lane == 0) {
            atomicCAS(status, 0, STR_ERR_TIMEOUT);
            for (int back = 1; back <= 2 && back <= n_loaded; ++back) {       // let copies already issued land before the CTA goes away
                const int j = n_loaded - back;
                tc::mbar_wait(bars + B_BCF + (j & 1), (j >> 1) & 1, abort_flag + 1);
                tc::mbar_wait(bars + B_XF + j % X_SLOTS, (j / X_SLOTS) & 1, abort_flag + 1);
            }
        }
    } else if (warp == 13) {
        // ------------------------------------------------------------------ MMA issuer
        // One elected thread runs the whole loop (the region is entered once, so the compiler knows it to be
        // single-threaded) and issues every product as one straight-line block of eight tcgen05.mma: issued any
        // other way the products cost two to five times the tensor pipe's own time as soon as the arithmetic
        // warps of this scheduler are busy.  Product order per iteration: CB_c, Y_intra_{c-1}, Y_inter_c, dS_c, dS'_c.
        if (tc::elect_one()) {
            const uint32_t id_cb = tc::make_idesc_bf16(128, 128, 0, 0);   // C (K-major) x B (K-major)
            const uint32_t id_kn = tc::make_idesc_bf16(128, 64, 0, 1);    // K-major / tensor-memory A x MN-major B
            const uint32_t id_nn = tc::make_idesc_bf16(128, 64, 1, 1);    // MN-major A x MN-major B
            const uint32_t sbase = tc::smem_u32(smem);
            const uint64_t dk_c0 = tc::desc_kmajor_sw128(sbase + OFF_C, 0), dk_b0 = tc::desc_kmajor_sw128(sbase + OFF_B, 0);
            const uint64_t dm_b0 = tc::make_smem_desc(sbase + OFF_B, TILE_16K, 1024, tc::SWZ_128B);
            const uint64_t dm_xs = tc::make_smem_desc(sbase + OFF_XS, TILE_16K, 1024, tc::SWZ_128B);
            const uint64_t dm_sb = tc::make_smem_desc(sbase + OFF_SB, TILE_16K, 1024, tc::SWZ_128B);
            const uint64_t dm_x0 = tc::make_smem_desc(sbase + OFF_X, TILE_16K, 1024, tc::SWZ_128B);
            bool ok = tc::mbar_wait(bars + B_FINE, 0, abort_flag);
            const int fine_c = ok ? fine_from[0] : 0;
            int n_fine = 0;
#pragma unroll 1
            for (int c = 0; c <= nchunks && ok; ++c) {
                const int s = c & 1;
                const uint64_t dk_c = desc_add(dk_c0, (uint32_t)s * 2 * TILE_16K), dk_b = desc_add(dk_b0, (uint32_t)s * 2 * TILE_16K);
                if (c < nchunks) {
                    ok = tc::mbar_wait(bars + B_BCF + s, (c >> 1) & 1, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    tc::mma8_ss<tc::StepKMajor2x64, tc::StepKMajor2x64>(tmem + TM_CB + (uint32_t)s * 128, dk_c, dk_b, id_cb, false);   // CB_c = C B^T
                    tc::mma_commit(bars + B_CBF + s);
                }
                if (c >= 1) {
                    const int cp = c - 1, sp = cp & 1;
                    // the epilogue has read the Y accumulators of chunk c-2; W_{c-1} is in tensor memory
                    ok = (c < 2 || tc::mbar_wait(bars + B_YE, (c - 2) & 1, abort_flag)) &&
                         tc::mbar_wait(bars + B_WF + sp, (cp >> 1) & 1, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    // Y_intra_{c-1} = W X; K-slice ks of W sits in columns [16 ks, 16 ks + 8)
                    tc::mma8_ts<tc::StepTmem16, tc::StepMNMajor>(tmem + TM_YI, tmem + TM_CB + (uint32_t)sp * 128,
                                                                     desc_add(dm_x0, (uint32_t)(cp % X_SLOTS) * TILE_16K), id_kn, false);
                    tc::mma_commit(bars + B_YF);
                }
                if (c < nchunks) {
                    ok = tc::mbar_wait(bars + B_SF, c & 1, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    if (c > 0 || init) {
                        // Y_inter_c = C S_{c-1}^T
                        tc::mma8_ss<tc::StepKMajor2x64, tc::StepMNMajor>(tmem + TM_YO + (uint32_t)s * 64, dk_c, dm_sb, id_kn, false);
                    }
                    // dS_c^T = B^T Xs, half of the tokens after the other, + B^T Xs' (+ the third piece)
                    const uint64_t dm_b = desc_add(dm_b0, (uint32_t)s * 2 * TILE_16K);
                    const uint64_t dm_lo = desc_add(dm_x0, (uint32_t)((c + X_SLOTS - 1) % X_SLOTS) * TILE_16K);
                    ok = tc::mbar_wait(bars + B_XSF, c & 1, abort_flag) && (c == 0 || tc::mbar_wait(bars + B_DSE, (c - 1) & 1, abort_flag));
                    if (!ok) break;
                    tc::tc_fence_after();
                    tc::mma4_ss<tc::StepMNMajor, tc::StepMNMajor>(tmem + TM_DS, dm_b, dm_xs, id_nn, false);
                    ok = tc::mbar_wait(bars + B_XSF + 1, c & 1, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    tc::mma4_ss<tc::StepMNMajor, tc::StepMNMajor>(tmem + TM_DS, desc_add(dm_b, 8192), desc_add(dm_xs, 8192), id_nn, true);
                    if (c >= fine_c) tc::mma_commit(bars + B_HIF);
                    ok = tc::mbar_wait(bars + B_XLF, c & 1, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    tc::mma8_ss<tc::StepMNMajor, tc::StepMNMajor>(tmem + TM_DS, dm_b, dm_lo, id_nn, true);
                    if (c >= fine_c) {
                        ok = tc::mbar_wait(bars + B_X3F, n_fine & 1, abort_flag);
                        if (!ok) break;
                        ++n_fine;
                        tc::tc_fence_after();
                        tc::mma8_ss<tc::StepMNMajor, tc::StepMNMajor>(tmem + TM_DS, dm_b, dm_xs, id_nn, true);
                    }
                    tc::mma_commit(bars + B_DSF + s);
                }
            }
            if (!ok) atomicCAS(status, 0, STR_ERR_TIMEOUT);
        }
        __syncwarp();
    } else if (warp < 4 || warp >= 14) {
        // ------------------------------------------------------------------ W_c = CB_c o decay
        // Work is dealt out in 16-column pieces of a 32-row quadrant (a warp can only reach the tensor-memory lanes
        // of its own quadrant); the later row quadrants have more pieces below the diagonal and get two warps:
        //   quadrant 0: columns 0-31        quadrant 1: 0-63        quadrant 2: 0-63 | 64-95        quadrant 3: 0-79 | 80-127
        // plus zeros for the pieces above the diagonal.  The bf16 result of piece [16k, 16k+16) goes to the 32-bit
        // columns [16k, 16k+8) of the same accumulator buffer, i.e. into columns the same thread has just read, so
        // pieces need no ordering among themselves.
        const int quad = warp & 3, half = warp >= 14 ? 1 : 0;
        const int row = quad * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const int first = half ? (quad == 2 ? 64 : 80) : 0;
        const int n_real = half ? (quad == 2 ? 2 : 3) : (quad == 0 ? 2 : quad == 1 ? 4 : quad + 2);
        const int zero_first = half ? 96 : (quad == 0 ? 32 : 64);
        const float2 skip2 = lane & 1 ? make_float2(0.f, skip) : make_float2(skip, 0.f);
        const int n_zero = half ? (quad == 2 ? 2 : 0) : (quad == 0 ? 6 : quad == 1 ? 4 : 0);
        bool ok = true;
#pragma unroll 1
        for (int c = 0; c < nchunks; ++c) {
            const int d = c & (DEC_DEPTH - 1), s = c & 1;
            const float *dec = decs + d * DEC_FLOATS;
            if (!tc::mbar_wait(bars + B_DECF + d, (c >> 2) & 1, abort_flag)) { ok = false; break; }
            const float l_t = dec[D_LS + row], rf = dec[D_ROWF + row];
            if (!tc::mbar_wait(bars + B_CBF + s, (c >> 1) & 1, abort_flag)) { ok = false; break; }
            tc::tc_fence_after();
            const uint32_t tW = tmem + lane_base + TM_CB + (uint32_t)(s * 128);
            // the next piece is on its way while one is worked on
            uint32_t va[16], vb[16];
            tc::tmem_ld16(tW + (uint32_t)first, va);
            tc::tmem_ld_wait();
#pragma unroll 1
            for (int k = 0; k < n_real; ++k) {
                const int col0 = first + 16 * k, bj = col0 >> 5;
                if (k + 1 < n_real) tc::tmem_ld16(tW + (uint32_t)(col0 + 16), vb);
                uint32_t packed[8];
                if (bj == quad) w_piece_diag(va, packed, dec, (const uint4 *)(smem + OFF_MASK), col0, lane, l_t, skip2);
                else w_piece_below(va, packed, dec, col0, rf * dec[D_BLK + quad * 4 + bj]);
                tc::tmem_st8(tW + (uint32_t)col0, packed);
                tc::tmem_ld_wait();
#pragma unroll
                for (int i = 0; i < 16; ++i) va[i] = vb[i];
            }
            if (n_zero > 0) {
                uint32_t zero[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) zero[i] = 0u;
#pragma unroll 1
                for (int k = 0; k < n_zero; ++k) tc::tmem_st8(tW + (uint32_t)(zero_first + 16 * k), zero);
            }
            tc::tmem_st_wait();
            tc::tc_fence_before();
            warp_arrive(bars + B_WF + s, lane);
            if (lane == 0) tc::mbar_arrive(bars + B_DECE + d);
        }
        if (!ok && lane == 0) atomicCAS(status, 0, STR_ERR_TIMEOUT);
    } else if (warp < 8) {
        // ------------------------------------------------------------------ state update
        const int quad = warp & 3, row = quad * 32 + lane;        // row = state index n
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        float S[64];
#pragma unroll
        for (int i = 0; i < 64; ++i) S[i] = init && i < p && row < n ? init[(size_t)i * n + row] : 0.f;
        bool ok = true;
        uint8_t *srow = smem + OFF_SB + (row >> 3) * 1024 + (row & 7) * 128;
        auto copy_state = [&](int hf) {               // bf16 copy of half of S^T for the next chunk's Y_inter
#pragma unroll
            for (int ci = 0; ci < 4; ++ci) {
                const int q4 = hf * 4 + ci;
                *(uint4 *)(srow + ((q4 ^ (row & 7)) << 4)) =
                    make_uint4(tc::pack_bf16x2(S[8 * q4], S[8 * q4 + 1]), tc::pack_bf16x2(S[8 * q4 + 2], S[8 * q4 + 3]),
                               tc::pack_bf16x2(S[8 * q4 + 4], S[8 * q4 + 5]), tc::pack_bf16x2(S[8 * q4 + 6], S[8 * q4 + 7]));
            }
        };
        if (init) {
            copy_state(0);
            copy_state(1);
            tc::fence_proxy_async();
        }
        warp_arrive(bars + B_SF, lane);
        const int tid_g = quad * 32 + lane;
        auto inputs_there = [&](int c) {              // decay vectors and X of chunk c
            return tc::mbar_wait(bars + B_DECF + (c & (DEC_DEPTH - 1)), (c >> 2) & 1, abort_flag) &&
                   tc::mbar_wait(bars + B_XF + c % X_SLOTS, (c / X_SLOTS) & 1, abort_flag);
        };
        ok = inputs_there(0);
#pragma unroll 1
        for (int c = 0; c < nchunks && ok; ++c) {
            const int d = c & (DEC_DEPTH - 1), sx = c % X_SLOTS;
            const float *dec = decs + d * DEC_FLOATS;
            const int valid = min(Tlen - c * Q, Q);
            if (valid < Q) {                          // B's rows behind the sequence (CB may be reading them: those columns are masked)
                if (!tc::mbar_wait(bars + B_BCF + (c & 1), (c >> 1) & 1, abort_flag)) { ok = false; break; }
                uint4 *bt = (uint4 *)(smem + OFF_B + (c & 1) * 2 * TILE_16K);
                for (int u = valid * 8 + tid_g; u < Q * 8; u += 128) bt[u] = bt[u + TILE_16K / 16] = make_uint4(0u, 0u, 0u, 0u);
            }
            // Xs: its last reader, dS_{c-1}, is complete (seen below, one chunk ago).  Xs': so has to be Y_intra of the chunk whose X it replaces.
            uint4 lo[2][4];
            split_x(smem + OFF_X + sx * TILE_16K, smem + OFF_XS, lo[0], dec + D_XW, tid_g, 0, valid);
            tc::fence_proxy_async();
            warp_arrive(bars + B_XSF, lane);
            split_x(smem + OFF_X + sx * TILE_16K, smem + OFF_XS, lo[1], dec + D_XW, tid_g, 1, valid);
            tc::fence_proxy_async();
            warp_arrive(bars + B_XSF + 1, lane);
            if (c > 0 && !tc::mbar_wait(bars + B_YF, (c - 1) & 1, abort_flag)) { ok = false; break; }
            {
                uint4 *lo_tile = (uint4 *)(smem + OFF_X + ((c + X_SLOTS - 1) % X_SLOTS) * TILE_16K) + tid_g;
#pragma unroll
                for (int i = 0; i < 8; ++i) lo_tile[128 * i] = lo[i >> 2][i & 3];
                tc::fence_proxy_async();
                // (inputs of the next chunk: waited for before dS, not behind it)
                if (c + 1 < nchunks && !inputs_there(c + 1)) { ok = false; break; }
                warp_arrive(bars + B_XLF, lane);
            }
            const float eend = dec[D_EEND];
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(bars + B_DECE + d);
            if (!tc::mbar_wait(bars + B_DSF + (c & 1), (c >> 1) & 1, abort_flag)) { ok = false; break; }
            tc::tc_fence_after();
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                uint32_t v[32];
                tc::tmem_ld32(tmem + lane_base + TM_DS + (uint32_t)(hf * 32), v);
                tc::tmem_ld_wait();
                if (hf == 1) {                        // both halves of dS_c are in registers: the accumulator is free
                    tc::tc_fence_before();
                    warp_arrive(bars + B_DSE, lane);
                }
#pragma unroll
                for (int i = 0; i < 32; i += 2) {
                    const float2 r = __ffma2_rn(make_float2(eend, eend), make_float2(S[hf * 32 + i], S[hf * 32 + i + 1]),
                                                make_float2(__uint_as_float(v[i]), __uint_as_float(v[i + 1])));
                    S[hf * 32 + i] = r.x;
                    S[hf * 32 + i + 1] = r.y;
                }
                // dS_c complete implies Y_inter_c complete: the previous copy is no longer being read
                copy_state(hf);
            }
            tc::fence_proxy_async();
            warp_arrive(bars + B_SF, lane);
        }
        if (!ok && lane == 0) atomicCAS(status, 0, STR_ERR_TIMEOUT);
        // An x that is not finite has made its column of dS, and with it of the state, NaN or infinite to the end.
        bool odd = false;
#pragma unroll
        for (int i = 0; i < 64; ++i) odd |= !isfinite(S[i]);
        if (odd) found[0] = 1;
        state_warps_sync();
        if (ok && fin && found[0] == 0 && row < n) {
#pragma unroll
            for (int i = 0; i < 64; ++i)
                if (i < p) fin[(size_t)i * n + row] = S[i];
        }
    } else if (warp < 12) {
        // ------------------------------------------------------------------ y of chunk c
        const int quad = warp & 3, row = quad * 32 + lane;
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        __nv_bfloat16 *yb = y + ((size_t)row0 * H + h) * p;   // (y NULL: only the final state and the sum of dt A are wanted)
        const bool wide = p % 16 == 0 && ((uintptr_t)y & 31) == 0;
        bool ok = true;
        if (warp == 8) {
            // While there is nothing to write yet: how far from the end a chunk has faded enough, four chunks' dt at a time.
            const float *dtb = dt + (size_t)row0 * H + h;
            const float rate = -A[h] * LOG2E;
            float faded = 0.f;
            int from = nchunks - 1, k = nchunks - 1;
#pragma unroll 1
            while (k > 0 && faded < FADED) {
                float sum[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    sum[j] = 0.f;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int t = (k - j) * Q + 32 * i + lane;
                        if (k - j > 0 && t < Tlen) sum[j] += __ldg(dtb + (size_t)t * H);
                    }
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float s = warp_sum(sum[j]) * rate;
                    if (k - j > 0 && faded < FADED) {
                        faded += s;
                        if (faded < FADED) from = k - j - 1;
                    }
                }
                k -= 4;
            }
            if (lane == 0) {
                fine_from[0] = from;
                tc::mbar_arrive(bars + B_FINE);
            }
            __syncwarp();
        }
        ok = tc::mbar_wait(bars + B_FINE, 0, abort_flag);
        const int fine_c = fine_from[0];
#pragma unroll 1
        for (int cp = 0; cp < nchunks && ok; ++cp) {
            {
                const int d = cp & (DEC_DEPTH - 1), t0 = cp * Q;
                if (!tc::mbar_wait(bars + B_DECF + d, (cp >> 2) & 1, abort_flag)) { ok = false; break; }
                const float er = decs[d * DEC_FLOATS + D_EROW + row];
                if (cp >= fine_c) {                   // the third piece, once the product with the first is through
                    if (!tc::mbar_wait(bars + B_HIF, (cp - fine_c) & 1, abort_flag)) { ok = false; break; }
                    third_x(smem + OFF_X + cp % X_SLOTS * TILE_16K, smem + OFF_XS, decs + d * DEC_FLOATS + D_XW, row);
                    tc::fence_proxy_async();
                    warp_arrive(bars + B_X3F, lane);
                }
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(bars + B_DECE + d);
                if (!tc::mbar_wait(bars + B_YF, cp & 1, abort_flag)) { ok = false; break; }
                tc::tc_fence_after();
                __nv_bfloat16 *dst = yb + (size_t)(t0 + row) * H * p;
                const bool valid = y && t0 + row < Tlen;
#pragma unroll 1
                for (int hf = 0; hf < 2; ++hf) {
                    uint32_t ya[32], yo[32];
                    tc::tmem_ld32(tmem + lane_base + TM_YI + (uint32_t)(hf * 32), ya);
                    if (cp > 0 || init) tc::tmem_ld32(tmem + lane_base + TM_YO + (uint32_t)((cp & 1) * 64 + hf * 32), yo);
                    tc::tmem_ld_wait();
                    if (hf == 1) {                    // both accumulators are in registers
                        tc::tc_fence_before();
                        warp_arrive(bars + B_YE, lane);
                    }
                    if (cp > 0 || init) {
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const float2 r = __ffma2_rn(make_float2(er, er), make_float2(__uint_as_float(yo[i]), __uint_as_float(yo[i + 1])),
                                                        make_float2(__uint_as_float(ya[i]), __uint_as_float(ya[i + 1])));
                            ya[i] = __float_as_uint(r.x);
                            ya[i + 1] = __float_as_uint(r.y);
                        }
                    }
                    if (valid) {
                        store16(dst + 32 * hf, ya, p - 32 * hf, wide);
                        store16(dst + 32 * hf + 16, ya + 16, p - 32 * hf - 16, wide);
                    }
                }
            }
        }
        if (!ok && lane == 0) atomicCAS(status, 0, STR_ERR_TIMEOUT);
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 13) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, 512); }
    if (found[0])
        scan_rows(x + ((size_t)row0 * H + h) * p, dt + (size_t)row0 * H + h, A[h], B + ((size_t)row0 * G + g) * n, C + ((size_t)row0 * G + g) * n, Dskip ? Dskip + h : nullptr, init,
                  y ? y + ((size_t)row0 * H + h) * p : nullptr, fin, Tlen, H, G, p, n);
}

}  // namespace

bool str_scan_packed_tc_shape(const str_ssd_packed_shape *s) {
    return s->dtype == STR_BF16 && s->p <= P && s->n <= NS && s->p % 8 == 0 && s->n % 8 == 0 && s->rows > 0;
}

bool str_scan_packed_tc_supported(const str_ssd_packed_shape *s, const void *x, const void *B, const void *C, const void *y) {
    return str_scan_packed_tc_shape(s) && (((uintptr_t)x | (uintptr_t)B | (uintptr_t)C | (uintptr_t)y) & 15) == 0 && (long long)s->H * s->n_seq <= INT32_MAX;
}

int str_scan_packed_tc(str_ctx *ctx, const str_ssd_packed_shape *s, const void *x, const float *dt, const float *A, const void *B, const void *C,
                       const float *D, const int32_t *start, const float *init_state, void *y, float *final_state, float *faded, cudaStream_t st) {
    CUtensorMap tx, tb, tcm;
    int rc = str_make_tmap_heads_bf16_sw128(ctx, &tx, x, s->p, s->H, s->rows, 1, Q);
    if (rc == STR_OK) rc = str_make_tmap_heads_bf16_sw128(ctx, &tb, B, s->n, s->G, s->rows, 1, Q);
    if (rc == STR_OK) rc = str_make_tmap_heads_bf16_sw128(ctx, &tcm, C, s->n, s->G, s->rows, 1, Q);
    if (rc != STR_OK) return rc;
    rc = str_ensure_smem(ctx, STR_SMEM_SCAN_PACKED, scan_packed_tc_kernel, SMEM_BYTES);
    if (rc != STR_OK) return rc;
    scan_packed_tc_kernel<<<s->H * s->n_seq, NUM_THREADS, SMEM_BYTES, st>>>(
        tx, tb, tcm, s->n_seq, s->rows, s->H, s->p, s->n, s->G, dt, A, D, start, (const __nv_bfloat16 *)x, (const __nv_bfloat16 *)B, (const __nv_bfloat16 *)C,
        init_state, (__nv_bfloat16 *)y, final_state, faded, ctx->status_dev);
    return str_launch_ok(ctx);
}

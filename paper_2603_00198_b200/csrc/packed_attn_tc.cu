// Causal attention of packed sequences on tcgen05 tensor cores (bf16 in/out, fp32 accumulate, head sizes up to 128 that are multiples of 8).
//
// Rows are (query, head) pairs: the 128 rows of a tile are 128 / R consecutive queries of one sequence for the R query heads of one key head, so
// that a key tile is fetched once for all of them and a turn of a few queries still fills the tile.  A CTA owns two such tiles that take turns on
// the tensor pipe; the softmax of one overlaps the products of the other.  Per key tile j of 128 keys and row tile i:
//   S_i  = Q_i K_j^T                 both operands K-major in shared memory (TMA, 128-byte swizzle, columns beyond d read as zero)
//   P_i  = exp2(c S_i - c m_i)       one thread per row; running maximum m_i and sum l_i in fp32; P_i is narrowed to bf16 (relative error 2^-8 of each
//                                    weight at most, random in sign: what the tensor pipe takes) over the first 64 columns of S_i, and is the A
//                                    operand of
//   O_i += P_i V_j                   A from tensor memory, V MN-major; issued half by half, as soon as 64 keys' weights are there
//   out  = O_i / l_i
// O_i is rescaled only when a row's maximum grows by more than 2^8: until then the stale maximum stays in use, which divides out through l_i.
//
// What a row does not see must not reach it.  Hidden scores are replaced before the maximum, so anything may stand there.  Hidden values meet weights of
// zero in the product, and zero times infinity or NaN is NaN: rows of V behind the sequence are zeroed in shared memory, and the tiles that some
// row of the CTA sees in part only are looked through for values that are not finite.  A CTA that found one computes its rows anew, row by row
// (attn_row): right, slow and rare.
//
// Tensor memory (512 columns): S_0 | S_1 | O_0 | O_1, 128 columns each.
// Warps: 0-3 softmax of tile 0, 4-7 softmax of tile 1 (warp w may touch TMEM lanes 32 (w % 4)...), 8 TMA producer (Q once, then a 2-slot ring for K and
// one for V), 9 MMA issuer, 10 the guard that zeroes and looks through tiles of V.
//
// Measured: one prompt of 16512 rows, 32 / 8 heads of 128: 1.80 to 1.85 ms on a cool card, 1207 to 1240 TFLOP/s, 0.72 to 0.74 of the measured burst figure; again and again, under the
// power cap, 2.09 to 2.15 ms, 0.74 to 0.76 of the sustained one; twelve turns of 8200 rows over 24800 keys 191 to 229 us; 300 rows over 4396 keys 44 us, 74 without sharing the walk.  A key tile takes 3600 clocks for 2048 of
// products: after its last weights a row tile waits 1200 to 1500 for the second half of P V, the next S and the barriers between them, in
// which the other tile's softmax runs; the special-function unit (2048 clocks for all exponentials) is the next limit, hence one pair in six on
// the FMA pipe.  Tried and not kept: steps of 64 keys with two S buffers a tile, which takes the wait away but makes every S product re-read Q for half the
// keys (2.13 ms); the first half's weights with the stale maximum while the new one is looked for, registers split 216 / 72 (1.90 ms); one pair
// in two or four on the FMA pipe (2.08, 1.92 ms).
// Every mbarrier wait is bounded; a give-up records STR_ERR_TIMEOUT and the CTA tears down.
#include "dispatch.cuh"
#include "packed.cuh"
#include "tc_common.cuh"

namespace {

constexpr int BQ = 128, BKV = 128, TILE_16K = 16384;      // rows x 64 bf16
enum { B_Q = 0, B_KF, B_KE = B_KF + 2, B_VF = B_KE + 2, B_VR = B_VF + 2, B_VE = B_VR + 2, B_SF = B_VE + 2, B_PA = B_SF + 2, B_PB = B_PA + 2, B_OF = B_PB + 2,
       B_COUNT = B_OF + 2 };
constexpr int NUM_WARPS = 11, NUM_THREADS = NUM_WARPS * 32;
constexpr int POLY_EVERY = 6;                             // every so many pairs of exponentials run on the FMA pipe (0: none)
constexpr uint32_t TM_S = 0, TM_O = 256;
constexpr float RESCALE_THRESHOLD = 8.0f;                 // in log2 units

template <int HD> struct Smem {
    static constexpr int TILE = HD / 64 * TILE_16K;       // one tile of Q, K or V
    static constexpr int Q = 0, K = 2 * TILE, V = 4 * TILE, MISC = 6 * TILE;
    static constexpr size_t BYTES = (size_t)MISC + B_COUNT * 8 + 32 + sizeof(PackedBlock);
};

// 2^x of two numbers on the FMA pipe: x = n + f with n the nearest whole number, a cubic in f on [-1/2, 1/2] (minimax, relative error 7.5e-5: a
// fiftieth of the rounding to bf16 that follows), and n added to the exponent.  x <= 2^7; below -126 it is zero, as the special-function unit's is: a
// hidden key's weight (x minus infinity) has to be nothing, whatever it is multiplied by.
__device__ __forceinline__ float2 ex2_poly(float2 x) {
    const float2 magic = make_float2(12582912.f, 12582912.f);         // 1.5 * 2^23: the sum's last bits are the whole number
    const float2 t = __fadd2_rn(x, magic);
    const float2 n = __fadd2_rn(t, make_float2(-12582912.f, -12582912.f));
    const float2 f = __ffma2_rn(n, make_float2(-1.f, -1.f), x);
    float2 p = __ffma2_rn(make_float2(0.05517166853f, 0.05517166853f), f, make_float2(0.24261112511f, 0.24261112511f));
    p = __ffma2_rn(p, f, make_float2(0.69326096773f, 0.69326096773f));
    p = __ffma2_rn(p, f, make_float2(0.99992805719f, 0.99992805719f));
    return make_float2(x.x < -126.f ? 0.f : __uint_as_float(__float_as_uint(p.x) + (__float_as_uint(t.x) << 23)),
                       x.y < -126.f ? 0.f : __uint_as_float(__float_as_uint(p.y) + (__float_as_uint(t.y) << 23)));
}

// Weights of 64 keys, exp2(scale (s - m)), narrowed and in pairs; their sum is added up as it was before.
__device__ __forceinline__ void weights(const uint32_t (&s0)[32], const uint32_t (&s1)[32], float2 scale2, float m, uint32_t (&pk)[32], float2 &sum) {
    const float mc = m == -INFINITY ? 0.f : m * scale2.x;
    const float2 nmc2 = make_float2(-mc, -mc);
#pragma unroll
    for (int e = 0; e < 32; ++e) {
        const uint32_t *s = e < 16 ? s0 : s1;
        const int k = (2 * e) & 31;
        const float2 a = __ffma2_rn(make_float2(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), scale2, nmc2);
        float2 p;
        if (POLY_EVERY > 0 && e % (POLY_EVERY > 0 ? POLY_EVERY : 1) == POLY_EVERY - 1) p = ex2_poly(a);
        else p = make_float2(tc::ex2(a.x), tc::ex2(a.y));
        sum = __fadd2_rn(sum, p);
        pk[e] = tc::pack_bf16x2(p.x, p.y);
    }
}

// One row's output in fp32 arithmetic, by one warp: a lane takes a key for the scores and every 32nd column for the values.
__device__ __noinline__ void attn_row(const __nv_bfloat16 *q, const __nv_bfloat16 *k, const __nv_bfloat16 *v, __nv_bfloat16 *o, size_t ld, int keys, int d,
                                      float scale_log2) {
    const int lane = threadIdx.x & 31;
    float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int j0 = 0; j0 < keys; j0 += 32) {
        float s = -INFINITY;
        if (j0 + lane < keys) {
            s = 0.f;
            for (int c = 0; c < d; ++c) s = fmaf(ldf(q + c), ldf(k + (size_t)(j0 + lane) * ld + c), s);
            s *= scale_log2;
        }
        const float nm = fmaxf(m, warp_max(s)), at = nm == -INFINITY ? 0.f : nm;
        const float f = exp2f(m - at), p = exp2f(s - at);
        l = fmaf(l, f, warp_sum(p));
        m = nm;
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] *= f;
        for (int j = 0; j < min(32, keys - j0); ++j) {
            const float pj = __shfl_sync(0xffffffffu, p, j);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 32 * i < d) acc[i] = fmaf(pj, ldf(v + (size_t)(j0 + j) * ld + lane + 32 * i), acc[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (lane + 32 * i < d) stf(o + lane + 32 * i, keys > 0 ? acc[i] / l : 0.f);
}

// What CTAs that share a block's key tiles leave for the joining kernel (number n of them: unscaled outputs, maxima and sums of 256 rows, and whether a
// hidden value was not finite).
struct Parts {
    int splits;                  // 1: there are none
    float *o;                    // [n][256][HD]
    float2 *stat;                // [n][256]: maximum (of unscaled scores), sum
    int *found;                  // [n]
    PackedBlock *block;          // [n / splits]: the block itself, so that the joining kernel need not look for it
};

template <int HD>
__global__ void __launch_bounds__(NUM_THREADS, 1)
attn_packed_tc_kernel(const __grid_constant__ CUtensorMap tmap_q, const __grid_constant__ CUtensorMap tmap_k, const __grid_constant__ CUtensorMap tmap_v,
                      const __grid_constant__ CUtensorMap tmap_o, const PackedBlockSize block_size, int n_seq, int rows_q, int rows_k, int Hq, int Hkv, int d,
                      float scale_log2, const int32_t *__restrict__ q_start, const int32_t *__restrict__ k_start, const __nv_bfloat16 *__restrict__ q, const __nv_bfloat16 *__restrict__ k,
                      const __nv_bfloat16 *__restrict__ v, __nv_bfloat16 *__restrict__ out, const Parts parts, int *status) {
    typedef Smem<HD> SM;
    constexpr int HALVES = HD / 64;
    extern __shared__ __align__(1024) uint8_t smem[];
    uint64_t *bars = (uint64_t *)(smem + SM::MISC);
    uint32_t *tmem_slot = (uint32_t *)(bars + B_COUNT);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);       // [2]
    volatile int *found = abort_flag + 2;                             // a hidden value that is not finite
    PackedBlock *blk = (PackedBlock *)(tmem_slot + 4);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = Hq / Hkv, TQ = BQ / group;                      // queries per tile
    const int kv = blockIdx.x % Hkv, split = blockIdx.x / Hkv % parts.splits, rank = blockIdx.x / Hkv / parts.splits;
    const size_t part = ((size_t)rank * Hkv + kv) * parts.splits + split;

    if ((tc::smem_u32(smem) & 1023u) != 0) {
        if (threadIdx.x == 0) atomicCAS(status, 0, STR_ERR_CUDA);
        return;
    }
    if (blockIdx.x == 0) {
        packed_check(q_start, n_seq, rows_q, status);
        packed_check(k_start, n_seq, rows_k, status);
    }
    // Query number t of the block sees the keys 0 .. first_limit + t.  Of the key tiles of its row tiles (tile 1 has no fewer than tile 0 unless it is
    // empty) this CTA takes its share: tiles j0 + j, j < n0 or n1.
    struct Walk {
        int first_limit, j0, n0, n1, nt;
        __device__ __forceinline__ Walk(const PackedBlock &b, int TQ, int splits, int split) {
            first_limit = b.lk - b.lq + b.first;
            const int all0 = (max(first_limit + min(b.n, TQ), 0) + BKV - 1) / BKV, all1 = b.n > TQ ? (max(first_limit + b.n, 0) + BKV - 1) / BKV : 0;
            const int share = (max(all0, all1) + splits - 1) / splits;
            j0 = split * share;
            n0 = max(min(all0, j0 + share) - j0, 0), n1 = max(min(all1, j0 + share) - j0, 0), nt = max(n0, n1);
        }
    };
    auto load_k = [&](const PackedBlock &b, int j0, int j) {
        tc::mbar_arrive_expect_tx(bars + B_KF + (j & 1), SM::TILE);
        for (int hf = 0; hf < HALVES; ++hf)
            tc::tma_load_3d(smem + SM::K + (j & 1) * SM::TILE + hf * TILE_16K, &tmap_k, bars + B_KF + (j & 1), hf * 64, kv, b.k0 + (j0 + j) * BKV);
    };
    // The producer finds the block and sends for its queries and first keys while the others make ready (with the bulk store at the end: sixteen sequences of
    // 1000 rows 76 -> 70 us, one of 16512 rows 1920 -> 1881).  A CTA leaves, whole, when there is no block for it or an earlier one failed.
    if (warp == 8) {
        const int failed = *(volatile const int *)status;
        if (lane == 0) {
            tc::mbar_init(bars + B_Q, 1);
            for (int s = 0; s < 2; ++s) {
                tc::mbar_init(bars + B_KF + s, 1); tc::mbar_init(bars + B_KE + s, 1);
                tc::mbar_init(bars + B_VF + s, 1); tc::mbar_init(bars + B_VR + s, 1); tc::mbar_init(bars + B_VE + s, 2);
                tc::mbar_init(bars + B_SF + s, 1); tc::mbar_init(bars + B_PA + s, 4); tc::mbar_init(bars + B_PB + s, 4);
                tc::mbar_init(bars + B_OF + s, 1);
            }
            abort_flag[0] = 0; abort_flag[1] = 0; found[0] = 0;
            tc::fence_mbar_init();
            tc::prefetch_tmap(&tmap_q); tc::prefetch_tmap(&tmap_k); tc::prefetch_tmap(&tmap_v);
        }
        __syncwarp();
        PackedBlock b = packed_block(q_start, k_start, n_seq, rows_q, rows_k, block_size, BKV, rank);
        if (failed) b.n = 0;
        if (lane == 0) {
            *blk = b;
            if (parts.splits > 1 && split == 0) parts.block[(size_t)rank * Hkv + kv] = b;
            const Walk w(b, TQ, parts.splits, split);
            if (b.n > 0 && w.nt > 0) {
                tc::mbar_arrive_expect_tx(bars + B_Q, (uint32_t)(2 * HALVES * TQ * group) * 128u);
                for (int i = 0; i < 2; ++i)
                    for (int hf = 0; hf < HALVES; ++hf)
                        tc::tma_load_3d(smem + SM::Q + i * SM::TILE + hf * TILE_16K, &tmap_q, bars + B_Q, hf * 64, kv * group, b.q0 + b.first + i * TQ);
                load_k(b, w.j0, 0);
            }
        }
        __syncwarp();
    }
    if (warp == 9) { tc::tmem_alloc(tmem_slot, 512); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    const PackedBlock b = *blk;
    if (b.n <= 0) {
        if (warp == 9) tc::tmem_dealloc(tmem, 512);
        return;
    }
    const Walk walk(b, TQ, parts.splits, split);
    const int first_limit = walk.first_limit, j0 = walk.j0, n0 = walk.n0, n1 = walk.n1, nt = walk.nt;

    if (warp == 8) {
        // ------------------------------------------------------------------ TMA producer
        if (lane == 0 && nt > 0) {
            bool ok = true;
            int issued_k = 1, issued_v = 0;                           // the queries and keys of tile 0 are on their way
            for (int j = 0; j < nt; ++j) {
                const int s = j & 1;
                const uint32_t ph = ((j >> 1) & 1) ^ 1;
                if (!tc::mbar_wait(bars + B_KE + s, ph, abort_flag)) { ok = false; break; }
                if (j > 0) {
                    load_k(b, j0, j);
                    ++issued_k;
                }
                if (!tc::mbar_wait(bars + B_VE + s, ph, abort_flag)) { ok = false; break; }
                tc::mbar_arrive_expect_tx(bars + B_VF + s, SM::TILE);
                for (int hf = 0; hf < HALVES; ++hf)
                    tc::tma_load_3d(smem + SM::V + s * SM::TILE + hf * TILE_16K, &tmap_v, bars + B_VF + s, hf * 64, kv, b.k0 + (j0 + j) * BKV);
                ++issued_v;
            }
            if (!ok) {
                atomicCAS(status, 0, STR_ERR_TIMEOUT);
                // let copies already issued land before the CTA's shared memory goes away
                tc::mbar_wait(bars + B_Q, 0, abort_flag + 1);
                for (int back = 1; back <= 2 && back <= issued_k; ++back) {
                    const int j = issued_k - back;
                    tc::mbar_wait(bars + B_KF + (j & 1), (j >> 1) & 1, abort_flag + 1);
                }
                for (int back = 1; back <= 2 && back <= issued_v; ++back) {
                    const int j = issued_v - back;
                    tc::mbar_wait(bars + B_VF + (j & 1), (j >> 1) & 1, abort_flag + 1);
                }
            }
        }
    } else if (warp == 9) {
        // ------------------------------------------------------------------ MMA issuer (one elected thread for the whole loop, see tc_common.cuh)
        if (tc::elect_one() && nt > 0) {
            const uint32_t id_s = tc::make_idesc_bf16(BQ, BKV, 0, 0);     // Q (K-major) x K (K-major)
            const uint32_t id_o = tc::make_idesc_bf16(BQ, HD, 0, 1);      // P (tensor memory) x V (MN-major)
            const uint32_t sbase = tc::smem_u32(smem);
            auto issue_s = [&](int i, int slot) {
                const uint64_t qd = tc::desc_kmajor_sw128(sbase + SM::Q + (uint32_t)i * SM::TILE, 0);
                const uint64_t kd = tc::desc_kmajor_sw128(sbase + SM::K + (uint32_t)slot * SM::TILE, 0);
                if constexpr (HD == 128) tc::mma8_ss<tc::StepKMajor2x64, tc::StepKMajor2x64>(tmem + TM_S + (uint32_t)i * 128, qd, kd, id_s, false);
                else tc::mma4_ss<tc::StepKMajor64, tc::StepKMajor64>(tmem + TM_S + (uint32_t)i * 128, qd, kd, id_s, false);
                tc::mma_commit(bars + B_SF + i);
            };
            auto issue_pv = [&](int i, int slot, int half, bool first) {
                const uint64_t vd = tc::make_smem_desc(sbase + SM::V + (uint32_t)slot * SM::TILE + (uint32_t)half * 8192u, TILE_16K, 1024, tc::SWZ_128B);
                tc::mma4_ts<tc::StepTmem8, tc::StepMNMajor>(tmem + TM_O + (uint32_t)i * 128, tmem + TM_S + (uint32_t)i * 128 + (uint32_t)half * 32, vd, id_o, !first);
            };
            bool ok = tc::mbar_wait(bars + B_Q, 0, abort_flag) && tc::mbar_wait(bars + B_KF, 0, abort_flag);
            if (ok) {
                tc::tc_fence_after();
                if (n0 > 0) issue_s(0, 0);
                if (n1 > 0) issue_s(1, 0);
                tc::mma_commit(bars + B_KE);
            }
            for (int j = 0; j < nt && ok; ++j) {
                const int s = j & 1, ns = (j + 1) & 1;
                if (!tc::mbar_wait(bars + B_VF + s, (j >> 1) & 1, abort_flag) || !tc::mbar_wait(bars + B_VR + s, (j >> 1) & 1, abort_flag)) { ok = false; break; }
                if (j < n0) {
                    if (!tc::mbar_wait(bars + B_PA, j & 1, abort_flag)) { ok = false; break; }
                    tc::tc_fence_after();
                    issue_pv(0, s, 0, j == 0);
                    if (!tc::mbar_wait(bars + B_PB, j & 1, abort_flag)) { ok = false; break; }
                    tc::tc_fence_after();
                    issue_pv(0, s, 1, false);
                    if (j == n0 - 1) tc::mma_commit(bars + B_OF);
                }
                if (j + 1 < nt) {
                    if (!tc::mbar_wait(bars + B_KF + ns, ((j + 1) >> 1) & 1, abort_flag)) { ok = false; break; }
                    tc::tc_fence_after();
                    if (j + 1 < n0) issue_s(0, ns);
                }
                if (j < n1) {
                    if (!tc::mbar_wait(bars + B_PA + 1, j & 1, abort_flag)) { ok = false; break; }
                    tc::tc_fence_after();
                    issue_pv(1, s, 0, j == 0);
                    if (!tc::mbar_wait(bars + B_PB + 1, j & 1, abort_flag)) { ok = false; break; }
                    tc::tc_fence_after();
                    issue_pv(1, s, 1, false);
                    if (j == n1 - 1) tc::mma_commit(bars + B_OF + 1);
                }
                tc::mma_commit(bars + B_VE + s);
                if (j + 1 < nt) {
                    if (j + 1 < n1) issue_s(1, ns);
                    tc::mma_commit(bars + B_KE + ns);
                }
            }
            if (!ok) atomicCAS(status, 0, STR_ERR_TIMEOUT);
        }
        __syncwarp();
    } else if (warp == 10) {
        // ------------------------------------------------------------------ guard over the tiles of V
        bool ok = true;
        for (int j = 0; j < nt; ++j) {
            const int s = j & 1;
            if (!tc::mbar_wait(bars + B_VF + s, (j >> 1) & 1, abort_flag)) { ok = false; break; }
            uint8_t *tile = smem + SM::V + s * SM::TILE;
            const int valid = min(b.lk - (j0 + j) * BKV, BKV);               // rows of the tile that are the sequence's
            if (valid < BKV) {
                for (int e = valid * 8 + lane; e < BKV * 8; e += 32)
#pragma unroll
                    for (int hf = 0; hf < HALVES; ++hf) *(uint4 *)(tile + hf * TILE_16K + e * 16) = make_uint4(0u, 0u, 0u, 0u);
                tc::fence_proxy_async();
                __syncwarp();
            }
            if (lane == 0) tc::mbar_arrive(bars + B_VR + s);
            if ((j0 + j) * BKV + BKV - 1 > first_limit) {                    // hidden in part: zero times what is finite stays zero
                const __nv_bfloat162 zero = __float2bfloat162_rn(0.f);
                __nv_bfloat162 sum = zero;
#pragma unroll 4
                for (int e = lane; e < BKV * 8 * HALVES; e += 32) {
                    const uint4 w = *(const uint4 *)(tile + e * 16);
                    const __nv_bfloat162 *x = reinterpret_cast<const __nv_bfloat162 *>(&w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum = __hfma2(x[i], zero, sum);
                }
                if (__low2float(sum) != 0.f || __high2float(sum) != 0.f) found[0] = 1;       // NaN
                __syncwarp();
            }
            if (lane == 0) tc::mbar_arrive(bars + B_VE + s);
        }
        if (!ok && lane == 0) atomicCAS(status, 0, STR_ERR_TIMEOUT);
    } else {
        // ------------------------------------------------------------------ softmax warps
        const int i = warp >> 2, quad = warp & 3;
        const int row = quad * 32 + lane, t = i * TQ + row / group;   // row of the tile, query of the block
        const uint32_t lane_base = (uint32_t)(quad * 32) << 16;
        const uint32_t tS = tmem + lane_base + TM_S + (uint32_t)i * 128;
        const uint32_t tO = tmem + lane_base + TM_O + (uint32_t)i * 128;
        const int ni = i == 0 ? n0 : n1;
        const bool live = row < TQ * group && t < b.n;
        const int limit = first_limit + min(t, b.n - 1);              // this row sees the keys 0 .. limit
        const float2 scale2 = make_float2(scale_log2, scale_log2);
        float m = -INFINITY, l = 0.f;
        bool ok = true;
        for (int j = 0; j < ni; ++j) {
            if (!tc::mbar_wait(bars + B_SF + i, j & 1, abort_flag)) { ok = false; break; }
            tc::tc_fence_after();
            uint32_t w[4][32];
#pragma unroll
            for (int c = 0; c < 4; ++c) tc::tmem_ld32(tS + c * 32, w[c]);
            tc::tmem_ld_wait();
            if (__any_sync(0xffffffffu, (j0 + j) * BKV + BKV - 1 > limit)) { // some row of this warp ends inside (or before) this tile
                const int lim = limit - (j0 + j) * BKV;
#pragma unroll
                for (int c = 0; c < 4; ++c)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (c * 32 + e > lim) w[c][e] = 0xFF800000u;  // -infinity
            }
            float top[4] = {m, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 32; e += 2)
#pragma unroll
                for (int c = 0; c < 4; ++c) top[c] = tc::max3_nan(top[c], __uint_as_float(w[c][e]), __uint_as_float(w[c][e + 1]));
            float m_new = tc::max3_nan(tc::max3_nan(top[0], top[1], top[2]), top[3], top[3]);
            if (m_new == INFINITY) m_new = __int_as_float(0x7FFFFFFF);    // infinity minus infinity: the row is NaN, as with a NaN score
            // A row raises its maximum only when it has grown by more than the threshold: a decision of the row alone.  From minus infinity
            // (nothing seen yet) any score is growth.
            const bool grow = (m_new - m) * scale_log2 > RESCALE_THRESHOLD || m_new != m_new;
            if (j == 0) {
                m = m_new;
            } else if (__any_sync(0xffffffffu, grow)) {
                // S_j complete implies the previous P V product of this tile is complete: O is stable.  The whole warp
                // runs the (warp-collective) accumulator update; rows that keep their maximum multiply by exactly 1.
                const float f = grow ? tc::ex2((m - m_new) * scale_log2) : 1.0f;
                if (grow) { l *= f; m = m_new; }
#pragma unroll 1
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t o[32];
                    tc::tmem_ld32(tO + c * 32, o);
                    tc::tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                    tc::tmem_st32(tO + c * 32, o);
                }
                tc::tmem_st_wait();
            }
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                uint32_t pk[32];
                weights(w[2 * hf], w[2 * hf + 1], scale2, m, pk, sum);
                tc::tmem_st32(tS + hf * 32, pk);
                tc::tmem_st_wait();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(bars + (hf == 0 ? B_PA : B_PB) + i);
            }
            l += sum.x + sum.y;
        }
        if (ok && ni > 0) ok = tc::mbar_wait(bars + B_OF + i, 0, abort_flag);
        else if (ok && nt > 0) ok = tc::mbar_wait(bars + B_Q, 0, abort_flag);        // nothing to see, but the queries' copy has to have landed
        // A whole tile goes out through shared memory, over its queries (every product that read them is through), by one bulk store: written by a
        // thread each, the rows take 3500 clocks a CTA.  The last tile of a sequence, whose rows beyond the end are not its own, is written so.
        const bool whole = parts.splits == 1 && (i + 1) * TQ <= b.n;
        uint8_t *tile = smem + SM::Q + i * SM::TILE;
        if (ok) {
            tc::tc_fence_after();
            if (parts.splits > 1) {
                const size_t at = part * 2 * BQ + i * BQ + row;
                parts.stat[at] = make_float2(ni > 0 ? m : -INFINITY, l);
                if (ni > 0) {
#pragma unroll 1
                    for (int c = 0; c < HD / 32; ++c) {
                        uint32_t o[32];
                        tc::tmem_ld32(tO + c * 32, o);
                        tc::tmem_ld_wait();
#pragma unroll
                        for (int g = 0; g < 8; ++g) *(uint4 *)(parts.o + at * HD + c * 32 + 4 * g) = make_uint4(o[4 * g], o[4 * g + 1], o[4 * g + 2], o[4 * g + 3]);
                    }
                }
            } else {
                const bool sees = limit >= 0;
                const float inv = sees ? 1.0f / l : 0.f;
                __nv_bfloat16 *dst = out + ((size_t)(b.q0 + b.first + t) * Hq + kv * group + row % group) * d;
#pragma unroll 1
                for (int c = 0; c < HD / 32; ++c) {
                    uint32_t o[32];
                    if (ni > 0) {
                        tc::tmem_ld32(tO + c * 32, o);
                        tc::tmem_ld_wait();
                    }
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        uint32_t r[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            r[e] = sees ? tc::pack_bf16x2(__uint_as_float(o[8 * g + 2 * e]) * inv, __uint_as_float(o[8 * g + 2 * e + 1]) * inv) : 0u;
                        const uint4 w4 = make_uint4(r[0], r[1], r[2], r[3]);
                        if (whole) *(uint4 *)(tile + (c >> 1) * TILE_16K + (row >> 3) * 1024 + (row & 7) * 128 + ((((c & 1) * 4 + g) ^ (row & 7)) << 4)) = w4;
                        else if (live && c * 32 + g * 8 < d) *reinterpret_cast<uint4 *>(dst + c * 32 + g * 8) = w4;
                    }
                }
                if (whole) tc::fence_proxy_async();
            }
        } else if (lane == 0) {
            atomicCAS(status, 0, STR_ERR_TIMEOUT);
        }
        if (whole) {                                                  // (alike in the tile's four warps, and all of them come here)
            asm volatile("barrier.sync %0, 128;" ::"r"(1 + i) : "memory");
            if (ok && quad == 0 && lane == 0) {
                for (int hf = 0; hf < HALVES && hf * 64 < d; ++hf) tc::tma_store_3d(&tmap_o, tile + hf * TILE_16K, hf * 64, kv * group, b.q0 + b.first + i * TQ);
                tc::bulk_commit();
                tc::bulk_wait_read();
            }
            __syncwarp();
        }
    }
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 9) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, 512); }
    if (parts.splits > 1 && threadIdx.x == 0) parts.found[part] = found[0];
    if (found[0] == 0 || parts.splits > 1) return;
    tc::bulk_wait_written();                                          // what the bulk stores wrote is written over
    __syncthreads();
    for (int r = warp; r < b.n * group; r += NUM_WARPS) {
        const int t = r / group;
        const size_t at = ((size_t)(b.q0 + b.first + t) * Hq + kv * group + r % group) * d, keys = ((size_t)b.k0 * Hkv + kv) * d;
        attn_row(q + at, k + keys, v + keys, out + at, (size_t)Hkv * d, max(first_limit + t + 1, 0), d, scale_log2);
    }
}

// Joins the shares of each block: o = sum_s exp2(scale (m_s - m)) o_s / sum_s exp2(scale (m_s - m)) l_s, a warp a row.
constexpr int JOIN_WARPS = 8, MAX_SPLITS = 16;
template <int HD>
__global__ void __launch_bounds__(JOIN_WARPS * 32)
attn_packed_join_kernel(int Hq, int Hkv, int d, float scale_log2, const __nv_bfloat16 *__restrict__ q, const __nv_bfloat16 *__restrict__ k,
                        const __nv_bfloat16 *__restrict__ v, __nv_bfloat16 *__restrict__ out, const Parts parts, const int *status) {
    if (*(volatile const int *)status != 0) return;   // a share may be missing
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int group = Hq / Hkv, TQ = BQ / group, kv = blockIdx.x % Hkv;
    const size_t part = (size_t)blockIdx.x * parts.splits;
    const PackedBlock b = parts.block[blockIdx.x];
    const bool any = b.n > 0 && __any_sync(0xffffffffu, lane < parts.splits && parts.found[part + lane] != 0);
    const int first_limit = b.lk - b.lq + b.first;
    for (int r = blockIdx.y * JOIN_WARPS + warp; r < b.n * group; r += gridDim.y * JOIN_WARPS) {
        const int t = r / group;
        const size_t at = ((size_t)(b.q0 + b.first + t) * Hq + kv * group + r % group) * d;
        const int keys = max(first_limit + t + 1, 0);
        if (any) {
            const size_t k0 = ((size_t)b.k0 * Hkv + kv) * d;
            attn_row(q + at, k + k0, v + k0, out + at, (size_t)Hkv * d, keys, d, scale_log2);
            continue;
        }
        const int row = t < TQ ? r : BQ + (t - TQ) * group + r % group;
        // lane s looks at share s; shares that saw nothing weigh nothing, and their outputs, which were never written, are not read
        const float2 st = lane < parts.splits ? parts.stat[(part + lane) * 2 * BQ + row] : make_float2(-INFINITY, 0.f);
        const float m = warp_max(st.x);
        const float w = st.x == -INFINITY ? 0.f : exp2f((st.x - m) * scale_log2);
        const float l = warp_sum(w * st.y);
        const unsigned saw = __ballot_sync(0xffffffffu, st.x != -INFINITY);
        float acc[HD / 32] = {};
#pragma unroll 4
        for (int s = 0; s < parts.splits; ++s) {
            const float ws = __shfl_sync(0xffffffffu, w, s);
            const float *o = parts.o + ((part + s) * 2 * BQ + row) * HD + lane * (HD / 32);
            alignas(16) float x[HD / 32] = {};
            if (saw >> s & 1) {
                if constexpr (HD == 128) *(float4 *)x = *(const float4 *)o;
                else *(float2 *)x = *(const float2 *)o;
            }
#pragma unroll
            for (int i = 0; i < HD / 32; ++i) acc[i] = fmaf(ws, x[i], acc[i]);
        }
#pragma unroll
        for (int i = 0; i < HD / 32; ++i)
            if (lane * (HD / 32) + i < d) stf(out + at + lane * (HD / 32) + i, keys > 0 ? acc[i] / l : 0.f);
    }
}

// CTAs a block's key tiles are shared out to.  A turn of a few queries over many earlier keys makes few blocks, each a long walk: where they leave half of
// the SMs without work, the walk is shared by as many CTAs as there is room for, four tiles each at least.  From the shape alone (the lengths are
// on the device), so that the workspace is known beforehand.
constexpr int SMS = 148;
int splits_of(const str_attn_packed_shape *s) {
    if (s->dtype != STR_BF16 || s->rows_q <= 0 || s->rows_k <= 0 || s->d > 128 || s->d % 8 != 0 || s->Hq / s->Hkv > BQ) return 1;
    const long long ctas = ((long long)s->rows_q / (2 * (BQ / (s->Hq / s->Hkv))) + s->n_seq) * s->Hkv, tiles = s->rows_k / s->n_seq / BKV;
    if (2 * ctas > SMS || tiles < 8) return 1;
    const long long n = SMS / ctas < tiles / 4 ? SMS / ctas : tiles / 4;
    return (int)(n < MAX_SPLITS ? n : MAX_SPLITS);
}
int blocks_of(const str_attn_packed_shape *s) { return s->rows_q / (2 * (BQ / (s->Hq / s->Hkv))) + s->n_seq; }   // at least as many as there are
int padded(int d) { return d <= 64 ? 64 : 128; }
Parts parts_in(const str_attn_packed_shape *s, void *workspace) {
    const int splits = splits_of(s);
    const size_t n = (size_t)blocks_of(s) * s->Hkv * splits;
    uint8_t *o = (uint8_t *)workspace, *stat = o + n * 2 * BQ * padded(s->d) * sizeof(float);
    int *found = (int *)(stat + n * 2 * BQ * sizeof(float2));
    return {splits, (float *)o, (float2 *)stat, found, (PackedBlock *)(found + n)};
}

template <int HD>
int launch(str_ctx *ctx, const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const int32_t *q_start, const int32_t *k_start,
           float scale, void *o, void *workspace, cudaStream_t st) {
    const int group = s->Hq / s->Hkv, TQ = BQ / group;
    CUtensorMap tq, tk, tv, to;
    int rc = str_make_tmap_heads_bf16_sw128(ctx, &tq, q, s->d, s->Hq, s->rows_q, group, TQ);
    if (rc == STR_OK) rc = str_make_tmap_heads_bf16_sw128(ctx, &tk, k, s->d, s->Hkv, s->rows_k, 1, BKV);
    if (rc == STR_OK) rc = str_make_tmap_heads_bf16_sw128(ctx, &tv, v, s->d, s->Hkv, s->rows_k, 1, BKV);
    if (rc == STR_OK) rc = str_make_tmap_heads_bf16_sw128(ctx, &to, o, s->d, s->Hq, s->rows_q, group, TQ);
    if (rc != STR_OK) return rc;
    rc = str_ensure_smem(ctx, HD == 64 ? STR_SMEM_ATTN_PACKED_64 : STR_SMEM_ATTN_PACKED_128, attn_packed_tc_kernel<HD>, Smem<HD>::BYTES);
    if (rc != STR_OK) return rc;
    const Parts parts = parts_in(s, workspace);
    const int blocks = blocks_of(s);
    const float scale_log2 = scale * 1.4426950408889634f;
    const __nv_bfloat16 *pq = (const __nv_bfloat16 *)q, *pk = (const __nv_bfloat16 *)k, *pv = (const __nv_bfloat16 *)v;
    attn_packed_tc_kernel<HD><<<blocks * s->Hkv * parts.splits, NUM_THREADS, Smem<HD>::BYTES, st>>>(
        tq, tk, tv, to, PackedBlockSize(2 * TQ), s->n_seq, s->rows_q, s->rows_k, s->Hq, s->Hkv, s->d, scale_log2, q_start, k_start, pq, pk, pv, (__nv_bfloat16 *)o, parts,
        ctx->status_dev);
    if (parts.splits == 1) return str_launch_ok(ctx);
    attn_packed_join_kernel<HD><<<dim3(blocks * s->Hkv, 16), JOIN_WARPS * 32, 0, st>>>(s->Hq, s->Hkv, s->d, scale_log2, pq, pk, pv, (__nv_bfloat16 *)o, parts,
                                                                                      ctx->status_dev);
    return str_launch_ok(ctx, 2);
}

}  // namespace

bool str_attn_packed_tc_supported(const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const void *o) {
    if (s->dtype != STR_BF16 || s->d > 128 || s->d % 8 != 0 || s->rows_k == 0 || s->Hq / s->Hkv > BQ) return false;
    return (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)o) & 15) == 0;
}

size_t str_attn_packed_tc_workspace(const str_attn_packed_shape *s) {
    const int splits = splits_of(s);
    if (splits == 1) return 0;
    const size_t n = (size_t)blocks_of(s) * s->Hkv;
    return align_up(n * splits * (2 * BQ * (padded(s->d) * sizeof(float) + sizeof(float2)) + sizeof(int)) + n * sizeof(PackedBlock), 256);
}

int str_attn_packed_tc(str_ctx *ctx, const str_attn_packed_shape *s, const void *q, const void *k, const void *v, const int32_t *q_start,
                       const int32_t *k_start, float scale, void *o, void *workspace, cudaStream_t st) {
    return s->d <= 64 ? launch<64>(ctx, s, q, k, v, q_start, k_start, scale, o, workspace, st)
                      : launch<128>(ctx, s, q, k, v, q_start, k_start, scale, o, workspace, st);
}

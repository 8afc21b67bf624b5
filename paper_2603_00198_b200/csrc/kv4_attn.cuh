// str_kv4_attn's kernels: attention of a sequence's newest tokens over its 4-bit cache, optionally adding the attention weights that
// every cached row has drawn to a running sum (the quantity str_kv4_evict ranks by).
//
// Mathematics.  A cached element is zero + scale * c with c in 0..15, so with the d elements of a row in groups g
//   q . k   = sum_g ( scale_g (q_g . c_g) + zero_g sum(q_g) )
//   o_e     = sum_t (p_t scale_t,g) (c_t,e - 8) + sum_t p_t (zero_t,g + 8 scale_t,g)      (g the group of element e)
// and q . k likewise with c - 8: the codes are centred so that neither sum is the small difference of two large ones.
// Both code products run on the matrix instruction, on codes turned into fp16 exactly: a byte put into the mantissa of 1024, its
// low nibble taken off again as c - 8 and what is left is 16 (c - 8) of the high one (codes2: eight instructions for eight codes; that
// small integers widen for nothing in a mantissa is well known);
// the powers of two go into q and into the output.  (The nibble as it stands would be the subnormal c 2^-24 for half of that, but the
// matrix instruction lines products up by the nominal exponent and then drops the last six to ten bits: measured, 5e-6 instead
// of 4e-7 of error.)
// The other factor is fp16: q scaled by a power of two to just below 2^15 (bf16 values fit exactly; fp32 storage takes two
// fp16 terms, 22 bits), and p scale times a power of two that a warp keeps for each query row and group (one rounding of 2^-11 for
// bf16 storage, two terms for fp32 storage).  One power for all of a warp's rows was 1 to 8 % faster (8448 rows 9.9 against 10.6 us,
// 65792 rows 22.8 against 23.3, five tokens over 18 x 16640 rows 269 against 283), but then a huge value took the bits of all others,
// even one without weight, in another group or seen by another head only.
// Products are summed in fp32; scales, zeros, the softmax and all sums stay fp32.
//
// Layout.  Codes are the A operand (16 rows of it 16 tokens for q.k, 16 elements for the output), the query rows of a
// key head (heads x tokens, padded to 8 or 16) the B operand, so one matrix instruction serves 8 query rows and the scores
// come out with the queries in the columns: the columns a lane holds are the same for the scores, the running maximum and
// the output.  The row order of the cache (kv4.cuh) is what makes a lane's codes one 16-byte (keys) or four 8-byte (values)
// loads.  Token order within 16 (slot r holds token r ^ (r >> 1 & 1)) keeps both free of worse than two-way bank conflicts.
//
// Split.  The work is one line of places: for every unit (sequence, key head, 4, 8 or 16 query rows) a few places for what it
// costs to begin one and then its tiles of 32 rows.  Two CTAs an SM take equal stretches of that line, whatever the lengths, so
// a long sequence is spread over the whole card and short ones share a CTA.  Within a CTA every warp takes every eighth
// tile, through its own ring of bulk copies, and keeps its own running maximum, sum and output; the warps meet in shared
// memory.  A unit that lies in one stretch is finished there; the parts of the others go to the workspace and a second
// kernel, set up while the first runs, joins them and adds the weights.  All sums are taken in a fixed order: no atomics.
#pragma once
#include <cuda_fp16.h>

#include <stddef.h>

#include <atomic>
#include <type_traits>

#include "kv4.cuh"
#include "tc_common.cuh"

namespace kv4_attn {

constexpr float LOG2E = 1.4426950408889634f;
constexpr int AT_TILE = 32;              // rows of a warp's tile
constexpr int AT_STAGES = 2;             // tiles in flight per warp
constexpr int WT_THREADS = 256;
constexpr int JOIN_BATCH = 5;            // parts a warp of the join loads at once: 8 x 5 cover one of 8 key heads spread over the card
constexpr float M_START = -3.0e38f;      // running maximum before the first row: finite, so that differences stay defined
constexpr float M_SLACK = 3.0f;          // the running maximum moves only when a score beats it by this (log2): p <= 2^3
// How far, in powers of two, an fp16 unit may be from the one that rows and maximum ask for: the largest p scale of a column and
// group is at least 2^(11 - window - lag) of its units, and half the smallest step of fp16 is 2^-25.
template <int TERMS> constexpr int UNIT_WINDOW = TERMS == 1 ? 12 : 8;
template <int TERMS> constexpr int UNIT_LAG = TERMS == 1 ? 4 : 3;
constexpr int UNIT_MAX = 253;            // biased exponent of the largest unit, 2^126: its reciprocal is a normal number

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                 : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// Transpose of an 8x8 tile of 16-bit elements held two per lane.
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t t;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(v));
    return t;
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *(const uint32_t *)&h;
}
// Bytes 0, 2 (LOW) or 1, 3 of a word as fp16: 1024 + byte, the byte put into the mantissa.  `magic` is 0x64006400 in a register
// that the compiler does not see through: mask and constant then are one instruction.
template <bool LOW>
__device__ __forceinline__ uint32_t bytes2(uint32_t w, uint32_t magic) {
    if constexpr (!LOW) return __byte_perm(w, magic, 0x7351);
    uint32_t v;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(v) : "r"(w), "n"(0x00FF00FF), "r"(magic));        // (w & mask) | magic
    return v;
}
// The two codes in each byte, c0 + 16 c1: with l = 1152 + c0 (`magic2` is 0x64806480), l - 1160 = c0 - 8 and
// (1024 + byte) - l = 16 (c1 - 8), exactly.
__device__ __forceinline__ void codes2(uint32_t byte, uint32_t magic2, uint32_t &lo, uint32_t &hi) {
    uint32_t l;
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(l) : "r"(byte), "n"(0x000F000F), "r"(magic2));
    const uint32_t k = 0xE488E488u;                                             // -1160
    const __half2 a = __hadd2(*(const __half2 *)&l, *(const __half2 *)&k), b = __hsub2(*(const __half2 *)&byte, *(const __half2 *)&l);
    lo = *(const uint32_t *)&a;
    hi = *(const uint32_t *)&b;
}
// x0, x1 as one (TERMS 1) or the sum of two (TERMS 2) fp16 pairs.
template <int TERMS>
__device__ __forceinline__ void split_half2(float x0, float x1, uint32_t (&t)[TERMS]) {
    const __half2 h = __floats2half2_rn(x0, x1);
    t[0] = *(const uint32_t *)&h;
    if constexpr (TERMS == 2) t[1] = pack_half2(x0 - __low2float(h), x1 - __high2float(h));
}
// N words of shared memory at a 32-bit address; stays behind the wait that says they are there.
template <int N>
__device__ __forceinline__ void load_words(uint32_t at, uint32_t (&w)[N]) {
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
    else if constexpr (N == 2)
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
    else
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
}

template <int D, int GROUP>
struct Stage {
    static constexpr int CODES = AT_TILE * D / 2, WORDS = AT_TILE * (D / GROUP) * 4, BYTES = 2 * CODES + 2 * WORDS;
};

// What p scale of a column and group is multiplied by to become the fp16 factor (a power of two; the output is kept in units of its
// reciprocal), for the two columns of a lane.  A unit comes from the scales and weights that its own column and group have met.
template <int NT, int NGP>
struct __align__(16) Units {
    uint32_t limit[4];                   // of group g: words up to this have p scale unit < 2^15 in all columns of the lane
    float2 of[NT][NGP];
    float2 change[NT][NGP];              // what they were last multiplied by
    float2 m[NT];                        // the running maximum when a column's units were last raised
};

// Neither the scale nor the zero of a word is infinite or NaN.
__device__ __forceinline__ bool finite_word(uint32_t w) { return (w & 0x7F800000u) != 0x7F800000u && (w & 0x7F80u) != 0x7F80u; }

struct AttnArgs {
    int Bz, cap, Hkv, Hq, n_q, chunks;
    const void *q;
    const int32_t *lens;
    float scale_log2;
    str_kv4_cache cache;
    void *o;
    float *part;         // [2 G][COLS][D] output of a run that is only a part of its unit, unnormalised, and
    float2 *part_ml;     // [2 G][COLS] its (maximum, sum)
    float *scores;       // [Bz,Hkv,cap,C] (log2 units) and
    float2 *stats;       // [Bz,Hkv,C] (maximum, 1 / sum) when the weights are wanted, else nullptr
    int *status;
};

// The flattened work: units (sequence, key head, block of columns) in that order; a unit is AT_UNIT_COST places, which stand
// for what it costs to begin one, and then its ceil(len / 32) tiles.  CTA i of G takes the places [i per, (i + 1) per).
constexpr int AT_UNIT_COST = 16;
__device__ __forceinline__ int clamp_len(int n, int cap) { return min(max(n, 0), cap); }
__device__ __forceinline__ int unit_places(int len) { return len ? (len + AT_TILE - 1) / AT_TILE + AT_UNIT_COST : 0; }
__device__ __forceinline__ long long divide(long long x, int y) {               // x >= 0, y > 0; the quick form nearly always
    return x >> 31 ? x / y : (long long)((uint32_t)x / (uint32_t)y);
}
// Places per CTA: a multiple of the warps, so that none idles while others work.
__device__ __forceinline__ int places_per_cta(long long total, int G, int NW) {
    return ((int)divide(total + G - 1, G) + NW - 1) / NW * NW;
}
// Places (of one column block of one head) of sequences 0 .. n-1, by one whole warp; every lane gets it.
__device__ __forceinline__ long long places_before(const int32_t *lens, int n, int cap, int lane) {
    long long sum = 0;
    for (int i = lane; i < n; i += 32) sum += unit_places(clamp_len(lens[i], cap));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    return sum;
}

// PACK 2: up to 4 query rows, and the eight columns of a matrix instruction hold them twice: columns 0-3 meet the first half
// of the groups, columns 4-7 the second half.  Scales, zeros and factors of a row are then split between the lanes instead
// of being worked on by all of them.
template <typename T, int D, int GROUP, int NT, int PACK, bool WEIGHTS, int NW>
__global__ void __launch_bounds__(NW * 32, NT == 1 ? 2 : 1)
kv4_attn_kernel(const AttnArgs a) {
    constexpr int TERMS = sizeof(T) == 2 ? 1 : 2;
    constexpr int NG = D / 32, NGR = D / GROUP, RPG = GROUP / 32, COLS = 8 * NT / PACK, NGP = NGR / PACK;
    static_assert(PACK == 1 || (NT == 1 && NGR % 2 == 0), "the halves of the groups share one set of columns");
    typedef Stage<D, GROUP> St;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t bars[NW][AT_STAGES];
    __shared__ float warp_m[NW][COLS], warp_l[NW][COLS];
    __shared__ float2 cta_ml[COLS];
    __shared__ Units<NT, NGP> units[NW][4];                                     // by a lane's c
    __shared__ uint4 q_frag[NT][NG][TERMS][32];                                 // q as the B operand, by lane
    __shared__ float q_top[NT][NG][8];                                          // max |q| of a column's elements of a run
    __shared__ float col_part[NG][COLS], col_mul[COLS];                         // sums of a column's scaled elements by run; what its scores are in
    __shared__ int col_limit[COLS];                                             // rows a column may see
    __shared__ int abort_flag;
    static_assert(NT * NG <= NW, "a warp prepares one run of one column block of q");

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = lane >> 2, c = lane & 3;
    const int R = a.Hq / a.Hkv, C = a.n_q * R, HC = a.Hkv * a.chunks;
    const int half = PACK == 2 ? c >> 1 : 0, cl = PACK == 2 ? c & 1 : c;        // half of the groups and column pair of this lane's results
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (tid == 0) abort_flag = 0;
    uint8_t *ring = smem + warp * AT_STAGES * St::BYTES;
    if (lane == 0) {
        for (int i = 0; i < AT_STAGES; ++i) tc::mbar_init(&bars[warp][i], 1);
        tc::fence_mbar_init();
    }
    if (blockIdx.x == 0)
        for (int i = tid; i < a.Bz; i += NW * 32)
            if (a.lens[i] < 0 || a.lens[i] > a.cap) kv4_report(a.status);
    // Every warp finds for itself where the CTA's places begin: the sequence and its first place.
    const int len32 = lane < a.Bz ? clamp_len(a.lens[lane], a.cap) : 0, places32 = unit_places(len32);
    long long total = __reduce_add_sync(0xffffffffu, places32);                 // below 2^31: a sequence has at most 2^25 tiles
    if (a.Bz > 32) total += places_before(a.lens + 32, a.Bz - 32, a.cap, lane);
    total *= HC;
    const int per = places_per_cta(total, gridDim.x, NW);
    const long long begin = (long long)blockIdx.x * per, end = min(begin + per, total);
    if (begin >= end) return;
    int b = 0, len = __shfl_sync(0xffffffffu, len32, 0);
    long long b_start = 0, b_end = (long long)__shfl_sync(0xffffffffu, places32, 0) * HC;      // places of sequence b: [b_start, b_end)
    if (begin >= b_end) {
        long long before = 0;
#pragma unroll 1
        for (int base = 0; base < a.Bz; base += 32) {
            const int n = base == 0 ? len32 : base + lane < a.Bz ? clamp_len(a.lens[base + lane], a.cap) : 0, t = unit_places(n);
            int incl = t;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += v;
            }
            const uint32_t past = __ballot_sync(0xffffffffu, before + (long long)incl * HC > begin);
            if (past) {
                const int k = __ffs(past) - 1;
                b = base + k;
                len = __shfl_sync(0xffffffffu, n, k);
                b_start = before + (long long)__shfl_sync(0xffffffffu, incl - t, k) * HC;
                b_end = before + (long long)__shfl_sync(0xffffffffu, incl, k) * HC;
                break;
            }
            before += (long long)__shfl_sync(0xffffffffu, incl, 31) * HC;
        }
    }
    long long at = begin;
    const int tr = r ^ ((r >> 1) & 1), va = 2 * c + (c & 1), vb = 2 * c + 1 - (c & 1);    // tokens of slots r, 2c, 2c+1
    int slot = 0;
    uint32_t phase = 0, magic, magic2;
    asm volatile("mov.b32 %0, 0x64006400;" : "=r"(magic));
    asm volatile("mov.b32 %0, 0x64806480;" : "=r"(magic2));

    while (at < end) {
        while (at >= b_end) {
            len = clamp_len(a.lens[++b], a.cap);
            b_start = b_end;
            b_end += (long long)unit_places(len) * HC;
        }
        const int places = unit_places(len), tiles = places - AT_UNIT_COST;
        const int hc = (int)divide(at - b_start, places), h = a.chunks == 1 ? hc : hc / a.chunks, col0 = (hc - h * a.chunks) * COLS;
        const long long u = b_start + (long long)hc * places;                   // the unit: [u, u + places)
        const int seg0 = max((int)(at - u) - AT_UNIT_COST, 0), seg1 = (int)min((long long)places, end - u) - AT_UNIT_COST;
        at = u + AT_UNIT_COST + seg1;
        if (seg1 <= 0) {                                                        // this CTA ends before the unit's first tile
            at = end;
            continue;
        }
        const int first = seg0 + warp, last = seg1;                             // this warp: every NW-th tile of the run
        const long long row0 = ((long long)b * a.Hkv + h) * a.cap;
        // q of this unit's columns as the B operand: lane (r, c) holds elements 32 s + 8 c + .. of column r (+ 8 j).  Warp
        // (j, s) prepares run s; the power of two that a column is scaled by goes by all its runs.
        const bool q_warp = warp < NT * NG;
        const int qj = warp / NG, qs = warp % NG, qcol = col0 + (PACK == 2 ? r & 3 : 8 * qj + r);
        float x[8];
        if (q_warp) {
            const int qc = min(qcol, C - 1), qi = a.n_q == 1 ? 0 : qc / R;
            kv4_load8((const T *)a.q + (((long long)b * a.n_q + qi) * a.Hq + h * R + qc - qi * R) * D + 8 * c + 32 * qs, x);
        }
        if (warp == NW - 1 && lane < COLS) {
            const int cc = col0 + lane;
            col_limit[lane] = cc < C ? len - a.n_q + (a.n_q == 1 ? 0 : cc / R) + 1 : 0;
        }
        // Lanes 0-3 fetch: key codes, value codes, key words, value words, each with its own source, place in the slot and
        // bytes per row.  The capacity is a multiple of 16 rows, so the 16 or 32 rows of a tile that are fetched are inside it.
        const int part_row = lane < 2 ? D / 2 : NGR * 4;
        const uint8_t *part_src = (const uint8_t *)(lane == 0 ? a.cache.k_codes : lane == 1 ? a.cache.v_codes : lane == 2 ? a.cache.k_scales : a.cache.v_scales) +
                                  (row0 + (long long)first * AT_TILE) * part_row;
        const uint32_t part_dst = tc::smem_u32(ring) + (lane < 2 ? lane * St::CODES : 2 * St::CODES + (lane - 2) * St::WORDS);
        auto fetch = [&](int tile, int sl) {                                    // tiles in the order in which the warp takes them
            if (lane < 4) {
                const uint32_t rows = len - tile * AT_TILE > 16 ? 32u : 16u, bar = tc::smem_u32(&bars[warp][sl]);
                if (lane == 0) tc::mbar_arrive_expect_tx(&bars[warp][sl], rows * (D + 2 * NGR * 4));
                bulk_load(part_dst + sl * St::BYTES, part_src, rows * part_row, bar);
                part_src += (long long)(NW * AT_TILE) * part_row;
            }
        };
#pragma unroll 1
        for (int i = 0; i < AT_STAGES; ++i)
            if (first + i * NW < last) fetch(first + i * NW, slot + i < AT_STAGES ? slot + i : slot + i - AT_STAGES);

        if (q_warp) {
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (qcol >= C) x[e] = 0.f;
                top = fmaxf(top, fabsf(x[e]));
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            if (c == 0) q_top[qj][qs][r] = top;
        }
        __syncthreads();
        if (q_warp) {
            float top = 0.f, sum = 0.f;
#pragma unroll
            for (int k = 0; k < NG; ++k) top = fmaxf(top, q_top[qj][k][r]);
            const int ex = max((int)(__float_as_uint(top) >> 23), 27);          // biased exponent
            const float mul = copysignf(__uint_as_float((uint32_t)(268 - ex) << 23), a.scale_log2);   // 2^(14 - exponent), with the scale's sign
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= mul;
            sum = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
            sum += __shfl_xor_sync(0xffffffffu, sum, 1);
            sum += __shfl_xor_sync(0xffffffffu, sum, 2);
            if (c == 0 && (PACK == 1 || r < 4)) {
                col_part[qs][8 * qj + r] = sum;
                if (qs == 0)                                                    // |scale| log2(e) 2^(exponent - 14); never zero: -inf x 0 is NaN
                    col_mul[8 * qj + r] = fmaxf((fabsf(a.scale_log2) * 6.103515625e-05f) * __uint_as_float((uint32_t)ex << 23), 1.2e-38f);
            }
            if (PACK == 2 && (r >> 2) != qs / RPG / NGP) {                      // these columns meet the other half of the groups
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = 0.f;
            }
            uint32_t t0[TERMS], t1[TERMS], t2[TERMS], t3[TERMS];
            split_half2<TERMS>(x[0], x[4], t0);
            split_half2<TERMS>(x[1] * 0.0625f, x[5] * 0.0625f, t1);
            split_half2<TERMS>(x[2], x[6], t2);
            split_half2<TERMS>(x[3] * 0.0625f, x[7] * 0.0625f, t3);
#pragma unroll
            for (int t = 0; t < TERMS; ++t) q_frag[qj][qs][t][lane] = make_uint4(t0[t], t1[t], t2[t], t3[t]);
        }
        __syncthreads();
        float q_sum[NT][NGP][2], q_mul[NT][2];
        int limit[NT][2];                                                       // rows that the columns of a lane's results may see
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int n = 8 * j + 2 * cl + i;
                q_mul[j][i] = col_mul[n];
                limit[j][i] = col_limit[n];
#pragma unroll
                for (int g = 0; g < NGP; ++g) {
                    float sum = col_part[(half * NGP + g) * RPG][n];
#pragma unroll
                    for (int k = 1; k < RPG; ++k) sum += col_part[(half * NGP + g) * RPG + k][n];
                    q_sum[j][g][i] = sum;
                }
            }

        // Scores stay in units of 1 / q_mul until the exponential; `bar` is where one of them moves the running maximum m (log2).
        float o[NT][2 * NG][4], z[NT][NGP][2], m[NT][2], l[NT][2], bar[NT][2];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
#pragma unroll
            for (int i = 0; i < 2 * NG; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[j][i][e] = 0.f;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                m[j][i] = M_START;
                bar[j][i] = -INFINITY;
                l[j][i] = 0.f;
#pragma unroll
                for (int g = 0; g < NGP; ++g) z[j][g][i] = 0.f;
            }
        }
        typedef Units<NT, NGP> Units_;
        Units_ &mine = units[warp][c];
        uint32_t units_at;                                                      // its address, kept (worked out anew it costs ten instructions a use)
        asm volatile("mov.u32 %0, %1;" : "=r"(units_at) : "r"(tc::smem_u32(&mine)));
        if (r == 0) {
            const float most = __uint_as_float((uint32_t)UNIT_MAX << 23);
#pragma unroll
            for (int g = 0; g < NGP; ++g) mine.limit[g] = 0u;
#pragma unroll
            for (int j = 0; j < NT; ++j) {
#pragma unroll
                for (int g = 0; g < NGP; ++g) mine.of[j][g] = make_float2(most, most);
                mine.m[j] = make_float2(M_START, M_START);
            }
        }
        __syncwarp();
        const int all = len - a.n_q + 1;                                        // rows that every column sees

        // One tile.  EDGE: some column may not see some row.
        const uint32_t q_at = tc::smem_u32(&q_frag[0][0][0][lane]);
        auto work = [&](auto edge_tag, const int sl, const int t0) {
            constexpr bool EDGE = decltype(edge_tag)::value;
            const uint32_t st = tc::smem_u32(ring) + sl * St::BYTES;
            if constexpr (EDGE) {
                // A row that only some columns see and whose value words are not finite: NaN for the groups of the columns that
                // see it, and zero words for the others.  Rows behind the sequence: zero words.
                uint32_t *kwords = (uint32_t *)(ring + sl * St::BYTES + 2 * St::CODES), *vwords = kwords + AT_TILE * NGR;
#pragma unroll 1
                for (int t = max(all - t0, 0); t < min(len - t0, AT_TILE); ++t) {
#pragma unroll
                    for (int g = 0; g < NGP; ++g)
                        if (!finite_word(vwords[t * NGR + half * NGP + g]))
#pragma unroll
                            for (int j = 0; j < NT; ++j)
#pragma unroll
                                for (int i = 0; i < 2; ++i)
                                    if (t0 + t < limit[j][i]) z[j][g][i] = __uint_as_float(0x7FFFFFFFu);
                }
                __syncwarp();
                const bool gone = t0 + lane >= len;                             // lane = row
                if (t0 + lane >= all) {
#pragma unroll
                    for (int g = 0; g < NGR; ++g) {
                        if (gone) kwords[lane * NGR + g] = 0u;
                        if (gone || !finite_word(vwords[lane * NGR + g])) vwords[lane * NGR + g] = 0u;
                    }
                }
                tc::fence_proxy_async();
                __syncwarp();
            }
            // Sixteen rows at a time: the code of one half serves both, which halves what has to come through the instruction cache.
#pragma unroll 1
            for (int t16 = 0; t16 < AT_TILE; t16 += 16) {
                const int ta = t16 + tr, tb = ta + 8;                           // rows of slots r, r + 8
                uint32_t ka[NG], kb[NG], wa[NGP], wb[NGP];
                load_words<NG>(st + ta * (D / 2) + c * (4 * NG), ka);
                load_words<NG>(st + tb * (D / 2) + c * (4 * NG), kb);
                load_words<NGP>(st + 2 * St::CODES + ta * (4 * NGR) + half * (4 * NGP), wa);
                load_words<NGP>(st + 2 * St::CODES + tb * (4 * NGR) + half * (4 * NGP), wb);
                float s[NT][4];
#pragma unroll
                for (int g = 0; g < NGP; ++g) {
                    const float sa = kv4_scale(wa[g]), za = fmaf(8.f, sa, kv4_zero(wa[g])), sb = kv4_scale(wb[g]), zb = fmaf(8.f, sb, kv4_zero(wb[g]));
                    float acc[NT][4];
#pragma unroll
                    for (int k = 0; k < PACK * RPG; ++k) {                      // the runs of group g (and with each that of its partner in the other half)
                        const int q = (g + k % PACK * NGP) * RPG + k / PACK;
                        // The instruction truncates its sums.  For bf16 storage a group is summed in it whole; for fp32 storage only a
                        // run, low terms first, and the runs outside it.
                        const bool fresh = TERMS == 2 ? k % PACK == 0 : k == 0, done = TERMS == 2 ? k % PACK == PACK - 1 : k == PACK * RPG - 1;
                        uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                        codes2(bytes2<true>(ka[q], magic), magic2, a0, a2);
                        codes2(bytes2<true>(kb[q], magic), magic2, a1, a3);
                        codes2(bytes2<false>(ka[q], magic), magic2, b0, b2);
                        codes2(bytes2<false>(kb[q], magic), magic2, b1, b3);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
#pragma unroll
                            for (int t = TERMS - 1; t >= 0; --t) {
                                uint32_t qf[4];                                 // from shared memory every time: registers are what is short
                                load_words<4>(q_at + ((j * NG + q) * TERMS + t) * 512, qf);
                                if (fresh && t == TERMS - 1) mma_f16_first(acc[j], a0, a1, a2, a3, qf[0], qf[1]);
                                else mma_f16(acc[j], a0, a1, a2, a3, qf[0], qf[1]);
                                mma_f16(acc[j], b0, b1, b2, b3, qf[2], qf[3]);
                            }
                            if (done) {
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float y = e < 2 ? za : zb;
                                    if (k / PACK == (TERMS == 2 ? 0 : RPG - 1))
                                        s[j][e] = g == 0 ? y * q_sum[j][g][e & 1] : fmaf(y, q_sum[j][g][e & 1], s[j][e]);
                                    s[j][e] = fmaf(e < 2 ? sa : sb, acc[j][e], s[j][e]);
                                }
                            }
                        }
                    }
                }
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if constexpr (PACK == 2) s[j][e] += __shfl_xor_sync(0xffffffffu, s[j][e], 2);
                    }
                if constexpr (EDGE) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (t0 + (e < 2 ? ta : tb) >= limit[j][e & 1]) s[j][e] = -INFINITY;
                }
                if (WEIGHTS && (PACK == 1 || half == 0)) {
#pragma unroll
                    for (int j = 0; j < NT; ++j)
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int t = t0 + (e < 2 ? ta : tb), cc = col0 + 8 * j + 2 * cl;
                            if ((!EDGE || t < len) && cc < C) {
                                float *dst = a.scores + (row0 + t) * C + cc;
                                const float s0 = __fmul_rn(s[j][e], q_mul[j][0]), s1 = __fmul_rn(s[j][e + 1], q_mul[j][1]);
                                if (C % 2 == 0) *(float2 *)dst = make_float2(s0, s1);
                                else {
                                    dst[0] = s0;
                                    if (cc + 1 < C) dst[1] = s1;
                                }
                            }
                        }
                }
                // value words of this lane's two rows; does the running maximum or a unit move?
                const uint32_t words_at = st + 2 * St::CODES + St::WORDS + half * (4 * NGP);
                load_words<NGP>(words_at + ta * (4 * NGR), wa);
                load_words<NGP>(words_at + tb * (4 * NGR), wb);
                bool rises = false, beyond = false;
                uint32_t limit_word[NGP];
                load_words<NGP>(units_at + (uint32_t)offsetof(Units_, limit), limit_word);
#pragma unroll
                for (int g = 0; g < NGP; ++g) beyond |= max(wa[g], wb[g]) > limit_word[g];
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < 2; ++i) rises |= fmaxf(s[j][i], s[j][i + 2]) > bar[j][i];
                if (__any_sync(0xffffffffu, rises || beyond)) {
                    float2 by[NT][NGP];                                         // what the output is multiplied by
                    bool scale_output = __any_sync(0xffffffffu, rises);
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        float f[2] = {1.f, 1.f};
                        if (scale_output)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                float t = fmaxf(s[j][i], s[j][i + 2]) * q_mul[j][i];
                                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 4));
                                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
                                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
                                t = fmaxf(t, m[j][i]);
                                f[i] = ex2(m[j][i] - t);
                                m[j][i] = t;
                                beyond |= t - (i ? mine.m[j].y : mine.m[j].x) > (float)UNIT_LAG<TERMS>;
                                // (t + slack) / q_mul, less what its roundings can add (1.5 2^-23 of the reciprocal and product): a score up to
                                // the bar lies no more than the slack above t once it has been multiplied and rounded (a quotient to nearest
                                // let scores of 3e7 lie 8 above); a scale of zero: beyond reach
                                const float over = __fadd_rd(t, M_SLACK) * rcp(q_mul[j][i]);
                                bar[j][i] = fmaf(fabsf(over), -4.76837158203125e-07f, over);
                                l[j][i] *= f[i];
#pragma unroll
                                for (int g = 0; g < NGP; ++g) z[j][g][i] *= f[i];
                            }
#pragma unroll
                        for (int g = 0; g < NGP; ++g) by[j][g] = make_float2(f[0], f[1]);
                    }
                    if (__any_sync(0xffffffffu, beyond)) {
                        // A maximum has risen by 2^up since its column's units were set, so what was added up weighs less by that and the
                        // units may grow; then these rows hold them down: the largest scale of the sixteen becomes 2^11 .. 2^12, as long as
                        // it is no more than 2^UNIT_WINDOW times the largest p scale, else that limit does.  Where nothing of that changes
                        // a unit (scales beyond the limit that draw next to no weight) this ends early.
                        constexpr int N = 2 * NT * NGP;
                        float v[N];
                        int up[NT][2];
                        beyond = false;
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const float t = m[j][i], rise = fminf(floorf(t - (i ? mine.m[j].y : mine.m[j].x)), 512.f);
                                const float pa = ex2(__fmul_rn(s[j][i], q_mul[j][i]) - t), pb = ex2(__fmul_rn(s[j][i + 2], q_mul[j][i]) - t);
                                up[j][i] = (int)rise;
                                beyond |= rise > (float)UNIT_LAG<TERMS>;
#pragma unroll
                                for (int g = 0; g < NGP; ++g) {
                                    const int n = (j * NGP + g) * 2 + i;
                                    v[n] = fmaxf(pa * fabsf(kv4_scale(wa[g])), pb * fabsf(kv4_scale(wb[g])));
                                    beyond |= v[n] * (i ? mine.of[j][g].y : mine.of[j][g].x) >= 4096.f / (1 << UNIT_WINDOW<TERMS>);
                                }
                            }
                        if (__any_sync(0xffffffffu, beyond)) {
                            // The largest are reduced and scattered over the lanes r: lane r ends up with the unit of index r (modulo their
                            // number; r and r + 8 of sixteen), in the order of `of`.
                            scale_output = true;
#pragma unroll
                            for (int g = 0; g < NGP; ++g) {
                                float top = fmaxf(fabsf(kv4_scale(wa[g])), fabsf(kv4_scale(wb[g])));
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 4));
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 8));
                                top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 16));
#pragma unroll
                                for (int j = 0; j < NT; ++j)
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        const int n = (j * NGP + g) * 2 + i;
                                        v[n] = fminf(v[n] * (1 << UNIT_WINDOW<TERMS>), top);
                                    }
                            }
                            if (r == 0)
#pragma unroll
                                for (int j = 0; j < NT; ++j) {
                                    float2 was = mine.m[j];
                                    was.x = up[j][0] < 512 ? was.x + (float)up[j][0] : m[j][0];
                                    was.y = up[j][1] < 512 ? was.y + (float)up[j][1] : m[j][1];
                                    mine.m[j] = was;
                                }
#pragma unroll
                            for (int o = 1, n = N; o < 8; o <<= 1, n = n > 1 ? n / 2 : 1) {
                                const bool odd = r & o;
                                if (n == 1) v[0] = fmaxf(v[0], __shfl_xor_sync(0xffffffffu, v[0], 4 * o));
                                else
#pragma unroll
                                    for (int k = 0; k < n / 2; ++k) {
                                        const float keep = odd ? v[2 * k + 1] : v[2 * k], send = odd ? v[2 * k] : v[2 * k + 1];
                                        v[k] = fmaxf(keep, __shfl_xor_sync(0xffffffffu, send, 4 * o));
                                    }
                            }
#pragma unroll
                            for (int k = 0; k < (N > 8 ? N / 8 : 1); ++k) {
                                const int n = 8 * k + (N < 8 ? r % N : r), j = NT == 1 ? 0 : n / (2 * NGP);
                                float *unit = (float *)mine.of + n;
                                int rise = n & 1 ? up[0][1] : up[0][0];
                                if (NT == 2 && j == 1) rise = n & 1 ? up[NT - 1][1] : up[NT - 1][0];
                                const int was = (int)(__float_as_uint(*unit) >> 23), now = min(min(was + rise, UNIT_MAX), 265 - (int)(__float_as_uint(v[k]) >> 23));
                                ((float *)mine.change)[n] = __uint_as_float((uint32_t)max(127 + min(now - was, 127), 0) << 23);
                                __syncwarp();
                                *unit = __uint_as_float((uint32_t)now << 23);
                            }
                            __syncwarp();
#pragma unroll
                            for (int g = 0; g < NGP; ++g) {
                                float most = 0.f;
#pragma unroll
                                for (int j = 0; j < NT; ++j) {
                                    by[j][g].x *= mine.change[j][g].x;
                                    by[j][g].y *= mine.change[j][g].y;
                                    most = fmaxf(most, fmaxf(mine.of[j][g].x, mine.of[j][g].y));
                                }
                                if (r == 0) mine.limit[g] = 0x84FFFFFFu - __float_as_uint(most);     // exponent 265 - the largest's, all ones behind
                            }
                            __syncwarp();
                        }
                    }
                    if (scale_output)
#pragma unroll
                        for (int j = 0; j < NT; ++j)
#pragma unroll
                            for (int q = 0; q < NG; ++q)                        // with PACK 2 a lane's values of the other half's groups are not used
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    o[j][2 * q][e] *= e & 1 ? by[j][q / RPG % NGP].y : by[j][q / RPG % NGP].x;
                                    o[j][2 * q + 1][e] *= e & 1 ? by[j][q / RPG % NGP].y : by[j][q / RPG % NGP].x;
                                }
                }
                float p[NT][4];
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        p[j][e] = ex2(__fmul_rn(s[j][e], q_mul[j][e & 1]) - m[j][e & 1]);   // the product as the weights' scores hold it
                        l[j][e & 1] += p[j][e];
                    }
                // codes of the tokens of slots 2c, 2c+1 (+8): this lane's quarter-words of all runs
                constexpr int NV = NG / 2;
                uint32_t v0[NV], v1[NV], v2[NV], v3[NV];
                const uint32_t vrow = st + St::CODES + t16 * (D / 2) + r * (4 * NV);
                load_words<NV>(vrow + va * (D / 2), v0);
                load_words<NV>(vrow + vb * (D / 2), v1);
                load_words<NV>(vrow + (va + 8) * (D / 2), v2);
                load_words<NV>(vrow + (vb + 8) * (D / 2), v3);
#pragma unroll
                for (int g = 0; g < NGP; ++g) {
                    const float ua = kv4_scale(wa[g]), ub = kv4_scale(wb[g]);
                    const float za = fmaf(8.f, ua, kv4_zero(wa[g])), zb = fmaf(8.f, ub, kv4_zero(wb[g]));
                    uint32_t pb[NT][TERMS][2];
#pragma unroll
                    for (int j = 0; j < NT; ++j) {
                        const float2 unit = mine.of[j][g];
                        float w[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) {                           // p times scale first: scale times unit may be infinite where p is tiny
                            w[e] = p[j][e] * (e < 2 ? ua : ub) * (e & 1 ? unit.y : unit.x);
                            z[j][g][e & 1] = fmaf(p[j][e], e < 2 ? za : zb, z[j][g][e & 1]);
                        }
                        uint32_t h0[TERMS], h1[TERMS];
                        split_half2<TERMS>(w[0], w[1], h0);
                        split_half2<TERMS>(w[2], w[3], h1);
#pragma unroll
                        for (int t = 0; t < TERMS; ++t) { pb[j][t][0] = transpose8x8(h0[t]); pb[j][t][1] = transpose8x8(h1[t]); }
                    }
#pragma unroll
                    for (int k = 0; k < PACK * RPG; ++k) {
                        const int q = g * RPG + k % RPG + (k / RPG) * NGP * RPG;
                        const uint32_t sel = q & 1 ? 0x7632u : 0x5410u;
                        const uint32_t xl = __byte_perm(v0[q / 2], v1[q / 2], sel), xh = __byte_perm(v2[q / 2], v3[q / 2], sel);
                        uint32_t a0, a1, a2, a3, b0, b1, b2, b3;
                        codes2(bytes2<true>(xl, magic), magic2, a0, a1);
                        codes2(bytes2<true>(xh, magic), magic2, a2, a3);
                        codes2(bytes2<false>(xl, magic), magic2, b0, b1);
                        codes2(bytes2<false>(xh, magic), magic2, b2, b3);
#pragma unroll
                        for (int j = 0; j < NT; ++j) {
                            if constexpr (TERMS == 1) {
                                mma_f16(o[j][2 * q], a0, a1, a2, a3, pb[j][0][0], pb[j][0][1]);
                                mma_f16(o[j][2 * q + 1], b0, b1, b2, b3, pb[j][0][0], pb[j][0][1]);
                            } else {
                                // The instruction truncates its sums, always the same way: for fp32 storage it only adds up the sixteen
                                // rows, low terms first, and the running sum is rounded to nearest outside it.
                                float f0[4], f1[4];
                                mma_f16_first(f0, a0, a1, a2, a3, pb[j][1][0], pb[j][1][1]);
                                mma_f16_first(f1, b0, b1, b2, b3, pb[j][1][0], pb[j][1][1]);
                                mma_f16(f0, a0, a1, a2, a3, pb[j][0][0], pb[j][0][1]);
                                mma_f16(f1, b0, b1, b2, b3, pb[j][0][0], pb[j][0][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    o[j][2 * q][e] += f0[e];
                                    o[j][2 * q + 1][e] += f1[e];
                                }
                            }
                        }
                    }
                }
            }
        };

        int tile = first;
        for (; tile < last; tile += NW) {
            if (!__all_sync(0xffffffffu, tc::mbar_wait(&bars[warp][slot], phase, &abort_flag))) {
                if (lane == 0) atomicCAS(a.status, 0, STR_ERR_TIMEOUT);
                break;
            }
            if (tile * AT_TILE + AT_TILE <= all) work(std::false_type{}, slot, tile * AT_TILE);
            else work(std::true_type{}, slot, tile * AT_TILE);
            __syncwarp();                                                       // every lane has taken its rows out of the slot
            if (tile + AT_STAGES * NW < last) fetch(tile + AT_STAGES * NW, slot);
            if (++slot == AT_STAGES) { slot = 0; phase ^= 1u; }
        }
        if (tile < last) {
            // a wait gave up: let the copies still under way land (again with a limit) before this shared memory is used otherwise
            uint32_t probes = 0;
            for (int i = 0; i < AT_STAGES && tile < last; ++i, tile += NW) {
                while (!tc::mbar_try_wait(&bars[warp][slot], phase) && ++probes < tc::WAIT_PROBE_LIMIT) { }
                if (++slot == AT_STAGES) { slot = 0; phase ^= 1u; }
            }
            __syncwarp();
        }

        // the warp's sums over its lanes, its output in true units: [column][element] in its own ring
        float *wo = (float *)ring;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int off = 4; off <= 16; off <<= 1) {
                    l[j][i] += __shfl_xor_sync(0xffffffffu, l[j][i], off);
#pragma unroll
                    for (int g = 0; g < NGP; ++g) z[j][g][i] += __shfl_xor_sync(0xffffffffu, z[j][g][i], off);
                }
                const int cc = 8 * j + 2 * cl + i;
                if (r == 0 && half == 0) { warp_m[warp][cc] = m[j][i]; warp_l[warp][cc] = l[j][i]; }
#pragma unroll
                for (int q = 0; q < NG; ++q) {
                    if (PACK == 2 && q / RPG / NGP != half) continue;           // the other half's columns hold these groups
                    const float zq = z[j][q / RPG % NGP][i], f1 = 0.0625f;
                    const float2 unit = mine.of[j][q / RPG % NGP];
                    const float e_out = __uint_as_float(0x7F000000u - __float_as_uint(i ? unit.y : unit.x));        // 1 / unit
                    *(float4 *)(wo + cc * D + 32 * q + 4 * r) =
                        make_float4(fmaf(o[j][2 * q][i], e_out, zq), fmaf(o[j][2 * q][i + 2] * f1, e_out, zq),
                                    fmaf(o[j][2 * q + 1][i], e_out, zq), fmaf(o[j][2 * q + 1][i + 2] * f1, e_out, zq));
                }
            }
        __syncthreads();
        if (tid < COLS) {                                                       // the run's maximum and what each warp counts for
            float top = M_START, sum = 0.f;
#pragma unroll
            for (int w = 0; w < NW; ++w) top = fmaxf(top, warp_m[w][tid]);
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = ex2(warp_m[w][tid] - top);
                sum = fmaf(warp_l[w][tid], f, sum);
                warp_m[w][tid] = f;
            }
            cta_ml[tid] = make_float2(top, sum);
        }
        __syncthreads();
        // Warps in order.  A whole unit is finished here; a part goes to the workspace, to the CTA's second slot if the
        // unit's first tile lies behind the CTA's first place, else to its first.
        const bool whole = seg0 == 0 && seg1 == tiles;
        const long long place = 2LL * blockIdx.x + (begin < u + AT_UNIT_COST ? 1 : 0);
        for (int i = tid; i < COLS * D / 4; i += NW * 32) {
            const int cc = 4 * i / D, col = col0 + cc;
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = warp_m[w][cc];
                const float4 v = ((const float4 *)(smem + w * AT_STAGES * St::BYTES))[i];
                sum[0] = fmaf(v.x, f, sum[0]); sum[1] = fmaf(v.y, f, sum[1]); sum[2] = fmaf(v.z, f, sum[2]); sum[3] = fmaf(v.w, f, sum[3]);
            }
            const float2 ml = cta_ml[cc];
            if (!whole) {
                ((float4 *)(a.part + place * (COLS * D)))[i] = make_float4(sum[0], sum[1], sum[2], sum[3]);
                if (4 * i % D == 0) a.part_ml[place * COLS + cc] = ml;
            } else if (col < C) {
                T *dst = (T *)a.o + (((long long)b * a.n_q + col / R) * a.Hq + h * R + col % R) * D + 4 * i % D;
#pragma unroll
                for (int e = 0; e < 4; ++e) stf(dst + e, ml.y == 0.f ? 0.f : sum[e] / ml.y);
                if (WEIGHTS && 4 * i % D == 0) a.stats[((long long)b * a.Hkv + h) * C + col] = make_float2(ml.x, ml.y == 0.f ? 0.f : 1.f / ml.y);
            }
        }
        tc::fence_proxy_async();                                                // what was written to the rings comes before the next copies into them
        __syncthreads();                                                        // the rings and the sums are free again
        if (abort_flag) return;                                                 // a wait gave up: its barriers are not to be used again
    }
}

// Joins the runs of the units that more than one CTA worked on, gives zeros to the units without rows, and adds the weights:
//   weight_out[b,h,t] = weight[b,h,t] + sum over the columns of exp2(s - m) / l, columns in order.
// Grid (blocks, Hkv, Bz).  Every block of a (sequence, key head) works out the columns' maxima and sums again; blocks share the
// output's elements and the rows.
template <typename T, int D>
__global__ void __launch_bounds__(WT_THREADS)
kv4_join_kernel(const AttnArgs a, int cols, int G, int NW, const float *weight, float *weight_out) {
    extern __shared__ float2 ml[];                                              // [C] (maximum, 1 / sum)
    const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x;
    const int R = a.Hq / a.Hkv, C = a.n_q * R, HC = a.Hkv * a.chunks;
    __shared__ long long before, total;
    __shared__ float4 sums[WT_THREADS / 32][32];
    __shared__ float2 runs[WT_THREADS / 32][32];
    const int len = clamp_len(a.lens[b], a.cap), places = unit_places(len), tiles = max(places - AT_UNIT_COST, 0);
    if (blockIdx.x * 128 >= C * D && (!weight_out || blockIdx.x * (4 * WT_THREADS) >= len)) return;   // nothing for this block
    if (tid < 32) {
        long long t0 = 0, t1 = 0;                                               // places before sequence b, and in all
        for (int base = 0; base < a.Bz; base += 32) {
            const int n = base + tid < a.Bz ? unit_places(clamp_len(a.lens[base + tid], a.cap)) : 0;
            t0 += __reduce_add_sync(0xffffffffu, base + tid < b ? n : 0);
            t1 += __reduce_add_sync(0xffffffffu, n);
        }
        if (tid == 0) { before = t0 * HC; total = t1 * HC; }
    }
    __syncthreads();
    const int per = max(places_per_cta(total, G, NW), 1);
    const int lane = tid & 31, warp = tid >> 5;
    // The output, 128 elements at a time: warp w takes the parts w, w + 8, .. with a running maximum, JOIN_BATCH of them in flight,
    // then the warps are joined in order.  Where the first elements' parts lie is worked out before the wait.
    int i0 = blockIdx.x * 128, i, col, block;
    long long u, c0, c1;
    auto locate = [&]() {
        i = i0 + 4 * lane;
        col = i / D;
        block = col / cols;
        u = before + (long long)(h * a.chunks + block) * places + AT_UNIT_COST;                        // the unit's first tile
        c0 = tiles ? divide(u, per) : 0;
        c1 = tiles ? divide(u + tiles - 1, per) : -1;
    };
    locate();
    asm volatile("griddepcontrol.wait;" ::: "memory");                          // all that the first kernel wrote is there
    while (i0 < C * D) {
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
        float2 run = make_float2(M_START, 0.f);
        const bool mine = i < C * D && c0 != c1;                                // else finished by the one CTA that had it
        for (long long k0 = c0 + warp; mine && k0 <= c1; k0 += JOIN_BATCH * (WT_THREADS / 32)) {
            float2 v[JOIN_BATCH];
            float4 w[JOIN_BATCH];
#pragma unroll
            for (int n = 0; n < JOIN_BATCH; ++n) {
                const long long k = k0 + n * (WT_THREADS / 32);
                if (k > c1) continue;
                const long long place = (2 * k + (k * per < u ? 1 : 0)) * cols + col - block * cols;
                v[n] = a.part_ml[place];
                w[n] = *(const float4 *)(a.part + place * D + i % D);
            }
#pragma unroll
            for (int n = 0; n < JOIN_BATCH; ++n) {
                if (k0 + n * (WT_THREADS / 32) > c1) continue;
                const float top = fmaxf(run.x, v[n].x), f = ex2(run.x - top), g = ex2(v[n].x - top);
                run = make_float2(top, fmaf(run.y, f, v[n].y * g));
                sum.x = fmaf(sum.x, f, w[n].x * g); sum.y = fmaf(sum.y, f, w[n].y * g);
                sum.z = fmaf(sum.z, f, w[n].z * g); sum.w = fmaf(sum.w, f, w[n].w * g);
            }
        }
        __syncthreads();                                                        // the sums of the round before have been read
        sums[warp][lane] = sum;
        runs[warp][lane] = run;
        __syncthreads();
        if (warp == 0 && mine) {
            float top = M_START, total_l = 0.f;
#pragma unroll
            for (int w = 0; w < WT_THREADS / 32; ++w) top = fmaxf(top, runs[w][lane].x);
            sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < WT_THREADS / 32; ++w) {
                const float4 v = sums[w][lane];
                const float f = ex2(runs[w][lane].x - top);
                total_l = fmaf(runs[w][lane].y, f, total_l);
                sum.x = fmaf(v.x, f, sum.x); sum.y = fmaf(v.y, f, sum.y); sum.z = fmaf(v.z, f, sum.z); sum.w = fmaf(v.w, f, sum.w);
            }
            const float inv = total_l == 0.f ? 0.f : 1.f / total_l;             // no row to see: zeros
            T *dst = (T *)a.o + (((long long)b * a.n_q + col / R) * a.Hq + h * R + col % R) * D + i % D;
            stf(dst, sum.x * inv); stf(dst + 1, sum.y * inv); stf(dst + 2, sum.z * inv); stf(dst + 3, sum.w * inv);
        }
        i0 += gridDim.x * 128;
        locate();
    }
    if (!weight_out) return;
    // The columns' maxima and sums: a warp a column, the lanes over its parts.
    for (int col = warp; col < C; col += WT_THREADS / 32) {
        const long long u = before + (long long)(h * a.chunks + col / cols) * places + AT_UNIT_COST;
        const long long c0 = tiles ? divide(u, per) : 0, c1 = tiles ? divide(u + tiles - 1, per) : -1;
        float top = M_START, sum = 0.f;
        if (c0 == c1) {
            if (lane == 0) ml[col] = a.stats[((long long)b * a.Hkv + h) * C + col];
            continue;
        }
        for (long long i = c0 + lane; i <= c1; i += 32) top = fmaxf(top, a.part_ml[(2 * i + (i * per < u ? 1 : 0)) * cols + col % cols].x);
        top = warp_max(top);
        for (long long i = c0 + lane; i <= c1; i += 32) {
            const float2 v = a.part_ml[(2 * i + (i * per < u ? 1 : 0)) * cols + col % cols];
            sum = fmaf(v.y, ex2(v.x - top), sum);
        }
        sum = warp_sum(sum);
        if (lane == 0) ml[col] = make_float2(top, sum == 0.f ? 0.f : 1.f / sum);
    }
    __syncthreads();
    const long long row0 = ((long long)b * a.Hkv + h) * a.cap;
    // Four rows a thread at a time, their loads together.
    for (int t0 = blockIdx.x * (4 * WT_THREADS) + tid; t0 < len; t0 += gridDim.x * (4 * WT_THREADS)) {
        float sum[4], old[4];
        int row[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            row[k] = min(t0 + k * WT_THREADS, len - 1);                         // behind the end: the last row again, not stored
            old[k] = weight[row0 + row[k]];
            sum[k] = 0.f;
        }
        if (C % 4 == 0) {
            for (int cc = 0; cc < C; cc += 4) {
                float4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = *(const float4 *)(a.scores + (row0 + row[k]) * C + cc);
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    sum[k] = fmaf(ex2(v[k].x - ml[cc].x), ml[cc].y, sum[k]);
                    sum[k] = fmaf(ex2(v[k].y - ml[cc + 1].x), ml[cc + 1].y, sum[k]);
                    sum[k] = fmaf(ex2(v[k].z - ml[cc + 2].x), ml[cc + 2].y, sum[k]);
                    sum[k] = fmaf(ex2(v[k].w - ml[cc + 3].x), ml[cc + 3].y, sum[k]);
                }
            }
        } else {
            for (int cc = 0; cc < C; ++cc) {
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = a.scores[(row0 + row[k]) * C + cc];
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] = fmaf(ex2(v[k] - ml[cc].x), ml[cc].y, sum[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (t0 + k * WT_THREADS < len) weight_out[row0 + row[k]] = old[k] + sum[k];
    }
}

constexpr int AT_WARPS = 8;

// Query rows of one unit: 4 (twice in the eight columns of a matrix instruction), 8, or 16.
inline int unit_columns(const str_kv4_shape *s, int C) { return C <= 4 && s->d / s->group >= 2 ? 4 : C <= 8 ? 8 : 16; }

// Workspace: parts | their maxima and sums | scores | maxima and sums of the columns (the last two with weights only).
struct Ws { size_t part, part_ml, scores, stats, bytes; };
inline Ws ws_layout(const str_kv4_shape *s, int Hq, int n_q, int G, bool weights) {
    const int C = n_q * (Hq / s->Hkv), cols = unit_columns(s, C);
    Ws w;
    w.part = 0;
    w.part_ml = w.part + align_up((size_t)2 * G * cols * s->d * sizeof(float), 256);
    w.scores = w.part_ml + align_up((size_t)2 * G * cols * sizeof(float2), 256);
    w.stats = w.scores + (weights ? align_up((size_t)s->Bz * n_q * Hq * s->cap * sizeof(float), 256) : 0);
    w.bytes = w.stats + (weights ? align_up((size_t)s->Bz * n_q * Hq * sizeof(float2), 256) : 0);
    return w;
}

template <typename T, int D, int GROUP, int NT, int PACK>
int launch_attn(str_ctx *ctx, const AttnArgs &a, int G, const float *weight, float *weight_out, cudaStream_t st) {
    constexpr int COLS = 8 * NT / PACK;
    auto kernel = a.scores ? kv4_attn_kernel<T, D, GROUP, NT, PACK, true, AT_WARPS> : kv4_attn_kernel<T, D, GROUP, NT, PACK, false, AT_WARPS>;
    const size_t smem = (size_t)AT_WARPS * AT_STAGES * Stage<D, GROUP>::BYTES;
    static_assert(AT_STAGES * Stage<D, GROUP>::BYTES >= COLS * D * 4, "a warp's output has to fit its ring");
    if (smem > (size_t)ctx->max_smem_optin) return STR_ERR_UNSUPPORTED_SHAPE;
    // The attribute belongs to the device's copy of the kernel: set once per device and kernel (twice by two threads does no harm).
    static std::atomic<uint64_t> opted[2];
    const uint64_t bit = ctx->device < 64 ? 1ull << ctx->device : 0;
    if (!(opted[a.scores != nullptr].load(std::memory_order_acquire) & bit)) {
        STR_CUDA_OK(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
        opted[a.scores != nullptr].fetch_or(bit, std::memory_order_release);
    }
    kernel<<<G, AT_WARPS * 32, smem, st>>>(a);
    int rc = str_launch_ok(ctx);
    if (rc != STR_OK) return rc;
    // The join may be set up while the first kernel runs; it waits for the first kernel's results by itself.
    const int C = a.n_q * (a.Hq / a.Hkv), out_blocks = ceil_div(C * D, 128), row_blocks = weight_out ? ceil_div(a.cap, 4 * WT_THREADS) : 0;
    // About eight blocks an SM: each works out the columns' sums again, so no more than keep the rows' loads in flight.
    const int most = max(8 * ctx->sm_count / max(a.Bz * a.Hkv, 1), 1), blocks = max(min(max(out_blocks, row_blocks), most), min(out_blocks, 8));
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks, a.Hkv, a.Bz);
    cfg.blockDim = dim3(WT_THREADS, 1, 1);
    cfg.dynamicSmemBytes = (size_t)C * sizeof(float2);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (cudaLaunchKernelEx(&cfg, kv4_join_kernel<T, D>, a, (int)COLS, G, (int)AT_WARPS, weight, weight_out) != cudaSuccess) return STR_ERR_CUDA;
    ctx->launches += 1;
    return STR_OK;
}

template <typename T, int D, int GROUP>
int launch_shape(str_ctx *ctx, const str_kv4_shape *s, AttnArgs &a, int G, const float *weight, float *weight_out, cudaStream_t st) {
    const int cols = unit_columns(s, a.n_q * (a.Hq / a.Hkv));
    if constexpr (D / GROUP >= 2)
        if (cols == 4) return launch_attn<T, D, GROUP, 1, 2>(ctx, a, G, weight, weight_out, st);
    return cols <= 8 ? launch_attn<T, D, GROUP, 1, 1>(ctx, a, G, weight, weight_out, st) : launch_attn<T, D, GROUP, 2, 1>(ctx, a, G, weight, weight_out, st);
}

template <typename T>
int launch_type(str_ctx *ctx, const str_kv4_shape *s, AttnArgs &a, int G, const float *weight, float *weight_out, cudaStream_t st) {
    if (s->d == 64) return s->group == 32 ? launch_shape<T, 64, 32>(ctx, s, a, G, weight, weight_out, st) : launch_shape<T, 64, 64>(ctx, s, a, G, weight, weight_out, st);
    if (s->group == 32) return launch_shape<T, 128, 32>(ctx, s, a, G, weight, weight_out, st);
    return s->group == 64 ? launch_shape<T, 128, 64>(ctx, s, a, G, weight, weight_out, st) : launch_shape<T, 128, 128>(ctx, s, a, G, weight, weight_out, st);
}

// CTAs of the first kernel: two per SM, one where 16 query rows take the registers.  The size query has no context: it
// counts for the larger.
constexpr int AT_MAX_GRID = 2 * 148;

}  // namespace kv4_attn

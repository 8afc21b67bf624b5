// Packed sequences: n_seq sequences lie one after the other in a tensor of `rows` rows; start[s] is the first row of sequence s and
// start[n_seq] the first row behind the last one (device int32, n_seq + 1 entries, ascending).  Rows outside are nobody's.
//
// The kernels trust nothing they read there: every start is held to [0, rows], and what follows from it (rows, lengths, indices of
// sequences) stays inside the tensors for any values at all.  Starts outside that range or descending are recorded as the decode
// calls record wrong counts.
#pragma once
#include "kv4.cuh"

__device__ __forceinline__ int packed_start(const int32_t *start, int i, int rows) { return min(max(__ldg(start + i), 0), rows); }

// Sequence that row t lies in: the last one that starts at or before it (empty ones share their start with the next).  -1 before the
// first, n_seq behind the last.  All threads of the block call it; one pass over the starts, one barrier.
__device__ __forceinline__ int packed_sequence_of(const int32_t *start, int n_seq, int t) {
    int at_or_before = 0;
    for (int i0 = 0; i0 <= n_seq; i0 += blockDim.x) {
        const int i = i0 + (int)threadIdx.x;
        at_or_before += __syncthreads_count(i <= n_seq && __ldg(start + i) <= t);
    }
    return at_or_before - 1;
}

// One block looks all starts over and records what is wrong.
__device__ __forceinline__ void packed_check(const int32_t *start, int n_seq, int rows, int *status) {
    for (int i = threadIdx.x; i <= n_seq; i += blockDim.x) {
        const int v = __ldg(start + i);
        if (v < 0 || v > rows || (i > 0 && v < __ldg(start + i - 1))) kv4_report(status);
    }
}

// ---- the order of attention's query blocks ------------------------------------------------------
// A query block is block.d consecutive queries of one sequence; it costs as many key tiles as its last query sees.  CTA number r
// takes the r-th most expensive block of all sequences, so that the long ones start first and the short ones fill the gaps.
// No list is made: the number of blocks that cost `tiles` or more is a sum over the sequences of a closed form, and a binary search over the
// cost, then a prefix sum over the sequences, find block r.  Run by one whole warp.
//
// Starts that descend can name more blocks than an int counts.  A lane's count is held to MOST_BLOCKS, so that the sum over a warp stays an int, grows
// with the cost's bound falling as the search supposes, and an index within a sequence is never negative.  Right calls never get there: with
// rows_q * group * Hkv below 2^31 and blocks of 64 (query, head) pairs or more there are 6.6e7 at most (a group of 33 in blocks of one query).
constexpr int MOST_BLOCKS = (1 << 26) - 1;

struct PackedBlock {
    int seq, first, n;           // sequence, first query within it, queries (0: there is no block r)
    int q0, lq, k0, lk;          // the sequence's rows
};

// Queries a block, and what divides by it: x / d = high half of x * (2^64 / d, rounded up), exact for 32-bit x.
// (A division by a number known at run time only costs some 40 instructions, and the search makes one a step and sequence.)
struct PackedBlockSize {
    int d;
    unsigned long long m;
    explicit PackedBlockSize(int size) : d(size), m(size > 1 ? ~0ULL / (unsigned)size + 1 : 0) {}
    __device__ __forceinline__ int into(int x) const { return d > 1 ? (int)__umul64hi((unsigned long long)(unsigned)x, m) : x; }
};

struct PackedAttnSeq {
    int q0, lq, k0, lk, blocks;
};
__device__ __forceinline__ PackedAttnSeq packed_attn_seq(const int32_t *q_start, const int32_t *k_start, int s, int rows_q, int rows_k, const PackedBlockSize &block) {
    PackedAttnSeq r;
    r.q0 = packed_start(q_start, s, rows_q);
    r.lq = max(packed_start(q_start, s + 1, rows_q) - r.q0, 0);
    r.k0 = packed_start(k_start, s, rows_k);
    r.lk = max(packed_start(k_start, s + 1, rows_k) - r.k0, 0);
    r.blocks = r.lq > 0 ? block.into(r.lq - 1) + 1 : 0;
    return r;
}
// Blocks of the sequence whose last query sees more than (tiles - 1) * key_tile keys; all of them for tiles <= 0.
__device__ __forceinline__ int packed_blocks_of_cost(const PackedAttnSeq &q, const PackedBlockSize &block, int key_tile, int tiles) {
    if (tiles <= 0) return q.blocks;
    const long long below = (long long)(tiles - 1) * key_tile;
    if (q.lk <= below) return 0;
    const long long y = below - q.lk + q.lq;             // the last query of a block has to be number y (< lq) or later
    return y <= 0 ? q.blocks : q.blocks - block.into((int)y);
}
__device__ __forceinline__ PackedBlock packed_block(const int32_t *q_start, const int32_t *k_start, int n_seq, int rows_q, int rows_k, const PackedBlockSize &block,
                                                    int key_tile, int r) {
    const int lane = threadIdx.x & 31;
    // the lane's first sequence stays in registers: most calls have no more than 32
    const PackedAttnSeq own = lane < n_seq ? packed_attn_seq(q_start, k_start, lane, rows_q, rows_k, block) : PackedAttnSeq{};
    auto blocks = [&](int tiles) {
        int n = min(packed_blocks_of_cost(own, block, key_tile, tiles), MOST_BLOCKS);
        for (int s = lane + 32; s < n_seq; s += 32)
            n = min(n + packed_blocks_of_cost(packed_attn_seq(q_start, k_start, s, rows_q, rows_k, block), block, key_tile, tiles), MOST_BLOCKS);
        return (int)__reduce_add_sync(0xffffffffu, (unsigned)n);
    };
    PackedBlock b = {};
    if (r >= blocks(0)) return b;
    int lo = 0, hi = (rows_k + key_tile - 1) / key_tile;  // blocks(lo) > r; no block costs more than hi
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (blocks(mid) > r) lo = mid;
        else hi = mid - 1;
    }
    int left = r - blocks(lo + 1);                        // among the blocks that cost exactly lo, in the order of the sequences
    for (int s0 = 0; s0 < n_seq; s0 += 32) {
        PackedAttnSeq q = {};
        int from = 0, n = 0;
        if (s0 + lane < n_seq) {
            q = s0 == 0 ? own : packed_attn_seq(q_start, k_start, s0 + lane, rows_q, rows_k, block);
            const int more = packed_blocks_of_cost(q, block, key_tile, lo + 1);
            n = packed_blocks_of_cost(q, block, key_tile, lo) - more;
            from = q.blocks - more - n;
            n = min(n, MOST_BLOCKS);
        }
        int upto = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        const unsigned found = __ballot_sync(0xffffffffu, upto > left);
        if (found) {
            const int l = __ffs(found) - 1;
            const int i = from + left - (upto - n);       // meaningful in lane l only
            b.seq = s0 + l;
            b.first = __shfl_sync(0xffffffffu, i, l) * block.d;
            b.q0 = __shfl_sync(0xffffffffu, q.q0, l);
            b.lq = __shfl_sync(0xffffffffu, q.lq, l);
            b.k0 = __shfl_sync(0xffffffffu, q.k0, l);
            b.lk = __shfl_sync(0xffffffffu, q.lk, l);
            b.n = min(block.d, b.lq - b.first);
            return b;
        }
        left -= __shfl_sync(0xffffffffu, upto, 31);
    }
    return b;
}

// The 4-bit key/value cache: packed layout, argument checks and device helpers shared by its kernels.
//
// A row (one token, one key head, keys or values) of d elements is d / 2 bytes of codes and d / group 32-bit words.  The
// word of a group holds (scale bf16) << 16 | (zero bf16); the group's elements stand for zero + scale * code.
// With ng = d / 32, the codes of a row are stored in the order in which the attention kernel's lanes take them:
//   keys    element 32 g + 8 c + j (c < 4, j < 8) is nibble j of the 32-bit word c * ng + g: the lane that holds columns
//           2c, 2c+1, 2c+8, 2c+9 of a matrix fragment finds its words of all 32-element runs side by side;
//   values  element 32 g + 4 r + i (r < 8, i < 4) is nibble i of the 16-bit word r * ng + g: the lane that holds row r of
//           a fragment finds its quarter-words side by side.
#pragma once
#include "common.cuh"

// Makes the context's device current for the launches of one call and puts the caller's back.  Comes before the call's StrProfScope:
// its events are made on, and recorded on a stream of, the current device.
struct StrDeviceScope {
    int prev;
    bool ok;
    explicit StrDeviceScope(const str_ctx *ctx) : prev(-1), ok(true) {
        int cur = 0;
        if (cudaGetDevice(&cur) != cudaSuccess) { ok = false; return; }
        if (cur != ctx->device) {
            ok = cudaSetDevice(ctx->device) == cudaSuccess;
            prev = cur;
        }
    }
    ~StrDeviceScope() { if (prev >= 0) cudaSetDevice(prev); }
};

// STR_OK, or why the shape of a cache is refused.
static inline int kv4_check_shape(const str_kv4_shape *s) {
    if (!s || s->Bz <= 0 || s->cap <= 0 || s->Hkv <= 0 || s->d <= 0 || s->group <= 0) return STR_ERR_INVALID_ARG;
    if ((s->d != 64 && s->d != 128) || (s->group != 32 && s->group != 64 && s->group != 128) || s->group > s->d) return STR_ERR_UNSUPPORTED_SHAPE;
    if (s->cap % 16 != 0 || s->Bz > 65535 || s->Hkv > 65535 || s->cap > (1 << 30)) return STR_ERR_UNSUPPORTED_SHAPE;
    return STR_OK;
}
static inline bool kv4_pointers_ok(const str_kv4_cache *c) {
    if (!c || !c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales) return false;
    return (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes | (uintptr_t)c->k_scales | (uintptr_t)c->v_scales | (uintptr_t)c->pos |
             (uintptr_t)c->weight) & 15) == 0;
}

// Do two buffers share memory?
static inline bool kv4_overlap(const void *a, size_t na, const void *b, size_t nb) {
    return a && b && na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

__device__ __forceinline__ float kv4_scale(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ float kv4_zero(uint32_t w) { return __uint_as_float(w << 16); }

// Eight consecutive elements as they are stored, and widened.
template <typename T> struct Kv4Raw8;
template <> struct Kv4Raw8<__nv_bfloat16> { uint4 u; };
template <> struct Kv4Raw8<float> { float4 a, b; };
__device__ __forceinline__ Kv4Raw8<__nv_bfloat16> kv4_raw8(const __nv_bfloat16 *p) { return {__ldg((const uint4 *)p)}; }
__device__ __forceinline__ Kv4Raw8<float> kv4_raw8(const float *p) { return {__ldg((const float4 *)p), __ldg((const float4 *)p + 1)}; }
__device__ __forceinline__ void kv4_widen8(const Kv4Raw8<__nv_bfloat16> &r, float (&x)[8]) {
    const uint32_t w[4] = {r.u.x, r.u.y, r.u.z, r.u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void kv4_widen8(const Kv4Raw8<float> &r, float (&x)[8]) {
    x[0] = r.a.x; x[1] = r.a.y; x[2] = r.a.z; x[3] = r.a.w;
    x[4] = r.b.x; x[5] = r.b.y; x[6] = r.b.z; x[7] = r.b.w;
}
template <typename T>
__device__ __forceinline__ void kv4_load8(const T *p, float (&x)[8]) { kv4_widen8(kv4_raw8(p), x); }

// A count or row that the caller got wrong: recorded in the second status word, which str_check_status reads too.  (The first
// makes the tensor-core kernels of the context leave at once; a wrong count is no reason for that.)
__device__ __forceinline__ void kv4_report(int *status) { atomicCAS(status + 1, 0, STR_ERR_INVALID_ARG); }

// Row count of a sequence as the kernels use it: what the caller says, held to [0, cap]; a value outside is recorded.
__device__ __forceinline__ int kv4_len(const int32_t *lens, int b, int cap, int *status) {
    const int n = lens[b];
    if (n < 0 || n > cap) {
        if (threadIdx.x == 0) kv4_report(status);
        return n < 0 ? 0 : cap;
    }
    return n;
}

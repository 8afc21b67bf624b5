// str_mamba_conv_packed, str_mamba_conv_step: the Mamba block's pre-scan step with a window of earlier inputs,
//   u_t = bias + sum_j w_j in_{t-W+1+j},   x | B | C = SiLU(u),   dt = softplus(raw + dt_bias),
// where inputs before the sequence's first row come from its window (the last W - 1 inputs of what went before; zeros without one), and
// the last W - 1 inputs go out as the next window.
//
// Bound by memory: every column of x | B | C | dt in once and out once.  Rows travel to shared memory by cp.async, each thread's own four channels, 12 to 16
// rows ahead, since a thread that waits for its loads before it works keeps too little in flight (8 rows in registers: 320 us against 197 us for
// 24576 rows of the 8B-class layer, 5.2 TB/s).  The arithmetic is next: 16 instructions an element, two of them on the special-function unit.
#include "packed.cuh"

#define STR_DTYPE_OK(dt) ((dt) == STR_F32 || (dt) == STR_BF16)

namespace {

constexpr int THREADS = 128;
constexpr int GROUP = 4, GROUPS = 4;                      // rows fetched at a time, and how many such fetches a thread has room for

struct ConvDims {
    int d_inner, gn, H, ch, ld;                           // ch = d_inner + 2 gn channels behind the d_inner columns of the gate
};

// VEC consecutive elements as they are stored.
template <typename T, int VEC> struct alignas(VEC * sizeof(T)) Pack { T v[VEC]; };
template <int VEC, typename T>
__device__ __forceinline__ Pack<T, VEC> load_pack(const T *p) {
    Pack<T, VEC> r;
    if constexpr (VEC * sizeof(T) == 16) *(uint4 *)&r = __ldg((const uint4 *)p);
    else if constexpr (VEC * sizeof(T) == 8) *(uint2 *)&r = __ldg((const uint2 *)p);
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i) r.v[i] = p[i];
    return r;
}
// The same of memory that the kernel writes too (its window, in place): not through the read-only path.
template <int VEC, typename T>
__device__ __forceinline__ Pack<T, VEC> load_pack_written(const T *p) {
    Pack<T, VEC> r;
    if constexpr (VEC * sizeof(T) == 16) *(uint4 *)&r = *(const uint4 *)p;
    else if constexpr (VEC * sizeof(T) == 8) *(uint2 *)&r = *(const uint2 *)p;
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i) r.v[i] = p[i];
    return r;
}
template <int VEC, typename T>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, VEC> &r) {
    if constexpr (VEC * sizeof(T) == 16) *(uint4 *)p = *(const uint4 *)&r;
    else if constexpr (VEC * sizeof(T) == 8) *(uint2 *)p = *(const uint2 *)&r;
    else
#pragma unroll
        for (int i = 0; i < VEC; ++i) p[i] = r.v[i];
}
// Copy to shared memory in the background; single elements (which it does not take) at once.
template <int VEC, typename T>
__device__ __forceinline__ void fetch_pack(Pack<T, VEC> *to, const T *from) {
    if constexpr (VEC * sizeof(T) == 16)
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
    else if constexpr (VEC * sizeof(T) == 8)
        asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
    else *to = load_pack<VEC>(from);
}
template <typename T, int VEC>
__device__ __forceinline__ Pack<T, VEC> zero_pack() {
    Pack<T, VEC> r;
#pragma unroll
    for (int i = 0; i < VEC; ++i) stf(&r.v[i], 0.f);
    return r;
}

// A row's VEC elements in fp32, and the outputs narrowed to the storage type.  Packed fp32 arithmetic (two elements an instruction) where there
// are two.
template <int VEC> struct Row { float f[VEC]; };
template <int VEC, typename T>
__device__ __forceinline__ Row<VEC> widen(const Pack<T, VEC> &p) {
    Row<VEC> r;
    if constexpr (sizeof(T) == 2 && VEC % 2 == 0) {
        const uint32_t *w = (const uint32_t *)&p;
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            r.f[2 * i] = __uint_as_float(w[i] << 16);
            r.f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) r.f[i] = ldf(&p.v[i]);
    }
    return r;
}
// silu_fast of two values, operation for operation.
__device__ __forceinline__ float2 silu_fast2(float2 v) {
    const float2 t = __fmul2_rn(v, make_float2(-1.4426950408889634f, -1.4426950408889634f));
    float2 e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.x) : "f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e.y) : "f"(t.y));
    e = __fadd2_rn(e, make_float2(1.0f, 1.0f));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(e.x));
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(e.y));
    return __fmul2_rn(v, r);
}
template <int VEC>
__device__ __forceinline__ Pack<float, VEC> activate(const Row<VEC> &u, const float *) {
    Pack<float, VEC> o;
#pragma unroll
    for (int i = 0; i < VEC; ++i) o.v[i] = silu_f(u.f[i]);
    return o;
}
template <int VEC>
__device__ __forceinline__ Pack<__nv_bfloat16, VEC> activate(const Row<VEC> &u, const __nv_bfloat16 *) {
    Pack<__nv_bfloat16, VEC> o;
    if constexpr (VEC % 2 == 0) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
            const float2 v = silu_fast2(make_float2(u.f[2 * i], u.f[2 * i + 1]));
            const __nv_bfloat162 w = __floats2bfloat162_rn(v.x, v.y);
            ((uint32_t *)&o)[i] = *reinterpret_cast<const uint32_t *>(&w);
        }
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) o.v[i] = __float2bfloat16_rn(silu_fast(u.f[i]));
    }
    return o;
}

// Where a channel's outputs go: x, B or C, each [rows, width].
template <typename T>
__device__ __forceinline__ T *out_column(const ConvDims &c, int ch0, T *x, T *B, T *C, int &width) {
    if (ch0 < c.d_inner) { width = c.d_inner; return x + ch0; }
    width = c.gn;
    return ch0 < c.d_inner + c.gn ? B + (ch0 - c.d_inner) : C + (ch0 - c.d_inner - c.gn);
}

template <int VEC, int W>
struct Taps {
    float w[W][VEC], bias[VEC];
    __device__ __forceinline__ Taps(const float *conv_w, const float *conv_b, int ch0) {
        if constexpr (W == 4) {
            if (((uintptr_t)conv_w & 15) == 0) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    const float4 t = __ldg((const float4 *)conv_w + ch0 + i);
                    w[0][i] = t.x, w[1][i] = t.y, w[2][i] = t.z, w[3][i] = t.w;
                }
            } else {
                load(conv_w, ch0);
            }
        } else {
            load(conv_w, ch0);
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) bias[i] = __ldg(conv_b + ch0 + i);
    }
    __device__ __forceinline__ void load(const float *conv_w, int ch0) {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = __ldg(conv_w + (size_t)(ch0 + i) * W + j);
    }
    // The sum over a row's taps, from the W - 1 rows before it (oldest first) and its own; moves the history on.
    __device__ __forceinline__ Row<VEC> apply(Row<VEC> (&hist)[W - 1], const Row<VEC> &cur) const {
        Row<VEC> u;
        if constexpr (VEC % 2 == 0) {
#pragma unroll
            for (int i = 0; i < VEC; i += 2) {
                float2 a = make_float2(bias[i], bias[i + 1]);
#pragma unroll
                for (int j = 0; j < W - 1; ++j) a = __ffma2_rn(make_float2(w[j][i], w[j][i + 1]), make_float2(hist[j].f[i], hist[j].f[i + 1]), a);
                a = __ffma2_rn(make_float2(w[W - 1][i], w[W - 1][i + 1]), make_float2(cur.f[i], cur.f[i + 1]), a);
                u.f[i] = a.x, u.f[i + 1] = a.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                float a = bias[i];
#pragma unroll
                for (int j = 0; j < W - 1; ++j) a = fmaf(w[j][i], hist[j].f[i], a);
                u.f[i] = fmaf(w[W - 1][i], cur.f[i], a);
            }
        }
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) hist[j] = hist[j + 1];
        hist[W - 2] = cur;
        return u;
    }
};

// Blocks (i, j), j fastest: rows [tile i, tile i + tile) of the packed tensor, channels of column block j; the last j takes the dt columns.  Behind the row
// tiles one block i per sequence copies its window, column block by column block.
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(THREADS)
conv_packed_kernel(ConvDims c, int n_seq, int rows, int tile, int tiles, int cols, const T *__restrict__ zx, const float *__restrict__ conv_w,
                   const float *__restrict__ conv_b, const float *__restrict__ dt_bias, const int32_t *__restrict__ start,
                   const T *__restrict__ window, T *__restrict__ x, T *__restrict__ B, T *__restrict__ C, float *__restrict__ dt,
                   T *__restrict__ window_out, int *status) {
    const int bi = blockIdx.x / cols, bj = blockIdx.x % cols;
    const bool dt_block = bj == cols - 1;
    const int ch0 = (bj * THREADS + threadIdx.x) * VEC;
    const T *src = zx + c.d_inner + ch0;                  // + row * ld
    if (bi >= tiles) {
        const int s = bi - tiles;
        if (dt_block) {
            if (s == 0) packed_check(start, n_seq, rows, status);
            return;
        }
        if (!window_out || ch0 >= c.ch) return;
        const int s0 = packed_start(start, s, rows), T_s = max(packed_start(start, s + 1, rows) - s0, 0);
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int r = T_s - (W - 1) + j;              // row of the sequence, or (negative) of the window behind it
            Pack<T, VEC> v = zero_pack<T, VEC>();
            if (r >= 0) v = load_pack<VEC>(src + (size_t)(s0 + r) * c.ld);
            else if (window) v = load_pack<VEC>(window + ((size_t)s * (W - 1) + r + W - 1) * c.ch + ch0);
            store_pack<VEC>(window_out + ((size_t)s * (W - 1) + j) * c.ch + ch0, v);
        }
        return;
    }
    const int t0 = bi * tile, t1 = min(rows, t0 + tile);
    int s = packed_sequence_of(start, n_seq, t0);
    if (dt_block) {
        for (int e = threadIdx.x; e < (t1 - t0) * c.H; e += THREADS) {
            const int t = t0 + e / c.H, h = e % c.H;
            int st = s;
            while (st < n_seq && __ldg(start + st + 1) <= t) ++st;
            if (st >= 0 && st < n_seq) dt[(size_t)t * c.H + h] = softplus_f(ldf(zx + (size_t)t * c.ld + c.d_inner + c.ch + h) + dt_bias[h]);
        }
        return;
    }
    if (ch0 >= c.ch) return;
    __shared__ Pack<T, VEC> ring[GROUPS * GROUP * THREADS];
    const Taps<VEC, W> taps(conv_w, conv_b, ch0);
    int width;
    T *dst = out_column(c, ch0, x, B, C, width);
    Row<VEC> hist[W - 1];
    auto history = [&](int t) {                           // the W - 1 inputs before row t of sequence s
        const int s0 = s >= 0 && s < n_seq ? min(packed_start(start, s, rows), t) : t;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int r = t - (W - 1) + j;
            Pack<T, VEC> v = zero_pack<T, VEC>();
            if (s >= 0 && s < n_seq) {
                if (r >= s0) v = load_pack<VEC>(src + (size_t)r * c.ld);
                else if (window) v = load_pack<VEC>(window + ((size_t)s * (W - 1) + (r - s0 + W - 1)) * c.ch + ch0);
            }
            hist[j] = widen(v);
        }
    };
    // One sequence's rows after another, so that the loop over them has no edges in it.
#pragma unroll 1
    for (int t = t0; t < t1;) {
        while (s < n_seq && __ldg(start + s + 1) <= t) ++s;
        if (s >= n_seq) break;
        const int end = min(t1, __ldg(start + s + 1));
        if (s >= 0) {
            history(t);
            // Rows on their way to shared memory while earlier ones are worked on; a thread reads back what it fetched itself.
            auto fetch = [&](int g) {
#pragma unroll
                for (int u = 0; u < GROUP; ++u) {
                    const int r = t + g * GROUP + u;
                    if (r < end) fetch_pack<VEC>(&ring[((g % GROUPS) * GROUP + u) * THREADS + threadIdx.x], src + (size_t)r * c.ld);
                }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
#pragma unroll
            for (int g = 0; g < GROUPS - 1; ++g) fetch(g);
#pragma unroll 1
            for (int g = 0; t + g * GROUP < end; ++g) {
                asm volatile("cp.async.wait_group %0;" ::"n"(GROUPS - 2) : "memory");
                Pack<T, VEC> raw[GROUP];
#pragma unroll
                for (int u = 0; u < GROUP; ++u) raw[u] = ring[((g % GROUPS) * GROUP + u) * THREADS + threadIdx.x];
                fetch(g + GROUPS - 1);
#pragma unroll
                for (int u = 0; u < GROUP; ++u) {
                    const int r = t + g * GROUP + u;
                    const Pack<T, VEC> o = activate(taps.apply(hist, widen(raw[u])), (const T *)nullptr);
                    if (r < end) store_pack<VEC>(dst + (size_t)r * width, o);
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");          // empty fetches; the room is used anew
        }
        t = end;
    }
}

// A few tokens per sequence: a thread takes VEC channels of one sequence, window in registers.  The window may be written where it was read.
template <typename T, int VEC, int W>
__global__ void __launch_bounds__(THREADS)
conv_step_kernel(ConvDims c, int T_new, const T *__restrict__ zx, const float *__restrict__ conv_w, const float *__restrict__ conv_b,
                 const float *__restrict__ dt_bias, const T *window, T *__restrict__ x, T *__restrict__ B, T *__restrict__ C,
                 float *__restrict__ dt, T *window_out) {
    const int b = blockIdx.x;
    const size_t row0 = (size_t)b * T_new;
    if (blockIdx.y == gridDim.y - 1) {
        for (int e = threadIdx.x; e < T_new * c.H; e += THREADS) {
            const int t = e / c.H, h = e % c.H;
            dt[(row0 + t) * c.H + h] = softplus_f(ldf(zx + (row0 + t) * c.ld + c.d_inner + c.ch + h) + dt_bias[h]);
        }
        return;
    }
    const int ch0 = (blockIdx.y * THREADS + threadIdx.x) * VEC;
    if (ch0 >= c.ch) return;
    Pack<T, VEC> before[W - 1];                           // the window moves by whole elements: kept as they are stored
    Row<VEC> hist[W - 1];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) before[j] = load_pack_written<VEC>(window + ((size_t)b * (W - 1) + j) * c.ch + ch0);
    const Taps<VEC, W> taps(conv_w, conv_b, ch0);
#pragma unroll
    for (int j = 0; j < W - 1; ++j) hist[j] = widen(before[j]);
    int width;
    T *dst = out_column(c, ch0, x, B, C, width);
    for (int t = 0; t < T_new; ++t) {
        const Pack<T, VEC> cur = load_pack<VEC>(zx + (row0 + t) * c.ld + c.d_inner + ch0);
        store_pack<VEC>(dst + (row0 + t) * width, activate(taps.apply(hist, widen(cur)), (const T *)nullptr));
#pragma unroll
        for (int j = 0; j + 1 < W - 1; ++j) before[j] = before[j + 1];
        before[W - 2] = cur;
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_pack<VEC>(window_out + ((size_t)b * (W - 1) + j) * c.ch + ch0, before[j]);
}

// What both entry points are given.
struct ConvCall {
    ConvDims c;
    int n_seq, rows;                                      // conv_step: sequences and tokens per sequence
    const void *zx, *window;
    const float *conv_w, *conv_b, *dt_bias;
    const int32_t *start;
    void *x, *B, *C, *window_out;
    float *dt;
    int *status;
    int sms;
};

template <typename T, int VEC, int W>
void launch(const ConvCall &k, bool step, cudaStream_t st) {
    const int cols = ceil_div(ceil_div(k.c.ch, VEC), THREADS) + 1;
    if (step) {
        conv_step_kernel<T, VEC, W><<<dim3(k.n_seq, cols), THREADS, 0, st>>>(k.c, k.rows, (const T *)k.zx, k.conv_w, k.conv_b, k.dt_bias,
                                                                             (const T *)k.window, (T *)k.x, (T *)k.B, (T *)k.C, k.dt, (T *)k.window_out);
    } else {
        // Rows per block: a block's first rows wait for its taps and its history, and few large blocks leave SMs idle at the end (24576 rows of the
        // 8B-class layer: 64 rows 211 us, 32 rows 197, 16 rows 213); fewer where 32 would leave SMs without work.
        int tile = 32;
        while (tile > 8 && (long long)ceil_div(k.rows, tile) * cols < 8LL * k.sms) tile /= 2;
        const int tiles = ceil_div(k.rows, tile);
        conv_packed_kernel<T, VEC, W><<<(tiles + k.n_seq) * cols, THREADS, 0, st>>>(
            k.c, k.n_seq, k.rows, tile, tiles, cols, (const T *)k.zx, k.conv_w, k.conv_b, k.dt_bias, k.start, (const T *)k.window, (T *)k.x, (T *)k.B, (T *)k.C, k.dt,
            (T *)k.window_out, k.status);
    }
}
template <typename T, int VEC>
void dispatch_width(const ConvCall &k, int W, bool step, cudaStream_t st) {
    if (W == 2) launch<T, VEC, 2>(k, step, st);
    else if (W == 3) launch<T, VEC, 3>(k, step, st);
    else launch<T, VEC, 4>(k, step, st);
}
// Four channels a thread (16 bytes of fp32, 8 of bf16) where rows, columns and pointers allow it, else one channel.
template <typename T>
void dispatch_vec(const ConvCall &k, int W, bool step, cudaStream_t st) {
    constexpr int VEC = 4;
    const uintptr_t at = (uintptr_t)k.zx | (uintptr_t)k.window | (uintptr_t)k.window_out | (uintptr_t)k.x | (uintptr_t)k.B | (uintptr_t)k.C;
    if (k.c.d_inner % VEC == 0 && k.c.gn % VEC == 0 && k.c.ld % VEC == 0 && at % (VEC * sizeof(T)) == 0) dispatch_width<T, VEC>(k, W, step, st);
    else dispatch_width<T, 1>(k, W, step, st);
}

// Blocks of columns, the dt columns' included, at one channel a thread (vector accesses need fewer).
long long column_blocks(const ConvDims &c) { return (c.ch + THREADS - 1) / THREADS + 1; }

int check_dims(int dtype, int H, int p, int n, int G, int W, ConvDims *c) {
    if (H <= 0 || p <= 0 || n <= 0 || G <= 0 || H % G != 0 || W <= 0 || !STR_DTYPE_OK(dtype)) return STR_ERR_INVALID_ARG;
    const long long d_inner = (long long)H * p, gn = (long long)G * n, ld = 2 * d_inner + 2 * gn + H;
    if (W < 2 || W > 4 || d_inner > (1 << 24) || gn > (1 << 24)) return STR_ERR_UNSUPPORTED_SHAPE;
    *c = {(int)d_inner, (int)gn, H, (int)(d_inner + 2 * gn), (int)ld};
    return STR_OK;
}

// Does an output share memory with what other blocks may still have to read?  (The step's window in place, whose elements are read and written by one
// thread, is its caller's to allow.)
bool outputs_overlap(const ConvDims &c, size_t es, int n_seq, size_t rows, int W, const void *zx, const float *conv_w, const float *conv_b, const float *dt_bias,
                     const int32_t *start, const void *window, const void *x, const void *B, const void *C, const void *dt, const void *window_out, bool in_place) {
    const size_t wb = (size_t)n_seq * (W - 1) * c.ch * es;
    const struct { const void *at; size_t bytes; } in[] = {{zx, rows * c.ld * es}, {window, wb}, {conv_w, (size_t)c.ch * W * sizeof(float)}, {conv_b, c.ch * sizeof(float)},
                                                           {dt_bias, c.H * sizeof(float)}, {start, ((size_t)n_seq + 1) * sizeof(int32_t)}},
        out[] = {{x, rows * c.d_inner * es}, {B, rows * c.gn * es}, {C, rows * c.gn * es}, {dt, rows * c.H * sizeof(float)}, {window_out, wb}};
    for (const auto &i : in)
        for (const auto &o : out)
            if (kv4_overlap(i.at, i.bytes, o.at, o.bytes) && !(in_place && &i == in + 1 && &o == out + 4)) return true;
    return false;
}

}  // namespace

extern "C" int str_mamba_conv_packed(str_ctx *ctx, int dtype, int n_seq, int rows, int H, int p, int n, int G, int W, const void *zxbcdt,
                                     const float *conv_w, const float *conv_b, const float *dt_bias, const int32_t *seq_start, const void *window,
                                     void *x_out, void *B_out, void *C_out, float *dt_out, void *window_out, void *stream) {
    ConvDims c;
    if (!ctx || !conv_w || !conv_b || !dt_bias || !seq_start || n_seq <= 0 || rows < 0) return STR_ERR_INVALID_ARG;
    if (rows > 0 && (!zxbcdt || !x_out || !B_out || !C_out || !dt_out)) return STR_ERR_INVALID_ARG;
    const int rc = check_dims(dtype, H, p, n, G, W, &c);
    if (rc != STR_OK) return rc;
    if (n_seq > 65535 || rows > (1 << 30) || (rows / 8 + 1LL + n_seq) * column_blocks(c) > INT32_MAX) return STR_ERR_UNSUPPORTED_SHAPE;
    if (outputs_overlap(c, dtype_size(dtype), n_seq, rows, W, zxbcdt, conv_w, conv_b, dt_bias, seq_start, window, x_out, B_out, C_out, dt_out, window_out, false))
        return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    const ConvCall k = {c, n_seq, rows, zxbcdt, window, conv_w, conv_b, dt_bias, seq_start, x_out, B_out, C_out, window_out, dt_out, ctx->status_dev, ctx->sm_count};
    if (dtype == STR_BF16) dispatch_vec<__nv_bfloat16>(k, W, false, (cudaStream_t)stream);
    else dispatch_vec<float>(k, W, false, (cudaStream_t)stream);
    return str_launch_ok(ctx);
}

extern "C" int str_mamba_conv_step(str_ctx *ctx, int dtype, int Bz, int T, int H, int p, int n, int G, int W, const void *zxbcdt,
                                   const float *conv_w, const float *conv_b, const float *dt_bias, const void *window, void *x_out, void *B_out,
                                   void *C_out, float *dt_out, void *window_out, void *stream) {
    ConvDims c;
    if (!ctx || !zxbcdt || !conv_w || !conv_b || !dt_bias || !window || !x_out || !B_out || !C_out || !dt_out || !window_out || Bz <= 0 || T <= 0)
        return STR_ERR_INVALID_ARG;
    const int rc = check_dims(dtype, H, p, n, G, W, &c);
    if (rc != STR_OK) return rc;
    if ((long long)Bz * T > (1 << 30) || (long long)T * H > (1 << 30) || column_blocks(c) > 65535) return STR_ERR_UNSUPPORTED_SHAPE;
    if (outputs_overlap(c, dtype_size(dtype), Bz, (size_t)Bz * T, W, zxbcdt, conv_w, conv_b, dt_bias, nullptr, window, x_out, B_out, C_out, dt_out, window_out,
                        window == window_out))
        return STR_ERR_INVALID_ARG;
    StrDeviceScope dev(ctx);
    if (!dev.ok) return STR_ERR_CUDA;
    StrProfScope prof_scope(ctx, STR_CAT_ELEMENTWISE, stream);
    const ConvCall k = {c, Bz, T, zxbcdt, window, conv_w, conv_b, dt_bias, nullptr, x_out, B_out, C_out, window_out, dt_out, ctx->status_dev, ctx->sm_count};
    if (dtype == STR_BF16) dispatch_vec<__nv_bfloat16>(k, W, true, (cudaStream_t)stream);
    else dispatch_vec<float>(k, W, true, (cudaStream_t)stream);
    return str_launch_ok(ctx);
}

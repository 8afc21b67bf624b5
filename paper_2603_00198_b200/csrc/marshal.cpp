// _marshal: argument marshalling of the decode calls and of those on packed sequences for the Python binding, which are made once per layer and token
// or turn: checks of the
// tensors (type, device, shape, contiguity), outputs and workspace from torch's stream-ordered pool, the current stream of the
// context's device, and the call of the C entry point.  No arithmetic.  Host time of one call, launches included: append 4.6 us,
// read 5.1, attention 7.9 (two launches), eviction 7.4 (two), step 4.2; 0.2 of it looks at the tensors of a cache.  Through ctypes it was
// 1.6 to 2.2 times as much.
//
// The entry points are handed over by address (setup), so that the module needs no link to libstr.so.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include <initializer_list>
#include <sstream>
#include <string>

#include "str.h"

namespace {

decltype(&str_kv4_append) f_append;
decltype(&str_kv4_read) f_read;
decltype(&str_kv4_attn_workspace_size) f_attn_ws;
decltype(&str_kv4_attn) f_attn;
decltype(&str_kv4_evict_workspace_size) f_evict_ws;
decltype(&str_kv4_evict) f_evict;
decltype(&str_mamba2_step) f_step;
decltype(&str_rope_split_ex) f_rope;                 // null until setup_packed() was called, as the ones below
decltype(&str_mamba_conv_packed) f_conv;
decltype(&str_mamba_conv_step) f_conv_step;
decltype(&str_mamba2_prefill_packed_workspace_size) f_scan_ws;
decltype(&str_mamba2_prefill_packed) f_scan;
decltype(&str_attn_prefill_packed_workspace_size) f_attn_packed_ws;
decltype(&str_attn_prefill_packed) f_attn_packed;
PyObject *on_error;      // binding._check(code, name): raises
PyObject *out_of_memory; // torch.OutOfMemoryError

struct Refused {};       // a Python exception has been set

typedef std::initializer_list<int64_t> Shape;

std::string text(at::IntArrayRef s) {
    std::ostringstream o;
    o << "(";
    for (size_t i = 0; i < s.size(); ++i) o << (i ? ", " : "") << s[i];
    o << ")";
    return o.str();
}

const at::Tensor &tensor(PyObject *obj, const char *what) {
    if (!THPVariable_Check(obj)) {
        PyErr_Format(PyExc_TypeError, "%s: expected a tensor, got %s", what, Py_TYPE(obj)->tp_name);
        throw Refused();
    }
    return THPVariable_Unpack(obj);
}

// Device address of an argument, after the checks that the C side cannot make.
void *arg(const at::Tensor &t, int device, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
    if (t.scalar_type() != dtype) {
        PyErr_Format(PyExc_TypeError, "%s: expected %s, got %s", what, c10::toString(dtype), c10::toString(t.scalar_type()));
        throw Refused();
    }
    if (!t.is_cuda() || t.get_device() != device) {
        PyErr_Format(PyExc_ValueError, "%s: expected a tensor on cuda:%d, got %s", what, device, t.device().str().c_str());
        throw Refused();
    }
    if (t.sizes() != shape) {
        PyErr_Format(PyExc_ValueError, "%s: expected shape %s, got %s", what, text(shape).c_str(), text(t.sizes()).c_str());
        throw Refused();
    }
    if (!t.is_contiguous()) {
        PyErr_Format(PyExc_ValueError, "%s: tensors must be contiguous", what);
        throw Refused();
    }
    return t.data_ptr();
}
void *arg(PyObject *obj, int device, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
    return arg(tensor(obj, what), device, shape, dtype, what);
}
void *optional(PyObject *obj, int device, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
    return obj == Py_None ? nullptr : arg(obj, device, shape, dtype, what);
}

int type_code(at::ScalarType t) {
    if (t == at::kBFloat16) return STR_BF16;
    if (t == at::kFloat) return STR_F32;
    PyErr_Format(PyExc_TypeError, "unsupported dtype %s", c10::toString(t));
    throw Refused();
}

at::Tensor empty(at::IntArrayRef shape, at::ScalarType dtype, int device) {
    return at::empty(shape, at::TensorOptions().dtype(dtype).device(at::kCUDA, device));
}

// Several small outputs of one call in one allocation, 256 bytes apart: an allocation costs 0.6 us, as much as the rest of a small call's marshalling.
// They share a storage then, as the slices of a tensor do.  Beyond SHARED bytes together (kernels of 5 us and more) each has its own, so
// that keeping one does not keep the others' memory.
struct Parts {
    static constexpr int64_t SHARED = 2 << 20;
    struct Part {
        at::IntArrayRef shape;
        at::ScalarType dtype;
    };
    static int64_t bytes(const Part &p) {
        int64_t n = (int64_t)c10::elementSize(p.dtype);
        for (const int64_t v : p.shape) n *= v;
        return (n + 255) / 256 * 256;
    }
    // Fills `out` with as many tensors as there are parts.
    static void make(std::initializer_list<Part> parts, int device, at::Tensor *out) {
        int64_t total = 0, at = 0;
        for (const Part &p : parts) total += bytes(p);
        if (total > SHARED) {
            for (const Part &p : parts) *out++ = empty(p.shape, p.dtype, device);
            return;
        }
        const at::Tensor base = empty({total}, at::kByte, device);
        for (const Part &p : parts) {
            *out = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(base.storage()), base.key_set(), c10::scalarTypeToTypeMeta(p.dtype));
            out->unsafeGetTensorImpl()->set_sizes_contiguous(p.shape);
            out->unsafeGetTensorImpl()->set_storage_offset(at / (int64_t)c10::elementSize(p.dtype));
            at += bytes(p);
            ++out;
        }
    }
};

int64_t integer(PyObject *obj, int64_t lo, int64_t hi, const char *what) {
    const long long v = PyLong_AsLongLong(obj);
    if (v == -1 && PyErr_Occurred()) throw Refused();
    if (v < lo || v > hi) {
        PyErr_Format(PyExc_ValueError, "%s: %lld is out of range", what, v);
        throw Refused();
    }
    return v;
}
template <typename T>
T *address(PyObject *obj) {
    void *p = PyLong_AsVoidPtr(obj);
    if (!p && PyErr_Occurred()) throw Refused();
    return (T *)p;
}
void *stream_of(int device) { return c10::cuda::getCurrentCUDAStream(device).stream(); }

// The first arguments of every call: the context's handle and device.
struct Ctx {
    str_ctx *h;
    int device;
    explicit Ctx(PyObject *const *a) : h(address<str_ctx>(a[0])), device((int)integer(a[1], 0, 1 << 20, "device")) {}
};

// Allocation and the call run without the interpreter's lock, as torch's own calls do: the allocator and a full launch queue may wait.
struct Unlocked {
    PyThreadState *state = PyEval_SaveThread();
    Unlocked() = default;
    Unlocked(const Unlocked &) = delete;
    ~Unlocked() { PyEval_RestoreThread(state); }
};

void check(int code, const char *name) {
    if (code == STR_OK) return;
    PyObject *r = PyObject_CallFunction(on_error, "is", code, name);
    if (r) {             // it raises; if it did not, say so here
        Py_DECREF(r);
        PyErr_Format(PyExc_RuntimeError, "%s failed (%d)", name, code);
    }
    throw Refused();
}

void dims(const at::Tensor &t, int n, const char *what) {
    if (t.dim() == n) return;
    PyErr_Format(PyExc_ValueError, "%s: expected %d dimensions, got shape %s", what, n, text(t.sizes()).c_str());
    throw Refused();
}

// cache(ptrs, shape, device, k_codes, v_codes, k_scales, v_scales, pos, weight): checks the tensors that a cache's attributes name
// now and writes their addresses to `ptrs`.  Asked for before every call, as the attributes may be given other tensors, and
// tensors other memory, between two of them.
PyObject *cache(PyObject *const *a) {
    str_kv4_cache *p = address<str_kv4_cache>(a[0]);
    const str_kv4_shape *s = address<str_kv4_shape>(a[1]);
    const int device = (int)integer(a[2], 0, 1 << 20, "device");
    const Shape codes = {s->Bz, s->Hkv, s->cap, s->d / 2}, words = {s->Bz, s->Hkv, s->cap, s->d / s->group};
    str_kv4_cache c;
    c.k_codes = arg(a[3], device, codes, at::kByte, "Kv4Cache.k_codes");
    c.v_codes = arg(a[4], device, codes, at::kByte, "Kv4Cache.v_codes");
    c.k_scales = arg(a[5], device, words, at::kInt, "Kv4Cache.k_scales");
    c.v_scales = arg(a[6], device, words, at::kInt, "Kv4Cache.v_scales");
    c.pos = (int32_t *)optional(a[7], device, {s->Bz, s->cap}, at::kInt, "Kv4Cache.pos");
    c.weight = (float *)optional(a[8], device, {s->Bz, s->Hkv, s->cap}, at::kFloat, "Kv4Cache.weight");
    *p = c;
    Py_RETURN_NONE;
}

// append(handle, device, shape, cache, k, v, row_start, positions, n_new)
PyObject *append(PyObject *const *a) {
    const Ctx c(a);
    const str_kv4_shape *s = address<str_kv4_shape>(a[2]);
    const at::Tensor &k = tensor(a[4], "k");
    dims(k, 4, "k");
    const int64_t T = k.size(1);
    const Shape rows = {s->Bz, T, s->Hkv, s->d};
    const at::ScalarType dt = k.scalar_type();
    const int code = type_code(dt);
    void *pk = arg(k, c.device, rows, dt, "k"), *pv = arg(a[5], c.device, rows, dt, "v");
    void *start = arg(a[6], c.device, {s->Bz}, at::kInt, "row_start"), *pos = optional(a[7], c.device, {s->Bz, T}, at::kInt, "positions");
    void *n_new = optional(a[8], c.device, {s->Bz}, at::kInt, "n_new");
    const str_kv4_cache cache = *address<str_kv4_cache>(a[3]);      // as it is now: another thread may refill it once the lock is free
    int rc;
    {
        Unlocked free;
        rc = f_append(c.h, s, code, (int)T, pk, pv, (const int32_t *)pos, (const int32_t *)start, (const int32_t *)n_new, &cache, stream_of(c.device));
    }
    check(rc, "str_kv4_append");
    Py_RETURN_NONE;
}

// read(handle, device, shape, cache, row_start, T, dtype, n_rows) -> (k, v)
PyObject *read(PyObject *const *a) {
    const Ctx c(a);
    const str_kv4_shape *s = address<str_kv4_shape>(a[2]);
    const int64_t T = integer(a[5], 0, INT32_MAX, "T");
    if (!THPDtype_Check(a[6])) {
        PyErr_SetString(PyExc_TypeError, "dtype: expected a torch.dtype");
        throw Refused();
    }
    const at::ScalarType dt = ((THPDtype *)a[6])->scalar_type;
    const int code = type_code(dt);
    void *start = arg(a[4], c.device, {s->Bz}, at::kInt, "row_start"), *n_rows = optional(a[7], c.device, {s->Bz}, at::kInt, "n_rows");
    const str_kv4_cache cache = *address<str_kv4_cache>(a[3]);      // as it is now: another thread may refill it once the lock is free
    at::Tensor k, v;
    int rc;
    {
        Unlocked free;
        k = empty({s->Bz, T, s->Hkv, s->d}, dt, c.device);
        v = empty({s->Bz, T, s->Hkv, s->d}, dt, c.device);
        rc = f_read(c.h, s, code, (int)T, (const int32_t *)start, (const int32_t *)n_rows, &cache, k.data_ptr(), v.data_ptr(), stream_of(c.device));
    }
    check(rc, "str_kv4_read");
    return Py_BuildValue("NN", THPVariable_Wrap(k), THPVariable_Wrap(v));
}

// attn(handle, device, shape, cache, q, lens, softmax_scale, weight_out) -> o
PyObject *attn(PyObject *const *a) {
    const Ctx c(a);
    const str_kv4_shape *s = address<str_kv4_shape>(a[2]);
    const at::Tensor &q = tensor(a[4], "q");
    dims(q, 4, "q");
    const int64_t n_q = q.size(1), Hq = q.size(2);
    const int code = type_code(q.scalar_type());
    if (n_q > INT32_MAX || Hq > INT32_MAX) check(STR_ERR_UNSUPPORTED_SHAPE, "str_kv4_attn");
    void *pq = arg(q, c.device, {s->Bz, n_q, Hq, s->d}, q.scalar_type(), "q"), *lens = arg(a[5], c.device, {s->Bz}, at::kInt, "lens");
    const double scale = PyFloat_AsDouble(a[6]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    void *weight = optional(a[7], c.device, {s->Bz, s->Hkv, s->cap}, at::kFloat, "weight_out");
    const str_kv4_cache cache = *address<str_kv4_cache>(a[3]);      // as it is now: another thread may refill it once the lock is free
    at::Tensor o, ws;
    int rc;
    {
        Unlocked free;
        const size_t need = f_attn_ws(s, (int)Hq, (int)n_q, weight != nullptr);
        o = empty({s->Bz, n_q, Hq, s->d}, code == STR_BF16 ? at::kBFloat16 : at::kFloat, c.device);
        ws = empty({(int64_t)need}, at::kByte, c.device);
        rc = f_attn(c.h, s, code, (int)Hq, (int)n_q, pq, &cache, (const int32_t *)lens, (float)scale, o.data_ptr(), (float *)weight, ws.data_ptr(),
                    need, stream_of(c.device));
    }
    check(rc, "str_kv4_attn");
    return THPVariable_Wrap(o);
}

// evict(handle, device, shape, cache, lens, keep, n_recent, n_evictable, cap_out, out) -> (lens_out, kept)
PyObject *evict(PyObject *const *a) {
    const Ctx c(a);
    const str_kv4_shape *s = address<str_kv4_shape>(a[2]);
    const int64_t keep = integer(a[5], INT32_MIN, INT32_MAX, "keep"), recent = integer(a[6], INT32_MIN, INT32_MAX, "n_recent");
    void *lens = arg(a[4], c.device, {s->Bz}, at::kInt, "lens"), *evictable = optional(a[7], c.device, {s->Bz}, at::kInt, "n_evictable");
    const int64_t cap_out = integer(a[8], 0, INT32_MAX, "cap_out");
    const str_kv4_cache cache = *address<str_kv4_cache>(a[3]), out = *address<str_kv4_cache>(a[9]);
    at::Tensor n, kept, ws;
    int rc;
    {
        Unlocked free;
        const size_t need = f_evict_ws(s, (int)keep);
        n = empty({s->Bz}, at::kInt, c.device);
        kept = empty({s->Bz, keep > 0 && keep <= s->cap ? keep : 0}, at::kInt, c.device);         // more than cap rows are refused below
        if (need) ws = empty({(int64_t)need}, at::kByte, c.device);
        rc = f_evict(c.h, s, &cache, (const int32_t *)lens, (int)keep, (int)recent, (const int32_t *)evictable, (int)cap_out, &out,
                     (int32_t *)n.data_ptr(), (int32_t *)kept.data_ptr(), need ? ws.data_ptr() : nullptr, need, stream_of(c.device));
    }
    check(rc, "str_kv4_evict");
    return Py_BuildValue("NN", THPVariable_Wrap(n), THPVariable_Wrap(kept));
}

// step(handle, device, x, dt, A, B, C, state, D, state_out) -> y
PyObject *step(PyObject *const *a) {
    const Ctx c(a);
    const at::Tensor &x = tensor(a[2], "x"), &B = tensor(a[5], "B");
    dims(x, 4, "x");
    dims(B, 4, "B");
    const int64_t Bz = x.size(0), T = x.size(1), H = x.size(2), p = x.size(3), G = B.size(2), n = B.size(3);
    for (const int64_t v : {Bz, T, H, p, G, n})
        if (v > INT32_MAX) check(STR_ERR_UNSUPPORTED_SHAPE, "str_mamba2_step");
    const at::ScalarType dt = x.scalar_type();
    const str_ssd_shape s = {(int)Bz, (int)T, (int)H, (int)p, (int)n, (int)G, 0, type_code(dt)};
    void *px = arg(x, c.device, {Bz, T, H, p}, dt, "x"), *pdt = arg(a[3], c.device, {Bz, T, H}, at::kFloat, "dt");
    void *pA = arg(a[4], c.device, {H}, at::kFloat, "A"), *pB = arg(B, c.device, {Bz, T, G, n}, dt, "B"), *pC = arg(a[6], c.device, {Bz, T, G, n}, dt, "C");
    void *state = arg(a[7], c.device, {Bz, H, p, n}, at::kFloat, "state"), *D = optional(a[8], c.device, {H}, at::kFloat, "D");
    void *out = arg(a[9], c.device, {Bz, H, p, n}, at::kFloat, "state_out");
    at::Tensor y;
    int rc;
    {
        Unlocked free;
        y = empty({Bz, T, H, p}, dt, c.device);
        rc = f_step(c.h, &s, px, (const float *)pdt, (const float *)pA, pB, pC, (const float *)D, (const float *)state, y.data_ptr(), (float *)out,
                    stream_of(c.device));
    }
    check(rc, "str_mamba2_step");
    return THPVariable_Wrap(y);
}

int int32(int64_t v, const char *name) {
    if (v > INT32_MAX) check(STR_ERR_UNSUPPORTED_SHAPE, name);
    return (int)v;
}
// Sequences that a tensor of starts [n_seq + 1] describes.
int64_t sequences(const at::Tensor &start, const char *what) {
    dims(start, 1, what);
    if (start.size(0) < 2) {
        PyErr_Format(PyExc_ValueError, "%s: expected n_seq + 1 starts, got %lld", what, (long long)start.size(0));
        throw Refused();
    }
    return start.size(0) - 1;
}
// An output: the caller's tensor (checked) or, for None, a new one.
struct Out {
    at::Tensor t;
    void *p = nullptr;
    bool given = false;
    Out(PyObject *obj, int device, at::IntArrayRef shape, at::ScalarType dtype, const char *what) {
        if (obj == Py_None) return;
        t = tensor(obj, what);
        p = arg(t, device, shape, dtype, what);
        given = true;
    }
    void make(int device, at::IntArrayRef shape, at::ScalarType dtype) {
        if (given) return;
        t = empty(shape, dtype, device);
        p = t.data_ptr();
    }
};

// rope(handle, device, desc, qkv, positions, Hq, Hkv, d) -> (q, k, v)
PyObject *rope(PyObject *const *a) {
    const Ctx c(a);
    const str_rope_desc *desc = address<str_rope_desc>(a[2]);
    const at::Tensor &qkv = tensor(a[3], "qkv");
    dims(qkv, 2, "qkv");
    const int64_t Hq = integer(a[5], 1, 1 << 20, "Hq"), Hkv = integer(a[6], 1, 1 << 20, "Hkv"), d = integer(a[7], 1, 1 << 20, "d");
    const int rows = int32(qkv.size(0), "str_rope_split_ex");
    const at::ScalarType dt = qkv.scalar_type();
    const int code = type_code(dt);
    void *in = arg(qkv, c.device, {rows, (Hq + 2 * Hkv) * d}, dt, "qkv"), *pos = arg(a[4], c.device, {rows}, at::kInt, "positions");
    const str_rope_desc r = *desc;                                  // as it is now: another thread may change it once the lock is free
    const Shape qs = {rows, Hq, d}, ks = {rows, Hkv, d};
    at::Tensor o[3];
    int rc;
    {
        Unlocked free;
        Parts::make({{qs, dt}, {ks, dt}, {ks, dt}}, c.device, o);
        rc = f_rope(c.h, &r, code, rows, (int)Hq, (int)Hkv, (int)d, (const int32_t *)pos, in, o[0].data_ptr(), o[1].data_ptr(), o[2].data_ptr(), stream_of(c.device));
    }
    check(rc, "str_rope_split_ex");
    return Py_BuildValue("NNN", THPVariable_Wrap(o[0]), THPVariable_Wrap(o[1]), THPVariable_Wrap(o[2]));
}

// The arguments that both convolution calls share, a[2] ..: zxbcdt, conv_w, conv_b, dt_bias, H, p, n, G.
struct Conv {
    int rows, H, p, n, G, W, code;
    int64_t ch;
    at::ScalarType dt;
    void *zx, *w, *b, *dt_bias;
    Conv(PyObject *const *a, int device, const char *name) {
        const at::Tensor &z = tensor(a[2], "zxbcdt"), &taps = tensor(a[3], "conv_w");
        dims(z, 2, "zxbcdt");
        dims(taps, 2, "conv_w");
        H = (int)integer(a[6], 1, 1 << 20, "H"), p = (int)integer(a[7], 1, 1 << 20, "p"), n = (int)integer(a[8], 1, 1 << 20, "n"), G = (int)integer(a[9], 1, 1 << 20, "G");
        rows = int32(z.size(0), name);
        W = int32(taps.size(1), name);
        dt = z.scalar_type();
        code = type_code(dt);
        const int64_t d_inner = (int64_t)H * p;
        ch = d_inner + 2 * (int64_t)G * n;
        zx = arg(z, device, {rows, d_inner + ch + H}, dt, "zxbcdt");
        w = arg(taps, device, {ch, W}, at::kFloat, "conv_w");
        b = arg(a[4], device, {ch}, at::kFloat, "conv_b");
        dt_bias = arg(a[5], device, {H}, at::kFloat, "dt_bias");
    }
};

// conv_packed(handle, device, zxbcdt, conv_w, conv_b, dt_bias, H, p, n, G, seq_start, window, window_out, x, B, C, dt) -> (x, B, C, dt)
PyObject *conv_packed(PyObject *const *a) {
    const Ctx c(a);
    const Conv k(a, c.device, "str_mamba_conv_packed");
    const at::Tensor &start = tensor(a[10], "seq_start");
    const int n_seq = int32(sequences(start, "seq_start"), "str_mamba_conv_packed");
    void *st = arg(start, c.device, {(int64_t)n_seq + 1}, at::kInt, "seq_start");
    const Shape ws = {n_seq, k.W - 1, k.ch}, xs = {k.rows, k.H, k.p}, bs = {k.rows, k.G, k.n}, ds = {k.rows, k.H};
    void *win = optional(a[11], c.device, ws, k.dt, "window"), *wout = optional(a[12], c.device, ws, k.dt, "window_out");
    Out x(a[13], c.device, xs, k.dt, "out x"), B(a[14], c.device, bs, k.dt, "out B"), C(a[15], c.device, bs, k.dt, "out C"), dt(a[16], c.device, ds, at::kFloat, "out dt");
    int rc;
    {
        Unlocked free;
        x.make(c.device, xs, k.dt), B.make(c.device, bs, k.dt), C.make(c.device, bs, k.dt), dt.make(c.device, ds, at::kFloat);
        rc = f_conv(c.h, k.code, n_seq, k.rows, k.H, k.p, k.n, k.G, k.W, k.zx, (const float *)k.w, (const float *)k.b, (const float *)k.dt_bias,
                    (const int32_t *)st, win, x.p, B.p, C.p, (float *)dt.p, wout, stream_of(c.device));
    }
    check(rc, "str_mamba_conv_packed");
    return Py_BuildValue("NNNN", THPVariable_Wrap(x.t), THPVariable_Wrap(B.t), THPVariable_Wrap(C.t), THPVariable_Wrap(dt.t));
}

// conv_step(handle, device, zxbcdt, conv_w, conv_b, dt_bias, H, p, n, G, window, Bz, T, window_out) -> (x, B, C, dt)
PyObject *conv_step(PyObject *const *a) {
    const Ctx c(a);
    const Conv k(a, c.device, "str_mamba_conv_step");
    const int64_t Bz = integer(a[11], 0, INT32_MAX, "Bz"), T = integer(a[12], 0, INT32_MAX, "T");
    if (Bz * T != k.rows) {
        PyErr_Format(PyExc_ValueError, "zxbcdt: expected %lld x %lld rows, got %d", (long long)Bz, (long long)T, k.rows);
        throw Refused();
    }
    const Shape ws = {Bz, k.W - 1, k.ch};
    void *win = arg(a[10], c.device, ws, k.dt, "window"), *wout = arg(a[13], c.device, ws, k.dt, "window_out");
    const Shape xs = {Bz, T, k.H, k.p}, bs = {Bz, T, k.G, k.n}, ds = {Bz, T, k.H};
    at::Tensor o[4];
    int rc;
    {
        Unlocked free;
        Parts::make({{xs, k.dt}, {bs, k.dt}, {bs, k.dt}, {ds, at::kFloat}}, c.device, o);
        rc = f_conv_step(c.h, k.code, (int)Bz, (int)T, k.H, k.p, k.n, k.G, k.W, k.zx, (const float *)k.w, (const float *)k.b, (const float *)k.dt_bias, win,
                         o[0].data_ptr(), o[1].data_ptr(), o[2].data_ptr(), (float *)o[3].data_ptr(), wout, stream_of(c.device));
    }
    check(rc, "str_mamba_conv_step");
    return Py_BuildValue("NNNN", THPVariable_Wrap(o[0]), THPVariable_Wrap(o[1]), THPVariable_Wrap(o[2]), THPVariable_Wrap(o[3]));
}

// scan_packed(handle, device, x, dt, A, B, C, seq_start, D, init_state, final_state, y) -> y
PyObject *scan_packed(PyObject *const *a) {
    const Ctx c(a);
    const char *name = "str_mamba2_prefill_packed";
    const at::Tensor &x = tensor(a[2], "x"), &B = tensor(a[5], "B"), &start = tensor(a[7], "seq_start");
    dims(x, 3, "x");
    dims(B, 3, "B");
    const int64_t n_seq = sequences(start, "seq_start"), rows = x.size(0), H = x.size(1), p = x.size(2), G = B.size(1), n = B.size(2);
    const at::ScalarType t = x.scalar_type();
    const str_ssd_packed_shape s = {int32(n_seq, name), int32(rows, name), int32(H, name), int32(p, name), int32(n, name), int32(G, name), type_code(t)};
    const Shape states = {n_seq, H, p, n};
    void *px = arg(x, c.device, {rows, H, p}, t, "x"), *pdt = arg(a[3], c.device, {rows, H}, at::kFloat, "dt"), *pA = arg(a[4], c.device, {H}, at::kFloat, "A");
    void *pB = arg(B, c.device, {rows, G, n}, t, "B"), *pC = arg(a[6], c.device, {rows, G, n}, t, "C");
    void *ps = arg(start, c.device, {n_seq + 1}, at::kInt, "seq_start"), *pD = optional(a[8], c.device, {H}, at::kFloat, "D");
    void *init = optional(a[9], c.device, states, at::kFloat, "init_state"), *fin = optional(a[10], c.device, states, at::kFloat, "final_state");
    Out y(a[11], c.device, {rows, H, p}, t, "out");
    at::Tensor ws;
    int rc;
    {
        Unlocked free;
        const size_t need = f_scan_ws(&s);
        y.make(c.device, {rows, H, p}, t);
        if (need) ws = empty({(int64_t)need}, at::kByte, c.device);
        rc = f_scan(c.h, &s, px, (const float *)pdt, (const float *)pA, pB, pC, (const float *)pD, (const int32_t *)ps, (const float *)init, y.p, (float *)fin,
                    need ? ws.data_ptr() : nullptr, need, stream_of(c.device));
    }
    check(rc, name);
    return THPVariable_Wrap(y.t);
}

// attn_packed(handle, device, q, k, v, q_start, k_start, softmax_scale, o) -> o
PyObject *attn_packed(PyObject *const *a) {
    const Ctx c(a);
    const char *name = "str_attn_prefill_packed";
    const at::Tensor &q = tensor(a[2], "q"), &k = tensor(a[3], "k"), &start = tensor(a[5], "q_start");
    dims(q, 3, "q");
    dims(k, 3, "k");
    const int64_t n_seq = sequences(start, "q_start"), rows_q = q.size(0), Hq = q.size(1), d = q.size(2), rows_k = k.size(0), Hkv = k.size(1);
    const at::ScalarType t = q.scalar_type();
    const str_attn_packed_shape s = {int32(n_seq, name), int32(rows_q, name), int32(rows_k, name), int32(Hq, name), int32(Hkv, name), int32(d, name), type_code(t)};
    void *pq = arg(q, c.device, {rows_q, Hq, d}, t, "q"), *pk = arg(k, c.device, {rows_k, Hkv, d}, t, "k"), *pv = arg(a[4], c.device, {rows_k, Hkv, d}, t, "v");
    void *qs = arg(start, c.device, {n_seq + 1}, at::kInt, "q_start"), *ks = optional(a[6], c.device, {n_seq + 1}, at::kInt, "k_start");
    const double scale = PyFloat_AsDouble(a[7]);
    if (scale == -1.0 && PyErr_Occurred()) throw Refused();
    Out o(a[8], c.device, {rows_q, Hq, d}, t, "out");
    at::Tensor ws;
    int rc;
    {
        Unlocked free;
        const size_t need = f_attn_packed_ws(&s);
        o.make(c.device, {rows_q, Hq, d}, t);
        if (need) ws = empty({(int64_t)need}, at::kByte, c.device);
        rc = f_attn_packed(c.h, &s, pq, pk, pv, (const int32_t *)qs, (const int32_t *)ks, (float)scale, o.p, need ? ws.data_ptr() : nullptr, need, stream_of(c.device));
    }
    check(rc, name);
    return THPVariable_Wrap(o.t);
}

// No C++ exception leaves the module: what torch throws (out of memory, say) becomes a Python exception.
template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry(PyObject *, PyObject *const *args, Py_ssize_t n) {
    if (n != N) return PyErr_Format(PyExc_TypeError, "expected %d arguments, got %zd", N, n);
    if (!on_error) return PyErr_Format(PyExc_RuntimeError, "setup() has not been called");
    try {
        return F(args);
    } catch (const Refused &) {
        return nullptr;
    } catch (const c10::OutOfMemoryError &e) {
        PyErr_SetString(out_of_memory, e.what_without_backtrace());
    } catch (const c10::Error &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what_without_backtrace());
    } catch (const std::exception &e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}

// setup(on_error, out_of_memory, append, read, attn_workspace_size, attn, evict_workspace_size, evict, step): the last seven are the
// addresses of the entry points
PyObject *setup(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 9) return PyErr_Format(PyExc_TypeError, "expected 9 arguments, got %zd", n);
    void *p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i + 2]);
        if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "null entry point");
    }
    f_append = (decltype(f_append))p[0];
    f_read = (decltype(f_read))p[1];
    f_attn_ws = (decltype(f_attn_ws))p[2];
    f_attn = (decltype(f_attn))p[3];
    f_evict_ws = (decltype(f_evict_ws))p[4];
    f_evict = (decltype(f_evict))p[5];
    f_step = (decltype(f_step))p[6];
    Py_INCREF(a[0]);
    Py_XSETREF(on_error, a[0]);
    Py_INCREF(a[1]);
    Py_XSETREF(out_of_memory, a[1]);
    Py_RETURN_NONE;
}

// setup_packed(rope_split_ex, mamba_conv_packed, mamba_conv_step, mamba2_prefill_packed_workspace_size, mamba2_prefill_packed,
// attn_prefill_packed_workspace_size, attn_prefill_packed): the addresses of the entry points on packed sequences; after setup()
PyObject *setup_packed(PyObject *, PyObject *const *a, Py_ssize_t n) {
    if (n != 7) return PyErr_Format(PyExc_TypeError, "expected 7 arguments, got %zd", n);
    if (!on_error) return PyErr_Format(PyExc_RuntimeError, "setup() has not been called");
    void *p[7];
    for (int i = 0; i < 7; ++i) {
        p[i] = PyLong_AsVoidPtr(a[i]);
        if (!p[i]) return PyErr_Occurred() ? nullptr : PyErr_Format(PyExc_ValueError, "null entry point");
    }
    f_rope = (decltype(f_rope))p[0];
    f_conv = (decltype(f_conv))p[1];
    f_conv_step = (decltype(f_conv_step))p[2];
    f_scan_ws = (decltype(f_scan_ws))p[3];
    f_scan = (decltype(f_scan))p[4];
    f_attn_packed_ws = (decltype(f_attn_packed_ws))p[5];
    f_attn_packed = (decltype(f_attn_packed))p[6];
    Py_RETURN_NONE;
}

// The calls on packed sequences: entry(), once their entry points are known.
template <PyObject *(*F)(PyObject *const *), int N>
PyObject *entry_packed(PyObject *self, PyObject *const *args, Py_ssize_t n) {
    if (n == N && !f_rope) return PyErr_Format(PyExc_RuntimeError, "setup_packed() has not been called");
    return entry<F, N>(self, args, n);
}

#define ENTRY(name, N) {#name, (PyCFunction)(void (*)(void))entry<name, N>, METH_FASTCALL, nullptr}
#define ENTRY_PACKED(name, N) {#name, (PyCFunction)(void (*)(void))entry_packed<name, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, nullptr},
                         ENTRY(cache, 9), ENTRY(append, 9), ENTRY(read, 8), ENTRY(attn, 8), ENTRY(evict, 10), ENTRY(step, 10),
                         {"setup_packed", (PyCFunction)(void (*)(void))setup_packed, METH_FASTCALL, nullptr},
                         ENTRY_PACKED(rope, 8), ENTRY_PACKED(conv_packed, 17), ENTRY_PACKED(conv_step, 14), ENTRY_PACKED(scan_packed, 12),
                         ENTRY_PACKED(attn_packed, 9),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the decode calls and of those on packed sequences", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", STR_BUILT_FOR) < 0) Py_CLEAR(m);          // the torch whose headers it was built with
    return m;
}

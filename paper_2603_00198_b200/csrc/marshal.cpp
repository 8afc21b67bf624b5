// _marshal: argument marshalling of the decode calls for the Python binding, which are made once per layer and token: checks of the
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

#define ENTRY(name, N) {#name, (PyCFunction)(void (*)(void))entry<name, N>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"setup", (PyCFunction)(void (*)(void))setup, METH_FASTCALL, nullptr},
                         ENTRY(cache, 9), ENTRY(append, 9), ENTRY(read, 8), ENTRY(attn, 8), ENTRY(evict, 10), ENTRY(step, 10),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", "argument marshalling of the decode calls", -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject *m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", STR_BUILT_FOR) < 0) Py_CLEAR(m);          // the torch whose headers it was built with
    return m;
}

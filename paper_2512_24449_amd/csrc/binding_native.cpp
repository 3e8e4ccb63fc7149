// The calls of a decode step and of an append, marshalled in C++: binding.PackedKVCache, binding.FP4KVCache and binding.Rotary try these first.  A call whose
// arguments are not exactly what it expects (plain tensors of the right type, shape and layout) is answered with
// NotImplemented and made again by the Python code, which has the checks and raises the errors.
//
// A step of a small cache launches a few kernels of a few microseconds each, and marshalling through ctypes (1.3 us a call), checking shapes in Python (about 1)
// and torch.empty (1.5) took as long as they do.  Three steps over one
// stream of 1000 tokens 21.6 -> 18.0 us, over eight of 2296 24.8 -> 19.1; fused attention over eight of 650 13.2 -> 11.8.
#include <torch/csrc/autograd/python_variable.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/Exceptions.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/ops/empty.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>

#include <cstdint>
#include <cstring>
#include <string>

#include "../../include/packkv.h"

namespace {

// The library's entry points, by address (the library itself is loaded by binding.py), and what binding.py lends.
struct Library {
    int (*append)(void *, const void *, const void *, int32_t, void *);
    int (*append_bf16)(void *, const void *, const void *, int32_t, void *);
    int (*k_matvec)(void *, const void *, float, float *, int64_t, void *);
    int (*softmax)(void *, float *, int64_t, void *);
    int (*v_matvec)(void *, const float *, int64_t, float *, void *);
    int (*attention)(void *, const void *, float, float *, void *);
    int (*restore)(void *, int64_t);
    int (*release)(void *, void *);
    int64_t (*tokens)(const void *);
    int (*fp4_append)(void *, const void *, const void *, int64_t, const void *, int64_t, int32_t, int64_t, void *);
    int (*fp4_read)(void *, const void *, void *, void *, int32_t, int64_t, void *);
    int (*fp4_attention)(void *, const void *, const void *, int64_t, int32_t, int64_t, float, int32_t, int32_t, void *, int32_t,
                         float *, void *);
    int (*fp4_weights)(void *, const void *, const void *, int64_t, int32_t, int64_t, float, int32_t, int32_t, const float *,
                       const float *, float *, int64_t, void *);
    int (*fp4_select)(void *, const void *, const float *, int64_t, int32_t, const int32_t *, int32_t, int32_t, int32_t *, int32_t *,
                      void *);
    int (*fp4_compact)(void *, const void *, const void *, const int32_t *, int32_t, const int32_t *, const float *, int64_t, float *,
                       int64_t, void *);
    int (*rotary)(const void *, const int32_t *, int64_t, int32_t, int32_t, const void *, int64_t, int32_t, void *, int64_t, const void *,
                  int64_t, int32_t, void *, int64_t, void *);
} lib;
PyObject *check_code, *get_device, *get_stream, *in_bad_fork;

constexpr int64_t HEAD_DIM = 128;

struct Calls {
    PyObject_HEAD
    void *handle;
    int64_t batch, kv_heads, q_heads;
    c10::Device device;
};

PyObject *slow() { Py_RETURN_NOTIMPLEMENTED; }

// The hipStream_t meant by a `stream` argument: torch's current stream for None, or an integer.
bool stream_of(PyObject *stream, void *&out) {
    if (stream == Py_None) {
        PyObject *bad = PyObject_CallNoArgs(in_bad_fork);
        const bool fine = bad == Py_False;
        Py_XDECREF(bad);
        PyObject *device = fine ? PyObject_CallNoArgs(get_device) : nullptr;
        PyObject *raw = device ? PyObject_CallOneArg(get_stream, device) : nullptr;
        Py_XDECREF(device);
        if (raw) out = PyLong_AsVoidPtr(raw);
        Py_XDECREF(raw);
        if (!PyErr_Occurred()) return raw != nullptr;
        PyErr_Clear();
        return false;
    }
    if (!PyLong_CheckExact(stream)) return false;
    out = PyLong_AsVoidPtr(stream);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

bool scale_of(PyObject *o, float &out) {
    if (!PyFloat_CheckExact(o)) return false;
    out = float(PyFloat_AS_DOUBLE(o));
    return true;
}

// Function and dispatch modes (tracing, fake tensors, ...) see what the Python code calls.
bool modes() { return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set(); }

bool plain(PyObject *o, c10::ScalarType type) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.layout() == c10::kStrided && t.scalar_type() == type && t.is_contiguous();
}

bool rows(const at::Tensor &t, int64_t a, int64_t b) { return t.dim() == 3 && t.size(0) == a && t.size(1) == b; }

// `code` of the library as `result` (a new reference), or the error binding.py raises for it.
PyObject *answer(int code, const char *what, PyObject *result) {
    if (code == 0) return result;
    Py_XDECREF(result);
    PyObject *none = PyObject_CallFunction(check_code, "is", code, what);
    Py_XDECREF(none);
    if (none) PyErr_SetString(PyExc_RuntimeError, what);
    return nullptr;
}

template <class F>
int unlocked(F call) {   // as ctypes does: other Python threads run meanwhile
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = call();
    Py_END_ALLOW_THREADS
    return code;
}

at::Tensor new_floats(const Calls *c, int64_t last) {
    return at::empty({c->batch, c->q_heads, last}, at::TensorOptions().dtype(at::kFloat).device(c->device));
}

PyObject *append(Calls *c, PyObject *const *args, Py_ssize_t n) {   // k_new, v_new, stream
    HANDLE_TH_ERRORS
    void *s;
    if (n != 3 || !c->handle || modes() || !THPVariable_CheckExact(args[0])) return slow();
    const c10::ScalarType type = THPVariable_Unpack(args[0]).scalar_type();
    if ((type != at::kHalf && type != at::kBFloat16) || !plain(args[0], type) || !plain(args[1], type)) return slow();
    const at::Tensor &k = THPVariable_Unpack(args[0]), &v = THPVariable_Unpack(args[1]);
    if (k.dim() != 4 || k.sizes() != v.sizes() || k.size(0) != c->batch || k.size(2) != c->kv_heads || k.size(3) != HEAD_DIM ||
        k.size(1) > INT32_MAX || !stream_of(args[2], s))
        return slow();
    const void *kp = k.data_ptr(), *vp = v.data_ptr();
    const int32_t tokens = int32_t(k.size(1));
    const bool bf16 = type == at::kBFloat16;
    const int code = unlocked([&] { return (bf16 ? lib.append_bf16 : lib.append)(c->handle, kp, vp, tokens, s); });
    return answer(code, bf16 ? "kv_compress_append_bf16" : "kv_compress_append", Py_NewRef(Py_None));
    END_HANDLE_TH_ERRORS
}

PyObject *k_matvec(Calls *c, PyObject *const *args, Py_ssize_t n) {   // q, sm_scale, scores, stream
    HANDLE_TH_ERRORS
    void *s;
    float scale;
    if (n != 4 || !c->handle || modes() || !plain(args[0], at::kHalf) || !scale_of(args[1], scale)) return slow();
    const at::Tensor &q = THPVariable_Unpack(args[0]);
    if (!rows(q, c->batch, c->q_heads) || q.size(2) != HEAD_DIM) return slow();
    const bool fresh = args[2] == Py_None;
    if ((!fresh && (!plain(args[2], at::kFloat) || THPVariable_Unpack(args[2]).dim() != 3)) || !stream_of(args[3], s)) return slow();
    const at::Tensor scores = fresh ? new_floats(c, lib.tokens(c->handle)) : THPVariable_Unpack(args[2]);
    const void *qp = q.data_ptr();
    float *sp = static_cast<float *>(scores.data_ptr());
    const int64_t ld = scores.size(2);
    const int code = unlocked([&] { return lib.k_matvec(c->handle, qp, scale, sp, ld, s); });
    return answer(code, "kv_k_matvec", fresh ? THPVariable_Wrap(scores) : Py_NewRef(args[2]));
    END_HANDLE_TH_ERRORS
}

PyObject *softmax(Calls *c, PyObject *const *args, Py_ssize_t n) {   // scores, stream
    HANDLE_TH_ERRORS
    void *s;
    if (n != 2 || !c->handle || modes() || !plain(args[0], at::kFloat)) return slow();
    const at::Tensor &t = THPVariable_Unpack(args[0]);
    if (!rows(t, c->batch, c->q_heads) || !stream_of(args[1], s)) return slow();
    float *p = static_cast<float *>(t.data_ptr());
    const int64_t ld = t.size(2);
    const int code = unlocked([&] { return lib.softmax(c->handle, p, ld, s); });
    return answer(code, "kv_softmax", Py_NewRef(args[0]));
    END_HANDLE_TH_ERRORS
}

PyObject *v_matvec(Calls *c, PyObject *const *args, Py_ssize_t n) {   // p, stream; the output is new
    HANDLE_TH_ERRORS
    void *s;
    if (n != 2 || !c->handle || modes() || !plain(args[0], at::kFloat)) return slow();
    const at::Tensor &t = THPVariable_Unpack(args[0]);
    if (!rows(t, c->batch, c->q_heads) || !stream_of(args[1], s)) return slow();
    const at::Tensor out = new_floats(c, HEAD_DIM);
    const float *p = static_cast<const float *>(t.data_ptr());
    float *o = static_cast<float *>(out.data_ptr());
    const int64_t ld = t.size(2);
    const int code = unlocked([&] { return lib.v_matvec(c->handle, p, ld, o, s); });
    return answer(code, "kv_v_matvec", THPVariable_Wrap(out));
    END_HANDLE_TH_ERRORS
}

PyObject *attention(Calls *c, PyObject *const *args, Py_ssize_t n) {   // q, sm_scale, stream; the output is new
    HANDLE_TH_ERRORS
    void *s;
    float scale;
    if (n != 3 || !c->handle || modes() || !plain(args[0], at::kHalf) || !scale_of(args[1], scale)) return slow();
    const at::Tensor &q = THPVariable_Unpack(args[0]);
    if (!rows(q, c->batch, c->q_heads) || q.size(2) != HEAD_DIM || !stream_of(args[2], s)) return slow();
    const at::Tensor out = new_floats(c, HEAD_DIM);
    const void *qp = q.data_ptr();
    float *o = static_cast<float *>(out.data_ptr());
    const int code = unlocked([&] { return lib.attention(c->handle, qp, scale, o, s); });
    return answer(code, "kv_decode_attention", THPVariable_Wrap(out));
    END_HANDLE_TH_ERRORS
}

PyObject *restore(Calls *c, PyObject *tokens) {
    if (!c->handle || !PyLong_CheckExact(tokens)) return slow();
    int overflow;
    const long long t = PyLong_AsLongLongAndOverflow(tokens, &overflow);
    if (overflow) return slow();
    return answer(lib.restore(c->handle, t), "kv_cache_restore", Py_NewRef(Py_None));
}

PyObject *release(Calls *c, PyObject *stream) {
    void *s;
    if (!c->handle || !stream_of(stream, s)) return slow();
    return answer(unlocked([&] { return lib.release(c->handle, s); }), "kv_cache_release", Py_NewRef(Py_None));
}

PyObject *set_handle(Calls *c, PyObject *value) {   // an address, 0: every call takes the Python code
    void *h = PyLong_AsVoidPtr(value);
    if (PyErr_Occurred()) return nullptr;
    c->handle = h;
    Py_RETURN_NONE;
}

PyObject *calls_new(PyTypeObject *type, PyObject *args, PyObject *) {
    HANDLE_TH_ERRORS
    long long batch, kv_heads, q_heads;
    const char *device;
    if (!PyArg_ParseTuple(args, "LLLs", &batch, &kv_heads, &q_heads, &device)) return nullptr;
    const c10::Device d{std::string(device)};
    Calls *c = reinterpret_cast<Calls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->handle = nullptr;
    c->batch = batch, c->kv_heads = kv_heads, c->q_heads = q_heads;
    c->device = d;
    return reinterpret_cast<PyObject *>(c);
    END_HANDLE_TH_ERRORS
}

// ---- the 4-bit paged cache (binding.FP4KVCache) ----

struct FP4Calls {
    PyObject_HEAD
    void *handle;
    int64_t kv_heads, q_heads, head_dim;
    c10::Device device;
};

// torch's current stream, if `on` is the current device.
bool current_stream(const c10::Device &on, void *&out) {
    PyObject *bad = PyObject_CallNoArgs(in_bad_fork);
    const bool fine = bad == Py_False;
    Py_XDECREF(bad);
    PyObject *device = fine ? PyObject_CallNoArgs(get_device) : nullptr;
    PyObject *raw = device && PyLong_AsLong(device) == on.index() ? PyObject_CallOneArg(get_stream, device) : nullptr;
    Py_XDECREF(device);
    if (raw) out = PyLong_AsVoidPtr(raw);
    Py_XDECREF(raw);
    if (!PyErr_Occurred()) return raw != nullptr;
    PyErr_Clear();
    return false;
}

// A batch: its address and the index of its device.
bool batch_of(const FP4Calls *c, PyObject *address, PyObject *device, const void *&out) {
    if (!PyLong_CheckExact(address) || !PyLong_CheckExact(device) || PyLong_AsLong(device) != c->device.index()) return PyErr_Clear(), false;
    out = PyLong_AsVoidPtr(address);
    return PyErr_Occurred() ? (PyErr_Clear(), false) : out != nullptr;
}

struct Rows {
    const at::Tensor *t;
    int64_t rows, pitch;
};

// [rows, heads, D] of fp16 or bf16 on the cache's device, the heads of a row next to each other.
bool rows_of(const FP4Calls *c, PyObject *o, int64_t heads, Rows &out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.layout() != c10::kStrided || (t.scalar_type() != at::kHalf && t.scalar_type() != at::kBFloat16) || t.dim() != 3 ||
        t.device() != c->device || t.size(1) != heads || t.size(2) != c->head_dim || t.stride(2) != 1 ||
        (heads > 1 && t.stride(1) != c->head_dim) || t.is_conj() || t.is_neg())
        return false;
    out = {&t, t.size(0), t.size(0) > 1 ? t.stride(0) : heads * c->head_dim};
    return true;
}

bool count_of(PyObject *o, int32_t &out) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow;
    const long long x = PyLong_AsLongLongAndOverflow(o, &overflow);
    out = int32_t(x);
    return !overflow && x >= 0 && x <= INT32_MAX;
}

int32_t type_of(c10::ScalarType t) { return t == at::kHalf ? 0 : t == at::kBFloat16 ? 1 : 2; }

PyObject *fp4_append(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // k, v, batch, its device, stream
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    Rows k, v;
    if (n != 5 || !c->handle || args[4] != Py_None || modes() || !batch_of(c, args[2], args[3], batch) ||
        !rows_of(c, args[0], c->kv_heads, k) || !rows_of(c, args[1], c->kv_heads, v) || k.rows != v.rows ||
        k.t->scalar_type() != v.t->scalar_type() || !current_stream(c->device, s))
        return slow();
    const void *kp = k.t->data_ptr(), *vp = v.t->data_ptr();
    const int32_t type = type_of(k.t->scalar_type());
    const int code = unlocked([&] { return lib.fp4_append(c->handle, batch, kp, k.pitch, vp, v.pitch, type, k.rows, s); });
    return answer(code, "kv_fp4_append", Py_NewRef(Py_None));
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_read(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // batch, its device, n_rows, dtype, stream; the outputs are new
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    int32_t rows;
    if (n != 5 || !c->handle || args[4] != Py_None || modes() || !batch_of(c, args[0], args[1], batch) || !count_of(args[2], rows) ||
        !THPDtype_Check(args[3]))
        return slow();
    const c10::ScalarType type = reinterpret_cast<THPDtype *>(args[3])->scalar_type;
    if ((type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) || !current_stream(c->device, s)) return slow();
    const at::TensorOptions options = at::TensorOptions().dtype(type).device(c->device);
    const at::Tensor k = at::empty({rows, c->kv_heads, c->head_dim}, options), v = at::empty({rows, c->kv_heads, c->head_dim}, options);
    void *kp = k.data_ptr(), *vp = v.data_ptr();
    const int code = unlocked([&] { return lib.fp4_read(c->handle, batch, kp, vp, type_of(type), rows, s); });
    PyObject *first = THPVariable_Wrap(k), *second = THPVariable_Wrap(v);
    PyObject *both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both ? answer(code, "kv_fp4_read", both) : nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_attention(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // q, batch, its device, sm_scale, window, sinks, stream; the output is new
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    float scale;
    int32_t window, sinks;
    Rows q;
    if (n != 7 || !c->handle || args[6] != Py_None || modes() || !batch_of(c, args[1], args[2], batch) || !scale_of(args[3], scale) ||
        !count_of(args[4], window) || !count_of(args[5], sinks) || !rows_of(c, args[0], c->q_heads, q) || !current_stream(c->device, s))
        return slow();
    const c10::ScalarType type = q.t->scalar_type();
    const at::Tensor out = at::empty({q.rows, c->q_heads, c->head_dim}, at::TensorOptions().dtype(type).device(c->device));
    const void *qp = q.t->data_ptr();
    void *op = out.data_ptr();
    const int32_t t = type_of(type);
    const int code = unlocked([&] { return lib.fp4_attention(c->handle, batch, qp, q.pitch, t, q.rows, scale, window, sinks, op, t, nullptr, s); });
    return answer(code, "kv_fp4_attention", THPVariable_Wrap(out));
    END_HANDLE_TH_ERRORS
}

// A contiguous tensor of `type` on the device; its shape is the caller's to look at.
const at::Tensor *plain_on(const c10::Device &device, PyObject *o, c10::ScalarType type) {
    if (!plain(o, type)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.device() == device && !t.is_neg() ? &t : nullptr;
}

int32_t sequences(const void *batch) { return static_cast<const kv_fp4_batch_t *>(batch)->batch; }

bool streams_of(const FP4Calls *c, const at::Tensor &t, const void *batch) {
    return t.dim() == 3 && t.size(0) == sequences(batch) && t.size(1) == c->kv_heads;
}

PyObject *fp4_read_into(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // batch, its device, n_rows, k, v, stream
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    int32_t rows;
    if (n != 6 || !c->handle || args[5] != Py_None || modes() || !batch_of(c, args[0], args[1], batch) || !count_of(args[2], rows) ||
        !THPVariable_CheckExact(args[3]))
        return slow();
    const c10::ScalarType type = THPVariable_Unpack(args[3]).scalar_type();
    if (type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) return slow();
    const at::Tensor *k = plain_on(c->device, args[3], type), *v = plain_on(c->device, args[4], type);
    for (const at::Tensor *t : {k, v})
        if (!t || t->dim() != 3 || t->size(0) != rows || t->size(1) != c->kv_heads || t->size(2) != c->head_dim) return slow();
    if (!current_stream(c->device, s)) return slow();
    void *kp = k->data_ptr(), *vp = v->data_ptr();
    const int code = unlocked([&] { return lib.fp4_read(c->handle, batch, kp, vp, type_of(type), rows, s); });
    return answer(code, "kv_fp4_read", PyTuple_Pack(2, args[3], args[4]));
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_weights(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // q, lse, batch, its device, sm_scale, window, sinks, past, out, stream
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    float scale;
    int32_t window, sinks;
    Rows q;
    if (n != 10 || !c->handle || args[9] != Py_None || modes() || !batch_of(c, args[2], args[3], batch) || !scale_of(args[4], scale) ||
        !count_of(args[5], window) || !count_of(args[6], sinks) || !rows_of(c, args[0], c->q_heads, q))
        return slow();
    const at::Tensor *lse = plain_on(c->device, args[1], at::kFloat), *out = plain_on(c->device, args[8], at::kFloat);
    const bool added = args[7] != Py_None;
    const at::Tensor *past = added ? plain_on(c->device, args[7], at::kFloat) : nullptr;
    if (!lse || lse->dim() != 2 || lse->size(0) != q.rows || lse->size(1) != c->q_heads || !out || !streams_of(c, *out, batch) ||
        (added && (!past || past->sizes() != out->sizes())) || !current_stream(c->device, s))
        return slow();
    const void *qp = q.t->data_ptr();
    const float *lp = static_cast<const float *>(lse->data_ptr()), *pp = added ? static_cast<const float *>(past->data_ptr()) : nullptr;
    float *op = static_cast<float *>(out->data_ptr());
    const int32_t type = type_of(q.t->scalar_type());
    const int64_t tokens = out->size(2);
    const int code = unlocked([&] {
        return lib.fp4_weights(c->handle, batch, qp, q.pitch, type, q.rows, scale, window, sinks, lp, pp, op, tokens, s);
    });
    return answer(code, "kv_fp4_weights", Py_NewRef(args[8]));
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_select(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // mass, batch, its device, keep, sinks, recent, n_kept, stream; kept is new
    HANDLE_TH_ERRORS
    void *s;
    const void *batch;
    int32_t keep, sinks, recent;
    if (n != 8 || !c->handle || args[7] != Py_None || modes() || !batch_of(c, args[1], args[2], batch) || !count_of(args[3], keep) || keep < 1 ||
        !count_of(args[4], sinks) || !count_of(args[5], recent))
        return slow();
    const at::Tensor *mass = plain_on(c->device, args[0], at::kFloat);
    const bool fresh = args[6] == Py_None;
    const at::Tensor *given = fresh ? nullptr : plain_on(c->device, args[6], at::kInt);
    if (!mass || !streams_of(c, *mass, batch) || (!fresh && (!given || given->dim() != 1 || given->size(0) != sequences(batch))) ||
        !current_stream(c->device, s))
        return slow();
    const at::TensorOptions options = at::TensorOptions().dtype(at::kInt).device(c->device);
    const at::Tensor kept = at::empty({sequences(batch), c->kv_heads, keep}, options);
    const at::Tensor count = fresh ? at::empty({sequences(batch)}, options) : *given;
    const float *mp = static_cast<const float *>(mass->data_ptr());
    int32_t *kp = static_cast<int32_t *>(kept.data_ptr()), *cp = static_cast<int32_t *>(count.data_ptr());
    const int64_t tokens = mass->size(2);
    const int code = unlocked([&] { return lib.fp4_select(c->handle, batch, mp, tokens, keep, nullptr, sinks, recent, kp, cp, s); });
    PyObject *first = THPVariable_Wrap(kept), *second = fresh ? THPVariable_Wrap(count) : Py_NewRef(args[6]);
    PyObject *both = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return both ? answer(code, "kv_fp4_select", both) : nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_compact(FP4Calls *c, PyObject *const *args, Py_ssize_t n) {   // kept, n_kept, batch, its device, to, its device, mass, mass_out, stream
    HANDLE_TH_ERRORS
    void *s;
    const void *batch, *to;
    if (n != 9 || !c->handle || args[8] != Py_None || modes() || !batch_of(c, args[2], args[3], batch) || !batch_of(c, args[4], args[5], to) ||
        sequences(batch) != sequences(to))
        return slow();
    const at::Tensor *kept = plain_on(c->device, args[0], at::kInt), *count = plain_on(c->device, args[1], at::kInt);
    const bool weighed = args[6] != Py_None;
    const at::Tensor *mass = weighed ? plain_on(c->device, args[6], at::kFloat) : nullptr;
    const at::Tensor *out = weighed ? plain_on(c->device, args[7], at::kFloat) : nullptr;
    if (!kept || !streams_of(c, *kept, batch) || kept->size(2) > INT32_MAX || !count || count->dim() != 1 || count->size(0) != sequences(batch) ||
        (weighed && (!mass || !out || !streams_of(c, *mass, batch) || !streams_of(c, *out, batch))) || (!weighed && args[7] != Py_None) ||
        !current_stream(c->device, s))
        return slow();
    const int32_t *kp = static_cast<const int32_t *>(kept->data_ptr()), *cp = static_cast<const int32_t *>(count->data_ptr());
    const float *mp = weighed ? static_cast<const float *>(mass->data_ptr()) : nullptr;
    float *op = weighed ? static_cast<float *>(out->data_ptr()) : nullptr;
    const int64_t tokens = weighed ? mass->size(2) : 0, out_tokens = weighed ? out->size(2) : 0;
    const int32_t keep = int32_t(kept->size(2));
    const int code = unlocked([&] { return lib.fp4_compact(c->handle, batch, to, kp, keep, cp, mp, tokens, op, out_tokens, s); });
    return answer(code, "kv_fp4_compact", Py_NewRef(args[7]));
    END_HANDLE_TH_ERRORS
}

// ---- rotary positions (binding.Rotary) ----

struct RotaryCalls {
    PyObject_HEAD
    const void *table;       // kv_rotary_t, the caller's
    int64_t head_dim;
    c10::Device device;
};

// [rows, heads, head_dim] of `type`, the heads of a row next to each other.
bool turned_rows(const RotaryCalls *c, PyObject *o, c10::ScalarType type, Rows &out) {
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.layout() != c10::kStrided || t.scalar_type() != type || t.dim() != 3 || t.device() != c->device || t.size(2) != c->head_dim ||
        t.size(1) > INT32_MAX || t.stride(2) != 1 || (t.size(1) > 1 && t.stride(1) != c->head_dim) || t.is_conj() || t.is_neg())
        return false;
    out = {&t, t.size(0), t.size(0) > 1 ? t.stride(0) : t.size(1) * c->head_dim};
    return true;
}

PyObject *rotary_turn(RotaryCalls *c, PyObject *const *args, Py_ssize_t n) {   // q, positions, k, out, k_out, inverse, stream
    HANDLE_TH_ERRORS
    void *s;
    if (n != 7 || args[6] != Py_None || modes() || !THPVariable_CheckExact(args[0]) || (args[5] != Py_True && args[5] != Py_False)) return slow();
    const c10::ScalarType type = THPVariable_Unpack(args[0]).scalar_type();
    if (type != at::kHalf && type != at::kBFloat16 && type != at::kFloat) return slow();
    const bool both = args[2] != Py_None;
    Rows in[2], to[2];
    if (!turned_rows(c, args[0], type, in[0]) || (both && !turned_rows(c, args[2], type, in[1])) || (!both && args[4] != Py_None)) return slow();
    const at::Tensor *positions = plain_on(c->device, args[1], at::kInt);
    if (!positions || positions->dim() != 1 || positions->size(0) != in[0].rows || (both && in[1].rows != in[0].rows)) return slow();
    at::Tensor made[2];
    for (int i = 0; i < (both ? 2 : 1); ++i) {
        if (args[3 + i] != Py_None) {
            if (!turned_rows(c, args[3 + i], type, to[i]) || to[i].t->sizes() != in[i].t->sizes()) return slow();
        }
    }
    if (!current_stream(c->device, s)) return slow();
    for (int i = 0; i < (both ? 2 : 1); ++i) {
        if (args[3 + i] != Py_None) continue;
        made[i] = at::empty(in[i].t->sizes(), at::TensorOptions().dtype(type).device(c->device));
        to[i] = {&made[i], in[i].rows, in[i].t->size(1) * c->head_dim};
    }
    const void *from[2] = {in[0].t->data_ptr(), both ? in[1].t->data_ptr() : nullptr};
    void *into[2] = {to[0].t->data_ptr(), both ? to[1].t->data_ptr() : nullptr};
    const int32_t heads[2] = {int32_t(in[0].t->size(1)), both ? int32_t(in[1].t->size(1)) : 0};
    const int32_t *at = static_cast<const int32_t *>(positions->data_ptr());
    const int32_t inverse = args[5] == Py_True;
    const int code = unlocked([&] {
        return lib.rotary(c->table, at, in[0].rows, type_of(type), inverse, from[0], in[0].pitch, heads[0], into[0], to[0].pitch, from[1],
                          both ? in[1].pitch : 0, heads[1], into[1], both ? to[1].pitch : 0, s);
    });
    PyObject *first = args[3] == Py_None ? THPVariable_Wrap(made[0]) : Py_NewRef(args[3]);
    if (!both) return first ? answer(code, "kv_rotary", first) : nullptr;
    PyObject *second = args[4] == Py_None ? THPVariable_Wrap(made[1]) : Py_NewRef(args[4]);
    PyObject *pair = first && second ? PyTuple_Pack(2, first, second) : nullptr;
    Py_XDECREF(first);
    Py_XDECREF(second);
    return pair ? answer(code, "kv_rotary", pair) : nullptr;
    END_HANDLE_TH_ERRORS
}

PyObject *rotary_calls_new(PyTypeObject *type, PyObject *args, PyObject *) {   // address of the kv_rotary_t, head_dim, device
    HANDLE_TH_ERRORS
    unsigned long long table;
    long long head_dim;
    const char *device;
    if (!PyArg_ParseTuple(args, "KLs", &table, &head_dim, &device)) return nullptr;
    const c10::Device d{std::string(device)};
    RotaryCalls *c = reinterpret_cast<RotaryCalls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->table = reinterpret_cast<const void *>(uintptr_t(table));
    c->head_dim = head_dim;
    c->device = d;
    return reinterpret_cast<PyObject *>(c);
    END_HANDLE_TH_ERRORS
}

PyObject *fp4_set_handle(FP4Calls *c, PyObject *value) {
    void *h = PyLong_AsVoidPtr(value);
    if (PyErr_Occurred()) return nullptr;
    c->handle = h;
    Py_RETURN_NONE;
}

PyObject *fp4_calls_new(PyTypeObject *type, PyObject *args, PyObject *) {
    HANDLE_TH_ERRORS
    long long kv_heads, q_heads, head_dim;
    const char *device;
    if (!PyArg_ParseTuple(args, "LLLs", &kv_heads, &q_heads, &head_dim, &device)) return nullptr;
    const c10::Device d{std::string(device)};
    FP4Calls *c = reinterpret_cast<FP4Calls *>(type->tp_alloc(type, 0));
    if (!c) return nullptr;
    c->handle = nullptr;
    c->kv_heads = kv_heads, c->q_heads = q_heads, c->head_dim = head_dim;
    c->device = d;
    return reinterpret_cast<PyObject *>(c);
    END_HANDLE_TH_ERRORS
}

#define FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef calls_methods[] = {
    FAST(append), FAST(k_matvec), FAST(softmax), FAST(v_matvec), FAST(attention),
    {"restore", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(restore)), METH_O, nullptr},
    {"release", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(release)), METH_O, nullptr},
    {"set_handle", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(set_handle)), METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

#define FAST_FP4(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_##name)), METH_FASTCALL, nullptr}
PyMethodDef fp4_calls_methods[] = {
    FAST_FP4(append), FAST_FP4(read), FAST_FP4(read_into), FAST_FP4(attention), FAST_FP4(weights), FAST_FP4(select), FAST_FP4(compact),
    {"set_handle", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fp4_set_handle)), METH_O, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyMethodDef rotary_calls_methods[] = {
    {"turn", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(rotary_turn)), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};

PyTypeObject calls_type = {PyVarObject_HEAD_INIT(nullptr, 0)}, fp4_calls_type = {PyVarObject_HEAD_INIT(nullptr, 0)},
             rotary_calls_type = {PyVarObject_HEAD_INIT(nullptr, 0)};

// bind(addresses of the entry points in Library's order, _check, device getter, stream getter, bad-fork test)
PyObject *bind(PyObject *, PyObject *args) {
    PyObject *addresses, *check, *device, *stream, *fork;
    if (!PyArg_ParseTuple(args, "O!OOOO", &PyTuple_Type, &addresses, &check, &device, &stream, &fork)) return nullptr;
    constexpr Py_ssize_t COUNT = sizeof(Library) / sizeof(void *);
    if (PyTuple_GET_SIZE(addresses) != COUNT) return PyErr_SetString(PyExc_ValueError, "bind: wrong number of entry points"), nullptr;
    void *at[COUNT];
    for (Py_ssize_t i = 0; i < COUNT; ++i) at[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(addresses, i));
    if (PyErr_Occurred()) return nullptr;
    memcpy(&lib, at, sizeof(lib));
    PyObject **const lent[] = {&check_code, &get_device, &get_stream, &in_bad_fork};
    PyObject *const given[] = {check, device, stream, fork};
    for (int i = 0; i < 4; ++i) {
        Py_XDECREF(*lent[i]);
        *lent[i] = Py_NewRef(given[i]);
    }
    Py_RETURN_NONE;
}

PyMethodDef module_methods[] = {{"bind", bind, METH_VARARGS, nullptr}, {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_native", "Marshalling of binding.py's frequent calls.", -1, module_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native() {
    calls_type.tp_name = "paper_2512_24449_amd._native.Calls";
    calls_type.tp_basicsize = sizeof(Calls);
    calls_type.tp_flags = Py_TPFLAGS_DEFAULT;
    calls_type.tp_new = calls_new;
    calls_type.tp_methods = calls_methods;
    fp4_calls_type.tp_name = "paper_2512_24449_amd._native.FP4Calls";
    fp4_calls_type.tp_basicsize = sizeof(FP4Calls);
    fp4_calls_type.tp_flags = Py_TPFLAGS_DEFAULT;
    fp4_calls_type.tp_new = fp4_calls_new;
    fp4_calls_type.tp_methods = fp4_calls_methods;
    rotary_calls_type.tp_name = "paper_2512_24449_amd._native.RotaryCalls";
    rotary_calls_type.tp_basicsize = sizeof(RotaryCalls);
    rotary_calls_type.tp_flags = Py_TPFLAGS_DEFAULT;
    rotary_calls_type.tp_new = rotary_calls_new;
    rotary_calls_type.tp_methods = rotary_calls_methods;
    if (PyType_Ready(&calls_type) < 0 || PyType_Ready(&fp4_calls_type) < 0 || PyType_Ready(&rotary_calls_type) < 0) return nullptr;
    PyObject *m = PyModule_Create(&module);
    if (m && (PyModule_AddObject(m, "Calls", Py_NewRef(reinterpret_cast<PyObject *>(&calls_type))) < 0 ||
              PyModule_AddObject(m, "FP4Calls", Py_NewRef(reinterpret_cast<PyObject *>(&fp4_calls_type))) < 0 ||
              PyModule_AddObject(m, "RotaryCalls", Py_NewRef(reinterpret_cast<PyObject *>(&rotary_calls_type))) < 0)) {
        Py_DECREF(m);
        return nullptr;
    }
    return m;
}

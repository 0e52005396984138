// Host side of a Python call of the decoder's operators: reads the tensors, checks them and
// calls the C interface, in about half a microsecond; reading the same attributes from Python and passing
// them through ctypes takes 3.5, as long as the launch itself, and a step of single tokens is bound by it
// (packed_rmsnorm of 8 x 1024, call after call: 3.5 and 6.4 us).
// Only calls whose arguments are all as documented go this way; for every other one the functions
// return None and launch nothing, and the Python caller makes its own checks, which say
// what is wrong.  Tensors are read, never kept.
#include <Python.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstdint>

#include "ragged.h"

namespace {

PyObject *current_device, *raw_stream;  // torch's, as Python calls them
PyObject *name_c, *name_status, *name_stream;
struct {
    decltype(&packed_rmsnorm) rmsnorm;
    decltype(&packed_quantize_i8) quantize_i8;
    decltype(&packed_linear_i8) linear_i8;
    decltype(&packed_rotary) rotary;
    decltype(&ragged_attention_window) window;
    decltype(&ragged_attention_window_cached) window_cached;
} lib;

struct NotPlain {};  // an argument is not as documented
void need(bool ok) {
    if (!ok) throw NotPlain{};
}

struct Ref {  // a new reference; an error pending in Python is cleared and refused
    PyObject* p;
    explicit Ref(PyObject* q) : p(q) { need(q != nullptr); }
    ~Ref() { Py_XDECREF(p); }
    Ref(const Ref&) = delete;
};

const at::Tensor& tensor(PyObject* o) {
    need(THPVariable_CheckExact(o));
    const at::Tensor& t = THPVariable_Unpack(o);
    need(t.defined() && t.is_cuda() && t.layout() == at::kStrided);
    return t;
}

struct Mat {
    void* p = nullptr;
    int32_t ld = 0;
};

Mat mat(PyObject* o, int64_t rows, int64_t cols, at::ScalarType type, int dev) {
    if (o == Py_None) return {};
    const at::Tensor& t = tensor(o);
    need(t.dim() == 2 && t.size(0) == rows && t.size(1) == cols && t.scalar_type() == type && t.get_device() == dev &&
         t.stride(1) == 1 && t.stride(0) >= 0 && t.stride(0) <= INT32_MAX);
    return {t.data_ptr(), (int32_t)t.stride(0)};
}

void* vec(PyObject* o, int64_t n, at::ScalarType type, int dev) {
    if (o == Py_None) return nullptr;
    const at::Tensor& t = tensor(o);
    need(t.dim() == 1 && t.size(0) == n && t.scalar_type() == type && t.get_device() == dev && (n <= 1 || t.stride(0) == 1));
    return t.data_ptr();
}

int32_t dtype_of(const at::Tensor& t) {
    need(t.scalar_type() == at::kBFloat16 || t.scalar_type() == at::kFloat);
    return t.scalar_type() == at::kBFloat16 ? RAG_BF16 : RAG_F32;
}

int32_t size32(int64_t n) {
    need(n >= 0 && n <= INT32_MAX);
    return (int32_t)n;
}

int64_t integer(PyObject* o, bool clamp = false) {  // in 32 bits; larger ones refused, or held at the largest
    need(PyLong_Check(o));
    int over = 0;
    const long long v = PyLong_AsLongLongAndOverflow(o, &over);
    if (clamp && (over > 0 || v > INT32_MAX)) return INT32_MAX;
    need(!over && v >= INT32_MIN && v <= INT32_MAX);
    return v;
}

double real(PyObject* o) {
    need(PyFloat_Check(o) || PyLong_Check(o));
    const double v = PyFloat_AsDouble(o);
    need(!PyErr_Occurred());
    return v;
}

void* stream_on(PyObject* stream, int dev) {  // the stream to launch on, if `dev` is the current device
    const Ref cur(PyObject_CallNoArgs(current_device));
    need(PyLong_AsLong(cur.p) == dev);
    const Ref number(stream == Py_None ? PyObject_CallOneArg(raw_stream, cur.p) : PyObject_GetAttr(stream, name_stream));
    void* const s = PyLong_AsVoidPtr(number.p);
    need(!PyErr_Occurred());
    return s;
}

struct PlanRef {  // the C plan of a Python one
    Py_buffer view{};
    PlanRef(PyObject* plan, int dev) {
        const Ref c(PyObject_GetAttr(plan, name_c)), status(PyObject_GetAttr(plan, name_status));
        need(tensor(status.p).get_device() == dev);
        need(PyObject_GetBuffer(c.p, &view, PyBUF_SIMPLE) == 0);
        if (view.len != (Py_ssize_t)sizeof(rag_plan)) {
            PyBuffer_Release(&view);
            throw NotPlain{};
        }
    }
    ~PlanRef() { PyBuffer_Release(&view); }
    PlanRef(const PlanRef&) = delete;
    const rag_plan* operator->() const { return get(); }
    const rag_plan* get() const { return static_cast<const rag_plan*>(view.buf); }
};

template <typename F, typename... A>
PyObject* launch(F f, A... args) {
    rag_status st;
    Py_BEGIN_ALLOW_THREADS
    st = f(args...);
    Py_END_ALLOW_THREADS
    return PyLong_FromLong(st);
}

PyObject* rmsnorm(PyObject* const* a) {  // x, gamma, y, eps, residual, x_out, q, q_scale, stream
    const at::Tensor& x = tensor(a[0]);
    need(x.dim() == 2);
    const int64_t T = x.size(0), d = x.size(1);
    const auto type = x.scalar_type();
    const int dev = x.get_device();
    const int32_t dt = dtype_of(x);
    const Mat mx = mat(a[0], T, d, type, dev), mr = mat(a[4], T, d, type, dev), ms = mat(a[5], T, d, type, dev),
              my = mat(a[2], T, d, type, dev), mq = mat(a[6], T, d, at::kChar, dev);
    void *const g = vec(a[1], d, type, dev), *const qs = vec(a[7], T, at::kFloat, dev);
    return launch(lib.rmsnorm, mx.p, mx.ld, mr.p, mr.ld, g, (float)real(a[3]), ms.p, ms.ld, my.p, my.ld, (int8_t*)mq.p, mq.ld,
                  (float*)qs, size32(T), size32(d), dt, stream_on(a[8], dev));
}

PyObject* quantize_i8(PyObject* const* a) {  // x, q, scale, stream
    const at::Tensor& x = tensor(a[0]);
    need(x.dim() == 2);
    const int64_t T = x.size(0), d = x.size(1);
    const int dev = x.get_device();
    const int32_t dt = dtype_of(x);
    const Mat mx = mat(a[0], T, d, x.scalar_type(), dev), mq = mat(a[1], T, d, at::kChar, dev);
    void* const s = vec(a[2], T, at::kFloat, dev);
    return launch(lib.quantize_i8, mx.p, mx.ld, (int8_t*)mq.p, mq.ld, (float*)s, size32(T), size32(d), dt, stream_on(a[3], dev));
}

PyObject* linear_i8(PyObject* const* a) {  // x, x_scale, w, w_scale, y, bias, residual, act, stream
    const at::Tensor &y = tensor(a[4]), &x = tensor(a[0]), &w = tensor(a[2]);
    need(x.dim() == 2 && w.dim() == 2);
    const int64_t T = x.size(0), K = x.size(1), N = w.size(0);
    const auto type = y.scalar_type();
    const int dev = y.get_device();
    const int32_t dt = dtype_of(y);
    const Mat mx = mat(a[0], T, K, at::kChar, dev), mw = mat(a[2], N, K, at::kChar, dev), my = mat(a[4], T, N, type, dev),
              mr = mat(a[6], T, N, type, dev);
    need(mw.ld == K || N <= 1);
    void *const xs = vec(a[1], T, at::kFloat, dev), *const ws = vec(a[3], N, at::kFloat, dev), *const b = vec(a[5], N, type, dev);
    return launch(lib.linear_i8, (int8_t*)mx.p, mx.ld, (float*)xs, (int8_t*)mw.p, (float*)ws, b, mr.p, mr.ld,
                  (int32_t)integer(a[7]), my.p, my.ld, size32(T), size32(K), size32(N), dt, stream_on(a[8], dev));
}

PyObject* rotary(PyObject* const* a) {  // plan, x, y, inv_freq, heads, head_dim, layout, amplitude, pos_start, inverse, stream
    const at::Tensor &x = tensor(a[1]), &f = tensor(a[3]);
    const int dev = x.get_device();
    const int32_t dt = dtype_of(x);
    const PlanRef plan(a[0], dev);
    const int64_t heads = integer(a[4]), hd = integer(a[5]), n = f.numel();
    need(n <= (1 << 20) && PyBool_Check(a[9]));
    const Mat mx = mat(a[1], plan->total_tokens, heads * hd, x.scalar_type(), dev),
              my = mat(a[2], plan->total_tokens, heads * hd, x.scalar_type(), dev);
    need(a[2] != Py_None);
    void *const fr = vec(a[3], n, at::kDouble, dev), *const pos = vec(a[8], plan->batch, at::kInt, dev);
    const int32_t layout = (int32_t)integer(a[6]) | (a[9] == Py_True ? RAG_ROTARY_INVERSE : 0);
    return launch(lib.rotary, plan.get(), mx.p, mx.ld, my.p, my.ld, (int32_t)heads, (int32_t)hd, (int32_t)(2 * n), layout, (double*)fr,
                  (float)real(a[7]), (int32_t*)pos, dt, stream_on(a[10], dev));
}

struct Window {  // what the two window calls share
    int dev;
    int32_t dt, kv_heads, hd;
    Mat q, k, v, out;
    void* ws = nullptr;
    size_t ws_bytes = 0;
    Window(const rag_plan* plan, const at::Tensor& tq, PyObject* oq, PyObject* ok, PyObject* ov, PyObject* oout, int64_t rows,
           PyObject* kvh, PyObject* head_dim, PyObject* workspace)
        : dev(tq.get_device()), dt(dtype_of(tq)), kv_heads(kvh == Py_None ? 0 : (int32_t)integer(kvh)), hd((int32_t)integer(head_dim)) {
        if (kv_heads == 0) kv_heads = plan->heads;
        need(ok != Py_None && ov != Py_None && oout != Py_None);
        const int64_t T = plan->total_tokens, wide = (int64_t)plan->heads * hd, kv = (int64_t)kv_heads * hd;
        const auto type = tq.scalar_type();
        q = mat(oq, T, wide, type, dev);
        k = mat(ok, rows, kv, type, dev);
        v = mat(ov, rows, kv, type, dev);
        out = mat(oout, T, wide, type, dev);
        if (workspace != Py_None) {
            const at::Tensor& t = tensor(workspace);
            need(t.is_contiguous() && t.get_device() == dev);
            ws = t.data_ptr();
            ws_bytes = (size_t)t.numel() * t.element_size();
        }
    }
};

PyObject* window(PyObject* const* a) {  // plan, q, k, v, out, scale, window, sinks, kv_heads, head_dim, workspace, stream
    const at::Tensor& q = tensor(a[1]);
    const PlanRef plan(a[0], q.get_device());
    const Window w(plan.get(), q, a[1], a[2], a[3], a[4], plan->total_tokens, a[8], a[9], a[10]);
    return launch(lib.window, plan.get(), w.q.p, w.q.ld, w.k.p, w.k.ld, w.v.p, w.v.ld, w.kv_heads, w.hd, (float)real(a[5]),
                  (int32_t)integer(a[6], true), (int32_t)integer(a[7], true), w.out.p, w.out.ld, w.ws, w.ws_bytes, w.dt,
                  stream_on(a[11], w.dev));
}

// plan, q, k, v, kv_first, kv_len, max_kv_len, out, scale, window, sinks, kv_heads, head_dim, workspace, stream
PyObject* window_cached(PyObject* const* a) {
    const at::Tensor &q = tensor(a[1]), &k = tensor(a[2]);
    const PlanRef plan(a[0], q.get_device());
    need(k.dim() == 2);
    const Window w(plan.get(), q, a[1], a[2], a[3], a[7], k.size(0), a[11], a[12], a[13]);
    void *const first = vec(a[4], plan->batch, at::kLong, w.dev), *const len = vec(a[5], plan->batch, at::kInt, w.dev);
    return launch(lib.window_cached, plan.get(), w.q.p, w.q.ld, w.k.p, w.k.ld, w.v.p, w.v.ld, k.size(0), (int64_t*)first, (int32_t*)len,
                  (int32_t)integer(a[6], true), w.kv_heads, w.hd, (float)real(a[8]), (int32_t)integer(a[9], true),
                  (int32_t)integer(a[10], true), w.out.p, w.out.ld, w.ws, w.ws_bytes, w.dt, stream_on(a[14], w.dev));
}

// f's result, or None where an argument is not as documented
template <PyObject* (*f)(PyObject* const*), Py_ssize_t n>
PyObject* call(PyObject*, PyObject* const* args, Py_ssize_t got) {
    if (got != n) return PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", n, got);
    try {
        need(current_device != nullptr);  // (bound)
        return f(args);
    } catch (...) {  // (NotPlain, or torch's own error)
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// torch's current device and raw stream functions, then the C functions' addresses in the order of `lib`
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    constexpr Py_ssize_t kFunctions = sizeof(lib) / sizeof(void*);
    if (n != 2 + kFunctions) return PyErr_Format(PyExc_TypeError, "%zd arguments, not %zd", 2 + kFunctions, n);
    void* f[kFunctions];
    for (Py_ssize_t i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsVoidPtr(args[2 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    lib = {(decltype(lib.rmsnorm))f[0], (decltype(lib.quantize_i8))f[1], (decltype(lib.linear_i8))f[2], (decltype(lib.rotary))f[3],
           (decltype(lib.window))f[4], (decltype(lib.window_cached))f[5]};
    for (Py_ssize_t i = 0; i < 2; ++i) Py_INCREF(args[i]);
    current_device = args[0];
    raw_stream = args[1];
    Py_RETURN_NONE;
}

#define FAST(name, fn) {name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(fn)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FAST("bind", bind),
                         FAST("packed_rmsnorm", (&call<rmsnorm, 9>)),
                         FAST("packed_quantize_i8", (&call<quantize_i8, 4>)),
                         FAST("packed_linear_i8", (&call<linear_i8, 9>)),
                         FAST("packed_rotary", (&call<rotary, 11>)),
                         FAST("ragged_attention_window", (&call<window, 12>)),
                         FAST("ragged_attention_window_cached", (&call<window_cached, 15>)),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() {
    name_c = PyUnicode_InternFromString("c");
    name_status = PyUnicode_InternFromString("status");
    name_stream = PyUnicode_InternFromString("cuda_stream");
    if (!name_c || !name_status || !name_stream) return nullptr;
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", RAG_BUILT_FOR) != 0) Py_CLEAR(m);
    return m;
}

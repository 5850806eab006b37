// The checks and the marshalling of binding.py's calls for deep networks, compiled: the smallest of these calls run a kernel of two microseconds, and
// checking six tensors and converting twelve arguments in the interpreter takes twice as long.  Every function takes binding.py's arguments
// (the optional ones too, and the stream last) and returns the library's status code, or -1 where an argument is not what the call takes;
// binding.py then checks again in its own way and says what is wrong.  The library's functions are handed over by address.
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <torch/csrc/autograd/python_variable.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>

#include "../../include/pcl_dnn.h"

namespace {

struct Functions {
    decltype(&pcl_rms_norm_fwd) rms_norm_fwd = nullptr;
    decltype(&pcl_rms_norm_fwd_q8) rms_norm_fwd_q8 = nullptr;
    decltype(&pcl_rms_norm_bwd) rms_norm_bwd = nullptr;
    decltype(&pcl_quantize_rows) quantize_rows = nullptr;
    decltype(&pcl_fc_q8_fwd) fc_q8_fwd = nullptr;
    decltype(&pcl_grad_norm) grad_norm = nullptr;
    decltype(&pcl_grad_clip) grad_clip = nullptr;
    decltype(&pcl_sgd_update_clipped) sgd_update_clipped = nullptr;
    decltype(&pcl_sample_tokens) sample_tokens = nullptr;
} fn;

// Reads a call's arguments one after another; ok turns false at the first that is not what the call takes.
class Args {
  public:
    Args(PyObject* const* args, Py_ssize_t n, Py_ssize_t want) : args_(args), ok(n == want) {}
    // a size: 1 .. 2^31 - 1
    int size() {
        const long v = integer();
        if (ok && (v <= 0 || v > 2147483647L)) ok = false;
        return ok ? int(v) : 0;
    }
    long integer() {
        PyObject* o = next();
        if (!ok || !PyLong_CheckExact(o)) { ok = false; return 0; }
        int overflow = 0;
        const long v = PyLong_AsLongAndOverflow(o, &overflow);
        if (overflow) ok = false;
        return v;
    }
    float real() {
        PyObject* o = next();
        if (!ok || !(PyFloat_CheckExact(o) || PyLong_CheckExact(o))) { ok = false; return 0.f; }
        const double v = PyFloat_AsDouble(o);
        if (v == -1.0 && PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return float(v);
    }
    // tensors of n elements: of the type that the first one has (fp32, bf16, fp16); of a given type; of 8 bits.  optional: None is a null pointer.
    void* typed(int64_t n, bool optional = false) {
        const at::Tensor* t = tensor(n, optional);
        if (!t) return nullptr;
        if (dtype < 0) {
            first_ = t->scalar_type();
            dtype = first_ == at::kFloat ? PCL_F32 : first_ == at::kBFloat16 ? PCL_BF16 : first_ == at::kHalf ? PCL_F16 : -1;
            if (dtype < 0) ok = false;
        }
        return of_type(t, first_);
    }
    template <class V>
    V* plain(at::ScalarType type, int64_t n, bool optional = false) {
        const at::Tensor* t = tensor(n, optional);
        return t ? static_cast<V*>(of_type(t, type)) : nullptr;
    }
    float* real32(int64_t n, bool optional = false) { return plain<float>(at::kFloat, n, optional); }
    int* int32(int64_t n, bool optional = false) { return plain<int>(at::kInt, n, optional); }
    void* bytes(int64_t n) {
        const at::Tensor* t = tensor(n, false);
        if (!t) return nullptr;
        return of_type(t, t->scalar_type() == at::kByte ? at::kByte : at::kFloat8_e4m3fn);
    }
    struct Workspace { void* p; size_t bytes; };
    Workspace workspace() {
        const at::Tensor* t = tensor(-1, true);
        if (!t) return {nullptr, 0};
        return {of_type(t, t->scalar_type()), t->nbytes()};
    }
    // None: the current stream of the tensors' device, which has to be the current device
    void* stream() {
        PyObject* o = next();
        if (!ok) return nullptr;
        if (device < 0 || c10::cuda::current_device() != device) { ok = false; return nullptr; }
        if (o == Py_None) return c10::cuda::getCurrentCUDAStream(c10::DeviceIndex(device)).stream();
        PyObject* handle = PyObject_GetAttrString(o, "cuda_stream");
        void* s = handle ? PyLong_AsVoidPtr(handle) : nullptr;
        Py_XDECREF(handle);
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        return s;
    }
    template <class P> P address() { return reinterpret_cast<P>(integer()); }

  private:
    PyObject* const* args_;
    Py_ssize_t at_ = 0;
    at::ScalarType first_ = at::kFloat;
    PyObject* next() { return ok ? args_[at_++] : nullptr; }
    const at::Tensor* tensor(int64_t n, bool optional) {
        PyObject* o = next();
        if (!ok || (optional && o == Py_None)) return nullptr;
        if (!THPVariable_Check(o)) { ok = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!t.defined() || t.layout() != at::kStrided || !t.is_cuda() || (n >= 0 && t.numel() != n) || !t.is_contiguous()) { ok = false; return nullptr; }
        const int d = t.get_device();
        if (device < 0) device = d;
        if (d != device) { ok = false; return nullptr; }
        return &t;
    }
    void* of_type(const at::Tensor* t, at::ScalarType type) {
        if (t->scalar_type() != type) { ok = false; return nullptr; }
        return t->data_ptr();
    }

  public:
    bool ok;
    int dtype = -1, device = -1;
};

// The library's call, with the interpreter free for other threads: a launch waits where a stream's queue is full, maybe for a host function that
// needs the interpreter.  (The tensors are the caller's arguments, who holds them.)
template <class F>
int unlocked(F&& call) {
    int code;
    Py_BEGIN_ALLOW_THREADS
    code = call();
    Py_END_ALLOW_THREADS
    return code;
}

template <class F>
PyObject* guarded(Args& a, F&& call) {
    try {
        const int code = call();
        return PyLong_FromLong(a.ok ? code : -1);
    } catch (...) {                                            // (of torch: the call is not made, and the interpreter's checks say why)
        return PyLong_FromLong(-1);
    }
}

PyObject* rms_norm_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 10);
    return guarded(a, [&]() -> int {
        const int N = a.size(), C = a.size();
        const int64_t all = int64_t(N) * C;
        void* x = a.typed(all);
        void* res = a.typed(all, true);
        void* w = a.typed(C);
        const float eps = a.real();
        void* h = a.typed(all, true);
        void* y = a.typed(all);
        float* rstd = a.real32(N, true);
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.rms_norm_fwd(N, C, a.dtype, x, res, w, eps, h, y, rstd, st); }) : -1;
    });
}

PyObject* rms_norm_fwd_q8(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 11);
    return guarded(a, [&]() -> int {
        const int N = a.size(), C = a.size();
        const int64_t all = int64_t(N) * C;
        void* x = a.typed(all);
        void* res = a.typed(all, true);
        void* w = a.typed(C);
        const float eps = a.real();
        void* h = a.typed(all, true);
        void* y = a.bytes(all);
        float* scale = a.real32(N);
        float* rstd = a.real32(N, true);
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.rms_norm_fwd_q8(N, C, a.dtype, x, res, w, eps, h, y, scale, rstd, st); }) : -1;
    });
}

PyObject* rms_norm_bwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 11);
    return guarded(a, [&]() -> int {
        const int N = a.size(), C = a.size();
        const int64_t all = int64_t(N) * C;
        void* h = a.typed(all);
        void* w = a.typed(C);
        float* rstd = a.real32(N);
        void* dy = a.typed(all);
        void* dh = a.typed(all, true);
        void* dx = a.typed(all);
        void* dw = a.typed(C, true);
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.rms_norm_bwd(N, C, a.dtype, h, w, rstd, dy, dh, dx, dw, ws.p, ws.bytes, st); }) : -1;
    });
}

PyObject* quantize_rows(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 6);
    return guarded(a, [&]() -> int {
        const int N = a.size(), C = a.size();
        const int64_t all = int64_t(N) * C;
        void* x = a.typed(all);
        void* q = a.bytes(all);
        float* scale = a.real32(N);
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.quantize_rows(N, C, a.dtype, x, q, scale, st); }) : -1;
    });
}

PyObject* fc_q8_fwd(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 12);
    return guarded(a, [&]() -> int {
        const int N = a.size(), C = a.size(), K = a.size();
        void* y = a.typed(int64_t(N) * K);
        void* bias = a.typed(K, true);
        void* x = a.bytes(int64_t(N) * C);
        float* xs = a.real32(N);
        void* w = a.bytes(int64_t(K) * C);
        float* ws_ = a.real32(K);
        const long act = a.integer();
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.fc_q8_fwd(N, C, K, a.dtype, x, xs, w, ws_, bias, y, int(act), ws.p, ws.bytes, st); }) : -1;
    });
}

PyObject* sample_tokens(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 12);
    return guarded(a, [&]() -> int {
        const int N = a.size(), K = a.size();
        void* z = a.typed(int64_t(N) * K);
        float* u = a.real32(N);
        int* token = a.int32(N);
        float* temperature = a.real32(N, true);
        int* top_k = a.int32(N, true);
        float* top_p = a.real32(N, true);
        float* min_p = a.real32(N, true);
        float* logprob = a.real32(N, true);
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.sample_tokens(N, K, a.dtype, z, u, temperature, top_k, top_p, min_p, token, logprob, ws.p, ws.bytes, st); }) : -1;
    });
}

// The lists' addresses (host arrays that their TensorList keeps) come as integers, with the device of their tensors.
PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 8);
    return guarded(a, [&]() -> int {
        a.device = int(a.integer());
        const int count = a.size();
        const auto grads = a.address<const void* const*>();
        const auto sizes = a.address<const size_t*>();
        const auto types = a.address<const int*>();
        float* norm = a.real32(1);
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.grad_norm(count, grads, sizes, types, norm, ws.p, ws.bytes, st); }) : -1;
    });
}

PyObject* grad_clip(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 10);
    return guarded(a, [&]() -> int {
        a.device = int(a.integer());
        const int count = a.size();
        const auto grads = a.address<const void* const*>();
        const auto out = a.address<void* const*>();
        const auto sizes = a.address<const size_t*>();
        const auto types = a.address<const int*>();
        const float most = a.real();
        float* norm = a.real32(1);
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.grad_clip(count, grads, out, sizes, types, most, norm, ws.p, ws.bytes, st); }) : -1;
    });
}

PyObject* sgd_update_clipped(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 11);
    return guarded(a, [&]() -> int {
        a.device = int(a.integer());
        const int count = a.size();
        const auto w = a.address<void* const*>();
        const auto grads = a.address<const void* const*>();
        const auto sizes = a.address<const size_t*>();
        const auto types = a.address<const int*>();
        const float lr = a.real(), most = a.real();
        float* norm = a.real32(1);
        const Args::Workspace ws = a.workspace();
        void* st = a.stream();
        return a.ok ? unlocked([&] { return fn.sgd_update_clipped(count, w, grads, sizes, types, lr, most, norm, ws.p, ws.bytes, st); }) : -1;
    });
}

// bind({name: address}): the library's functions
PyObject* bind(PyObject*, PyObject* table) {
    struct { const char* name; void** to; } const all[] = {
        {"pcl_rms_norm_fwd", reinterpret_cast<void**>(&fn.rms_norm_fwd)}, {"pcl_rms_norm_fwd_q8", reinterpret_cast<void**>(&fn.rms_norm_fwd_q8)},
        {"pcl_rms_norm_bwd", reinterpret_cast<void**>(&fn.rms_norm_bwd)}, {"pcl_quantize_rows", reinterpret_cast<void**>(&fn.quantize_rows)},
        {"pcl_fc_q8_fwd", reinterpret_cast<void**>(&fn.fc_q8_fwd)}, {"pcl_grad_norm", reinterpret_cast<void**>(&fn.grad_norm)},
        {"pcl_grad_clip", reinterpret_cast<void**>(&fn.grad_clip)}, {"pcl_sgd_update_clipped", reinterpret_cast<void**>(&fn.sgd_update_clipped)},
        {"pcl_sample_tokens", reinterpret_cast<void**>(&fn.sample_tokens)}};
    if (!PyDict_Check(table)) { PyErr_SetString(PyExc_TypeError, "a dict of addresses is wanted"); return nullptr; }
    for (const auto& f : all) {
        PyObject* v = PyDict_GetItemString(table, f.name);
        void* p = v ? PyLong_AsVoidPtr(v) : nullptr;
        if (!p) {
            if (!PyErr_Occurred()) PyErr_Format(PyExc_ValueError, "no address of %s", f.name);
            return nullptr;
        }
        *f.to = p;
    }
    Py_RETURN_NONE;
}

#define PCL_FAST(name) {#name, reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(name)), METH_FASTCALL, nullptr}
PyMethodDef methods[] = {{"bind", bind, METH_O, nullptr}, PCL_FAST(rms_norm_fwd), PCL_FAST(rms_norm_fwd_q8), PCL_FAST(rms_norm_bwd), PCL_FAST(quantize_rows),
                         PCL_FAST(fc_q8_fwd), PCL_FAST(sample_tokens), PCL_FAST(grad_norm), PCL_FAST(grad_clip), PCL_FAST(sgd_update_clipped),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_pcl_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__pcl_calls() {
    PyObject* m = PyModule_Create(&module);
    if (m && PyModule_AddStringConstant(m, "built_for", PCL_BUILT_FOR) < 0) { Py_DECREF(m); return nullptr; }
    return m;
}

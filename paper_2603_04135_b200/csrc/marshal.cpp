// Argument marshalling of the scoring calls for the Python binding: the plain case (torch tensors, laid out as the call
// reads them) in native code.  What a call of a few microseconds on the device costs on the host is mostly the look at nine
// tensors through Python (3.5 us of 7); here it is a tenth of that.
//
// Each function takes the params object and the call's arguments in the order of binding.py, checks every tensor (exact
// torch.Tensor, element type, on the current device, dense or with the stated row pitch, large enough) and calls the
// library on the current stream.  It returns the library's return code, or None if anything is not the plain case: the
// binding then goes through its own checks, which name what is wrong.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "dppo.h"

namespace {

PyTypeObject *g_logprob_type, *g_quantize_type, *g_linear_type;
decltype(&dppo_token_logprobs) g_logprobs;
decltype(&dppo_token_logprobs_backward) g_backward;
decltype(&dppo_quantize_rows_i8) g_quantize;
decltype(&dppo_linear_i8) g_linear;

struct NotPlain {};

// The params structure behind a ctypes object of type `type`.
template <class P> P params_of(PyObject* o, PyTypeObject* type) {
    if (Py_TYPE(o) != type) throw NotPlain();
    Py_buffer b;
    if (PyObject_GetBuffer(o, &b, PyBUF_SIMPLE) != 0) { PyErr_Clear(); throw NotPlain(); }
    if (b.len != (Py_ssize_t)sizeof(P)) { PyBuffer_Release(&b); throw NotPlain(); }
    const P p = *static_cast<const P*>(b.buf);
    PyBuffer_Release(&b);
    return p;
}

const at::Tensor& tensor_of(PyObject* o, at::ScalarType type, int device) {
    if ((PyObject*)Py_TYPE(o) != THPVariableClass) throw NotPlain();
    const at::Tensor& x = THPVariable_Unpack(o);
    if (x.scalar_type() != type || !x.is_cuda() || x.get_device() != device) throw NotPlain();
    return x;
}
// n dense elements.
template <class T> T* dense(PyObject* o, at::ScalarType type, int device, int64_t n) {
    if (o == Py_None) return nullptr;
    const at::Tensor& x = tensor_of(o, type, device);
    if (x.numel() < n || !x.is_contiguous()) throw NotPlain();
    return static_cast<T*>(x.data_ptr());
}
// `rows` whole rows of a matrix with `stride` elements between rows.
void* matrix(PyObject* o, at::ScalarType type, int device, int64_t rows, int64_t stride) {
    if (o == Py_None) return nullptr;
    const at::Tensor& x = tensor_of(o, type, device);
    if (x.dim() != 2 || x.stride(0) != stride || x.stride(1) != 1 || x.size(1) > stride || rows < 0 || stride < 0 ||
        x.size(0) < rows || (rows > 0 && x.size(1) < stride))
        throw NotPlain();
    return x.data_ptr();
}
at::ScalarType element(int dtype) {
    if (dtype == DPPO_BF16) return at::kBFloat16;
    if (dtype == DPPO_F32) return at::kFloat;
    throw NotPlain();
}

// Runs `call` (which checks its arguments, then returns a closure over plain pointers) and the closure without the
// interpreter's lock: a launch may block while the device's queue is full.
template <class F> PyObject* guarded(PyObject* const* args, Py_ssize_t n, Py_ssize_t want, F call) {
    if (n != want || args[want - 1] != Py_None) Py_RETURN_NONE;          // the last one is the stream: the current one
    int rc;
    try {
        const int device = c10::cuda::current_device();
        void* stream = c10::cuda::getCurrentCUDAStream(device).stream();
        auto go = call(device, stream);
        Py_BEGIN_ALLOW_THREADS
        rc = go();
        Py_END_ALLOW_THREADS
    } catch (...) {                                                       // NotPlain, or torch's own refusal of a tensor
        Py_RETURN_NONE;
    }
    return PyLong_FromLong(rc);
}

PyObject* token_logprobs(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 12, [&](int d, void* stream) {
        const auto p = params_of<dppo_logprob_params>(a[0], g_logprob_type);
        const int64_t T = p.T_max, k = T * p.top_k;
        const void* logits = matrix(a[1], element(p.dtype), d, T, p.row_stride);
        const auto* target = dense<int32_t>(a[2], at::kInt, d, T);
        const auto* n_dev = dense<int32_t>(a[3], at::kInt, d, 1);
        auto *logp = dense<float>(a[4], at::kFloat, d, T), *entropy = dense<float>(a[5], at::kFloat, d, T);
        auto *lse = dense<float>(a[6], at::kFloat, d, T), *top_logp = dense<float>(a[8], at::kFloat, d, k);
        auto *ids = dense<int32_t>(a[7], at::kInt, d, k), *status = dense<int32_t>(a[10], at::kInt, d, 1);
        auto* stats = dense<float>(a[9], at::kFloat, d, 4 * T);
        return [=] { return g_logprobs(&p, logits, target, n_dev, logp, entropy, lse, ids, top_logp, stats, status, stream); };
    });
}

PyObject* token_logprobs_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [&](int d, void* stream) {
        const auto p = params_of<dppo_logprob_params>(a[0], g_logprob_type);
        const int64_t T = p.T_max;
        const void* logits = matrix(a[1], element(p.dtype), d, T, p.row_stride);
        const auto* target = dense<int32_t>(a[2], at::kInt, d, T);
        const auto* n_dev = dense<int32_t>(a[3], at::kInt, d, 1);
        const auto *stats = dense<float>(a[4], at::kFloat, d, 4 * T), *dlogp = dense<float>(a[5], at::kFloat, d, T);
        const auto* dentropy = dense<float>(a[6], at::kFloat, d, T);
        void* dlogits = matrix(a[7], element(p.dtype), d, T, p.row_stride);
        auto* status = dense<int32_t>(a[8], at::kInt, d, 1);
        return [=] { return g_backward(&p, logits, target, n_dev, stats, dlogp, dentropy, dlogits, status, stream); };
    });
}

PyObject* quantize_rows_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 7, [&](int d, void* stream) {
        const auto p = params_of<dppo_quantize_params>(a[0], g_quantize_type);
        const void* x = matrix(a[1], element(p.dtype), d, p.rows_max, p.x_stride);
        auto* q = static_cast<int8_t*>(matrix(a[2], at::kChar, d, p.rows_max, p.q_stride));
        auto* scale = dense<float>(a[3], at::kFloat, d, p.rows_max);
        const auto* n_dev = dense<int32_t>(a[4], at::kInt, d, 1);
        auto* status = dense<int32_t>(a[5], at::kInt, d, 1);
        return [=] { return g_quantize(&p, x, q, scale, n_dev, status, stream); };
    });
}

PyObject* linear_i8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 9, [&](int d, void* stream) {
        const auto p = params_of<dppo_linear_i8_params>(a[0], g_linear_type);
        const auto* x = static_cast<const int8_t*>(matrix(a[1], at::kChar, d, p.M_max, p.x_stride));
        const auto* xs = dense<float>(a[2], at::kFloat, d, p.M_max);
        const auto* w = static_cast<const int8_t*>(matrix(a[3], at::kChar, d, p.N, p.w_stride));
        const auto* ws = dense<float>(a[4], at::kFloat, d, p.N);
        void* out = matrix(a[5], element(p.out_dtype), d, p.M_max, p.out_stride);
        const auto* n_dev = dense<int32_t>(a[6], at::kInt, d, 1);
        auto* status = dense<int32_t>(a[7], at::kInt, d, 1);
        return [=] { return g_linear(&p, x, xs, w, ws, out, n_dev, status, stream); };
    });
}

// bind(LogprobParams, QuantizeParams, LinearI8Params, addresses of the four entry points in the order above)
PyObject* bind(PyObject*, PyObject* args) {
    unsigned long long f[4];
    PyObject *a, *b, *c;
    if (!PyArg_ParseTuple(args, "O!O!O!KKKK", &PyType_Type, &a, &PyType_Type, &b, &PyType_Type, &c, &f[0], &f[1], &f[2], &f[3])) return nullptr;
    Py_INCREF(a); Py_INCREF(b); Py_INCREF(c);
    g_logprob_type = (PyTypeObject*)a; g_quantize_type = (PyTypeObject*)b; g_linear_type = (PyTypeObject*)c;
    g_logprobs = reinterpret_cast<decltype(g_logprobs)>(f[0]);
    g_backward = reinterpret_cast<decltype(g_backward)>(f[1]);
    g_quantize = reinterpret_cast<decltype(g_quantize)>(f[2]);
    g_linear = reinterpret_cast<decltype(g_linear)>(f[3]);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"token_logprobs", (PyCFunction)(void (*)(void))token_logprobs, METH_FASTCALL, nullptr},
    {"token_logprobs_backward", (PyCFunction)(void (*)(void))token_logprobs_backward, METH_FASTCALL, nullptr},
    {"quantize_rows_i8", (PyCFunction)(void (*)(void))quantize_rows_i8, METH_FASTCALL, nullptr},
    {"linear_i8", (PyCFunction)(void (*)(void))linear_i8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the interpreter and torch whose layouts this code relies on; the binding uses it with no other.
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject* m = PyModule_Create(&kModule);
    if (m && PyModule_AddStringConstant(m, "built_for", DPPO_BUILT_FOR) != 0) { Py_DECREF(m); return nullptr; }
    return m;
}

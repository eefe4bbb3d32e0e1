// Argument marshalling of the scoring, distillation and verification calls and the 8-bit products for the Python binding: the plain case
// (torch tensors, laid out as the call reads them) in native code.  What a call of a few microseconds on the device costs on the host is mostly the look at nine
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

// The params classes and the library's entry points, in the order of bind()'s arguments.
enum { kLogprob, kQuantize, kLinear, kDistill, kVerify, kQuantizeF8, kLinearF8, kTypes };
PyTypeObject* g_type[kTypes];
decltype(&dppo_token_logprobs) g_logprobs;
decltype(&dppo_token_logprobs_backward) g_backward;
decltype(&dppo_quantize_rows_i8) g_quantize;
decltype(&dppo_linear_i8) g_linear;
decltype(&dppo_distill_topk) g_distill;
decltype(&dppo_distill_topk_backward) g_distill_backward;
decltype(&dppo_verify_drafts) g_verify;
decltype(&dppo_quantize_f8) g_quantize_f8;
decltype(&dppo_linear_f8) g_linear_f8;
constexpr int kFunctions = 9;

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
        const auto p = params_of<dppo_logprob_params>(a[0], g_type[kLogprob]);
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
        const auto p = params_of<dppo_logprob_params>(a[0], g_type[kLogprob]);
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
        const auto p = params_of<dppo_quantize_params>(a[0], g_type[kQuantize]);
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
        const auto p = params_of<dppo_linear_i8_params>(a[0], g_type[kLinear]);
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

PyObject* distill_topk(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 12, [&](int d, void* stream) {
        const auto p = params_of<dppo_distill_params>(a[0], g_type[kDistill]);
        const int64_t T = p.T_max, k = T * p.top_k;
        const void* logits = matrix(a[1], element(p.dtype), d, T, p.row_stride);
        const auto* ids = dense<int32_t>(a[2], at::kInt, d, k);
        const auto *top_logp = dense<float>(a[3], at::kFloat, d, k), *weight = dense<float>(a[5], at::kFloat, d, T);
        const auto* n_dev = dense<int32_t>(a[4], at::kInt, d, 1);
        auto *loss = dense<float>(a[6], at::kFloat, d, T), *lse = dense<float>(a[7], at::kFloat, d, T), *stats = dense<float>(a[8], at::kFloat, d, 4 * T);
        void* dlogits = matrix(a[9], element(p.dtype), d, T, p.row_stride);
        auto* status = dense<int32_t>(a[10], at::kInt, d, 1);
        return [=] { return g_distill(&p, logits, ids, top_logp, n_dev, weight, loss, lse, stats, dlogits, status, stream); };
    });
}

PyObject* distill_topk_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 10, [&](int d, void* stream) {
        const auto p = params_of<dppo_distill_params>(a[0], g_type[kDistill]);
        const int64_t T = p.T_max, k = T * p.top_k;
        const void* logits = matrix(a[1], element(p.dtype), d, T, p.row_stride);
        const auto* ids = dense<int32_t>(a[2], at::kInt, d, k);
        const auto* top_logp = dense<float>(a[3], at::kFloat, d, k);
        const auto* n_dev = dense<int32_t>(a[4], at::kInt, d, 1);
        const auto *stats = dense<float>(a[5], at::kFloat, d, 4 * T), *dloss = dense<float>(a[6], at::kFloat, d, T);
        void* dlogits = matrix(a[7], element(p.dtype), d, T, p.row_stride);
        auto* status = dense<int32_t>(a[8], at::kInt, d, 1);
        return [=] { return g_distill_backward(&p, logits, ids, top_logp, n_dev, stats, dloss, dlogits, status, stream); };
    });
}

PyObject* verify_drafts(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 14, [&](int d, void* stream) {
        const auto p = params_of<dppo_verify_params>(a[0], g_type[kVerify]);
        const int64_t T = p.T_max, B = p.n_seqs;
        const void* target = matrix(a[1], element(p.dtype), d, T + B, p.target_stride);
        const void* draft = matrix(a[2], element(p.dtype), d, T, p.draft_stride);
        const auto *drafts = dense<int32_t>(a[3], at::kInt, d, T), *cu = dense<int32_t>(a[4], at::kInt, d, B + 1);
        const auto* u = dense<float>(a[5], at::kFloat, d, T);
        const auto* noise = static_cast<const float*>(matrix(a[6], at::kFloat, d, B, p.noise_stride));
        auto *n_acc = dense<int32_t>(a[7], at::kInt, d, B), *tokens = dense<int32_t>(a[8], at::kInt, d, T + B);
        auto* logp = dense<float>(a[9], at::kFloat, d, T + B);
        const int64_t bytes = PyLong_AsLongLong(a[11]);
        if (bytes < 0) { PyErr_Clear(); throw NotPlain(); }
        auto* ws = dense<uint8_t>(a[10], at::kByte, d, bytes);
        auto* status = dense<int32_t>(a[12], at::kInt, d, 1);
        return [=] { return g_verify(&p, target, draft, drafts, cu, u, noise, n_acc, tokens, logp, ws, (size_t)bytes, status, stream); };
    });
}

PyObject* quantize_f8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 7, [&](int d, void* stream) {
        const auto p = params_of<dppo_quantize_f8_params>(a[0], g_type[kQuantizeF8]);
        const int64_t blocks = (p.K + 127ll) / 128;
        const void* x = matrix(a[1], element(p.dtype), d, p.rows_max, p.x_stride);
        auto* q = static_cast<uint8_t*>(matrix(a[2], at::kFloat8_e4m3fn, d, p.rows_max, p.q_stride));
        auto* scale = static_cast<float*>(matrix(a[3], at::kFloat, d, p.block_rows == 1 ? blocks : (p.rows_max + 127) / 128, p.scale_stride));
        const auto* n_dev = dense<int32_t>(a[4], at::kInt, d, 1);
        auto* status = dense<int32_t>(a[5], at::kInt, d, 1);
        return [=] { return g_quantize_f8(&p, x, q, scale, n_dev, status, stream); };
    });
}

PyObject* linear_f8(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded(a, n, 9, [&](int d, void* stream) {
        const auto p = params_of<dppo_linear_f8_params>(a[0], g_type[kLinearF8]);
        const auto* x = static_cast<const uint8_t*>(matrix(a[1], at::kFloat8_e4m3fn, d, p.M_max, p.x_stride));
        const auto* xs = static_cast<const float*>(matrix(a[2], at::kFloat, d, (p.K + 127ll) / 128, p.x_scale_stride));
        const auto* w = static_cast<const uint8_t*>(matrix(a[3], at::kFloat8_e4m3fn, d, p.N, p.w_stride));
        const auto* ws = static_cast<const float*>(matrix(a[4], at::kFloat, d, (p.N + 127ll) / 128, p.w_scale_stride));
        void* out = matrix(a[5], element(p.out_dtype), d, p.M_max, p.out_stride);
        const auto* n_dev = dense<int32_t>(a[6], at::kInt, d, 1);
        auto* status = dense<int32_t>(a[7], at::kInt, d, 1);
        return [=] { return g_linear_f8(&p, x, xs, w, ws, out, n_dev, status, stream); };
    });
}

// bind(params classes, addresses of the entry points), each a tuple in the order above
PyObject* bind(PyObject*, PyObject* args) {
    PyObject *types, *functions;
    if (!PyArg_ParseTuple(args, "O!O!", &PyTuple_Type, &types, &PyTuple_Type, &functions)) return nullptr;
    if (PyTuple_GET_SIZE(types) != kTypes || PyTuple_GET_SIZE(functions) != kFunctions) {
        PyErr_SetString(PyExc_ValueError, "bind: another number of classes or functions");
        return nullptr;
    }
    unsigned long long f[kFunctions];
    for (int i = 0; i < kFunctions; ++i) {
        f[i] = PyLong_AsUnsignedLongLong(PyTuple_GET_ITEM(functions, i));
        if (PyErr_Occurred()) return nullptr;
    }
    for (int i = 0; i < kTypes; ++i) {
        PyObject* t = PyTuple_GET_ITEM(types, i);
        Py_INCREF(t);
        g_type[i] = (PyTypeObject*)t;
    }
    g_logprobs = reinterpret_cast<decltype(g_logprobs)>(f[0]);
    g_backward = reinterpret_cast<decltype(g_backward)>(f[1]);
    g_quantize = reinterpret_cast<decltype(g_quantize)>(f[2]);
    g_linear = reinterpret_cast<decltype(g_linear)>(f[3]);
    g_distill = reinterpret_cast<decltype(g_distill)>(f[4]);
    g_distill_backward = reinterpret_cast<decltype(g_distill_backward)>(f[5]);
    g_verify = reinterpret_cast<decltype(g_verify)>(f[6]);
    g_quantize_f8 = reinterpret_cast<decltype(g_quantize_f8)>(f[7]);
    g_linear_f8 = reinterpret_cast<decltype(g_linear_f8)>(f[8]);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"bind", bind, METH_VARARGS, nullptr},
    {"token_logprobs", (PyCFunction)(void (*)(void))token_logprobs, METH_FASTCALL, nullptr},
    {"token_logprobs_backward", (PyCFunction)(void (*)(void))token_logprobs_backward, METH_FASTCALL, nullptr},
    {"quantize_rows_i8", (PyCFunction)(void (*)(void))quantize_rows_i8, METH_FASTCALL, nullptr},
    {"linear_i8", (PyCFunction)(void (*)(void))linear_i8, METH_FASTCALL, nullptr},
    {"distill_topk", (PyCFunction)(void (*)(void))distill_topk, METH_FASTCALL, nullptr},
    {"distill_topk_backward", (PyCFunction)(void (*)(void))distill_topk_backward, METH_FASTCALL, nullptr},
    {"verify_drafts", (PyCFunction)(void (*)(void))verify_drafts, METH_FASTCALL, nullptr},
    {"quantize_f8", (PyCFunction)(void (*)(void))quantize_f8, METH_FASTCALL, nullptr},
    {"linear_f8", (PyCFunction)(void (*)(void))linear_f8, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

// built_for: the interpreter and torch whose layouts this code relies on; the binding uses it with no other.
PyMODINIT_FUNC PyInit__marshal(void) {
    PyObject* m = PyModule_Create(&kModule);
    if (m && PyModule_AddStringConstant(m, "built_for", DPPO_BUILT_FOR) != 0) { Py_DECREF(m); return nullptr; }
    return m;
}

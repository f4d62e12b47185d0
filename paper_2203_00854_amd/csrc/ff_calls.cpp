// _calls: the training operators' entry points for torch tensors, as a CPython module beside libff.so.
//
// The kernels of a small call take 3 us, a ctypes call that allocates its results from Python 12 to 15.  Here the checks, the allocations and the C call
// are one step, which takes 6 to 8, with the interpreter lock let go.  The functions take every argument by place (binding.py holds the
// signatures and defaults) and return the results, or ff_status as a number where the library refuses the call.
#include <Python.h>

#include <algorithm>

#include <ATen/ATen.h>
#include <c10/core/DeviceGuard.h>
#include <c10/hip/HIPCachingAllocator.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "ff.h"

namespace {

// an argument that no kernel may see: raised as TypeError or ValueError
struct Refused {
    PyObject* error;
    std::string text;
};
template <typename... A> [[noreturn]] void type_error(const A&... a) { throw Refused{PyExc_TypeError, c10::str(a...)}; }
template <typename... A> [[noreturn]] void value_error(const A&... a) { throw Refused{PyExc_ValueError, c10::str(a...)}; }

at::Tensor optional(PyObject* o, const char* name) {
    if (o == Py_None) return {};
    if (!THPVariable_Check(o)) type_error(name, " is a ", Py_TYPE(o)->tp_name, ", not a tensor");
    return THPVariable_Unpack(o);
}
at::Tensor tensor(PyObject* o, const char* name) {
    if (o == Py_None) type_error(name, " is missing");
    return optional(o, name);
}
// t as the kernels take it: this type and shape, dense, on this GPU
void fit(const at::Tensor& t, const char* name, at::ScalarType dtype, at::IntArrayRef shape, at::Device device) {
    if (t.scalar_type() != dtype) type_error(name, " is ", t.scalar_type(), ", not ", dtype);
    if (t.device() != device) value_error(name, " is on ", t.device(), ", not on ", device);
    if (!t.is_contiguous()) value_error(name, " is not contiguous");
    if (t.sizes() != shape) value_error(name, " has shape ", t.sizes(), ", not ", shape);
}
void fit_optional(const at::Tensor& t, const char* name, at::ScalarType dtype, at::IntArrayRef shape, at::Device device) {
    if (t.defined()) fit(t, name, dtype, shape, device);
}
// the given result tensor, checked, or a new one
void result(at::Tensor& t, const char* name, at::ScalarType dtype, at::IntArrayRef shape, at::Device device) {
    if (t.defined()) fit(t, name, dtype, shape, device);
    else t = at::empty(shape, at::TensorOptions().dtype(dtype).device(device));
}
const void* in(const at::Tensor& t) { return t.defined() ? t.const_data_ptr() : nullptr; }
template <typename T = void> T* out(const at::Tensor& t) { return t.defined() ? (T*)t.mutable_data_ptr() : nullptr; }

// Memory that the binding has allocated for one stream (`own`) and another one still reads: the allocator is told, and does not hand it out before.
void in_use(const at::Tensor& t, const c10::hip::HIPStream& stream, void* own) {
    if (stream.stream() != own) c10::hip::HIPCachingAllocator::recordStream(t.storage().data_ptr(), stream);
}

struct Unlocked {                      // without the interpreter lock
    PyThreadState* state = PyEval_SaveThread();
    ~Unlocked() { PyEval_RestoreThread(state); }
};

struct Norm {
    ff_norm_desc desc;
    at::ScalarType dtype;
    at::Device device;
    at::IntArrayRef shape, rows, channels;
    Norm(const at::Tensor& x, const at::Tensor& gamma, double eps) : dtype(x.scalar_type()), device(x.device()), shape(x.sizes()) {
        if (shape.empty() || shape.back() < 1) value_error("no channels in shape ", shape);
        if (!x.is_cuda()) value_error("x is on ", device, ", not on a GPU");
        if (!x.is_contiguous()) value_error("x is not contiguous");
        rows = shape.slice(0, shape.size() - 1);
        channels = shape.slice(shape.size() - 1);
        fit(gamma, "gamma", dtype, channels, device);
        if (dtype != at::kFloat && dtype != at::kBFloat16) type_error("unsupported dtype ", dtype);
        if (channels[0] > INT32_MAX) value_error("too many channels in shape ", shape);
        desc = ff_norm_desc{dtype == at::kFloat ? FF_F32 : FF_BF16, (int32_t)channels[0], x.numel() / channels[0], (float)eps};
    }
};

// C++ errors become Python's at the module's edge
template <typename F> PyObject* guarded(const char* name, Py_ssize_t want, Py_ssize_t given, F body) {
    HANDLE_TH_ERRORS
    if (given != want) return PyErr_Format(PyExc_TypeError, "%s takes %zd arguments, not %zd", name, want, given);
    try {
        return body();
    } catch (const Refused& r) {
        PyErr_SetString(r.error, r.text.c_str());
        return nullptr;
    }
    END_HANDLE_TH_ERRORS
}

// a tuple of tensors, None for those that are none
template <typename... T> PyObject* tuple_of(const T&... t) {
    PyObject* all = PyTuple_New(sizeof...(t));
    Py_ssize_t i = 0;
    if (all) (PyTuple_SET_ITEM(all, i++, t.defined() ? THPVariable_Wrap(t) : Py_NewRef(Py_None)), ...);
    return all;
}

// x, gamma, beta, residual, eps, stats, out, sum_out -> (y, sum, mean, rstd)
PyObject* layernorm_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("layernorm_forward", 8, n, [&]() -> PyObject* {
        const at::Tensor x = tensor(a[0], "x"), gamma = tensor(a[1], "gamma"), beta = tensor(a[2], "beta"), residual = optional(a[3], "residual");
        const double eps = PyFloat_AsDouble(a[4]);
        const int stats = PyObject_IsTrue(a[5]);
        if (PyErr_Occurred()) return nullptr;
        at::Tensor y = optional(a[6], "out"), sum = optional(a[7], "sum_out"), mean, rstd;
        const Norm norm(x, gamma, eps);
        fit(beta, "beta", norm.dtype, norm.channels, norm.device);
        fit_optional(residual, "residual", norm.dtype, norm.shape, norm.device);
        if (sum.defined() && !residual.defined()) value_error("sum_out needs a residual");
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(norm.device);
            result(y, "out", norm.dtype, norm.shape, norm.device);
            if (residual.defined()) result(sum, "sum_out", norm.dtype, norm.shape, norm.device);
            if (stats) {
                result(mean, "mean", at::kFloat, norm.rows, norm.device);
                result(rstd, "rstd", at::kFloat, norm.rows, norm.device);
            }
            status = ff_layernorm_forward(&norm.desc, in(x), in(residual), in(gamma), in(beta), out(sum), out(y), out<float>(mean), out<float>(rstd),
                                          c10::hip::getCurrentHIPStream(norm.device.index()).stream());
        }
        return status == FF_OK ? tuple_of(y, sum, mean, rstd) : PyLong_FromLong(status);
    });
}

// s, gamma, dy, mean, rstd, dsum, eps, dx, dgamma, dbeta, accumulate, ws -> (dx, dgamma, dbeta)
PyObject* layernorm_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("layernorm_backward", 12, n, [&]() -> PyObject* {
        const at::Tensor s = tensor(a[0], "s"), gamma = tensor(a[1], "gamma"), dy = tensor(a[2], "dy"), mean = optional(a[3], "mean"),
                         rstd = optional(a[4], "rstd"), dsum = optional(a[5], "dsum");
        const double eps = PyFloat_AsDouble(a[6]);
        const int accumulate = PyObject_IsTrue(a[10]);
        if (PyErr_Occurred()) return nullptr;
        at::Tensor dx = optional(a[7], "dx"), dgamma = optional(a[8], "dgamma"), dbeta = optional(a[9], "dbeta"), ws = optional(a[11], "ws");
        const Norm norm(s, gamma, eps);
        fit(dy, "dy", norm.dtype, norm.shape, norm.device);
        fit_optional(dsum, "dsum", norm.dtype, norm.shape, norm.device);
        fit_optional(mean, "mean", at::kFloat, norm.rows, norm.device);
        fit_optional(rstd, "rstd", at::kFloat, norm.rows, norm.device);
        if (accumulate && !(dgamma.defined() && dbeta.defined())) value_error("accumulate needs dgamma and dbeta");
        if (ws.defined() && (ws.device() != norm.device || !ws.is_contiguous())) value_error("ws is on ", ws.device(), " or not contiguous");
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(norm.device);
            result(dx, "dx", norm.dtype, norm.shape, norm.device);
            result(dgamma, "dgamma", at::kFloat, norm.channels, norm.device);
            result(dbeta, "dbeta", at::kFloat, norm.channels, norm.device);
            if (!ws.defined()) ws = at::empty((int64_t)ff_layernorm_backward_workspace_bytes(&norm.desc), at::TensorOptions().dtype(at::kByte).device(norm.device));
            status = ff_layernorm_backward(&norm.desc, in(s), in(gamma), (const float*)in(mean), (const float*)in(rstd), in(dy), in(dsum), out(dx),
                                           out<float>(dgamma), out<float>(dbeta), accumulate, out(ws), ws.nbytes(),
                                           c10::hip::getCurrentHIPStream(norm.device.index()).stream());
        }
        return status == FF_OK ? tuple_of(dx, dgamma, dbeta) : PyLong_FromLong(status);
    });
}

// address of the plan's ff_adamw_desc, the plan, out, ws, the plan's stream -> norm
PyObject* grad_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("grad_norm", 5, n, [&]() -> PyObject* {
        const auto* desc = (const ff_adamw_desc*)PyLong_AsVoidPtr(a[0]);
        void* const own = PyLong_AsVoidPtr(a[4]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor plan = tensor(a[1], "plan"), ws = tensor(a[3], "ws");
        at::Tensor norm = optional(a[2], "out");
        const at::Device device = plan.device();
        if (ws.device() != device || !ws.is_contiguous()) value_error("ws is on ", ws.device(), " or not contiguous");
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(device);
            result(norm, "out", at::kFloat, {1}, device);
            const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(device.index());
            status = ff_grad_norm(desc, in(plan), plan.nbytes(), out<float>(norm), out(ws), ws.nbytes(), stream.stream());
            in_use(plan, stream, own);
            in_use(ws, stream, own);
        }
        return status == FF_OK ? THPVariable_Wrap(norm) : PyLong_FromLong(status);
    });
}

// address of the plan's ff_adamw_desc, the plan, step, lr, beta1, beta2, eps, norm, max_norm, seed, the plan's stream -> status
PyObject* adamw_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("adamw_step", 11, n, [&]() -> PyObject* {
        const auto* desc = (const ff_adamw_desc*)PyLong_AsVoidPtr(a[0]);
        void* const own = PyLong_AsVoidPtr(a[10]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor plan = tensor(a[1], "plan"), norm = optional(a[7], "norm");
        if (norm.defined() != (a[8] != Py_None)) value_error("norm and max_norm are given together");
        const at::Device device = plan.device();
        fit_optional(norm, "norm", at::kFloat, {1}, device);
        ff_adamw_hyper h;
        h.step = PyLong_AsLongLong(a[2]);
        h.lr = PyFloat_AsDouble(a[3]);
        h.beta1 = PyFloat_AsDouble(a[4]);
        h.beta2 = PyFloat_AsDouble(a[5]);
        h.eps = PyFloat_AsDouble(a[6]);
        h.max_norm = norm.defined() ? PyFloat_AsDouble(a[8]) : 0.;
        h.seed = (uint32_t)PyLong_AsUnsignedLongLongMask(a[9]);
        if (PyErr_Occurred()) return nullptr;
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(device);
            const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(device.index());
            status = ff_adamw_step(desc, in(plan), plan.nbytes(), &h, (const float*)in(norm), stream.stream());
            in_use(plan, stream, own);
        }
        return PyLong_FromLong(status);
    });
}

// address of the plan's ff_adamw_desc, the plan, its values, m, v, the plan's stream -> (m, v)
PyObject* adamw_moments(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("adamw_moments", 6, n, [&]() -> PyObject* {
        const auto* desc = (const ff_adamw_desc*)PyLong_AsVoidPtr(a[0]);
        void* const own = PyLong_AsVoidPtr(a[5]);
        if (PyErr_Occurred()) return nullptr;
        const int64_t values = PyLong_AsLongLong(a[2]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor plan = tensor(a[1], "plan");
        at::Tensor m = optional(a[3], "m"), v = optional(a[4], "v");
        const at::Device device = plan.device();
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(device);
            result(m, "m", at::kFloat, {values}, device);
            result(v, "v", at::kFloat, {values}, device);
            const char *from_m = (const char*)in(m), *from_v = (const char*)in(v);
            if (from_m < from_v + v.nbytes() && from_v < from_m + m.nbytes()) value_error("m and v share memory");
            const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(device.index());
            status = ff_adamw_moments(desc, in(plan), plan.nbytes(), out<float>(m), out<float>(v), stream.stream());
            in_use(plan, stream, own);
        }
        return status == FF_OK ? tuple_of(m, v) : PyLong_FromLong(status);
    });
}

struct Transition {
    ff_transition_desc desc;
    at::ScalarType dtype;
    at::Device device;
    at::IntArrayRef shape, rows;
    int64_t in[2], back[2];                    // shapes of w_a and w_b, of w_o
    Transition(const at::Tensor& x, const at::Tensor& w_a, const at::Tensor& w_b, const at::Tensor& w_o, const at::Tensor& mask, long act)
        : dtype(x.scalar_type()), device(x.device()), shape(x.sizes()) {
        if (shape.empty() || shape.back() < 1) value_error("no channels in shape ", shape);
        if (!x.is_cuda()) value_error("x is on ", device, ", not on a GPU");
        if (!x.is_contiguous()) value_error("x is not contiguous");
        if (dtype != at::kFloat && dtype != at::kBFloat16) type_error("unsupported dtype ", dtype);
        if (w_a.dim() != 2 || w_a.size(0) < 1) value_error("w_a has shape ", w_a.sizes(), ", not [hidden channels, channels]");
        rows = shape.slice(0, shape.size() - 1);
        in[0] = back[1] = w_a.size(0);
        in[1] = back[0] = shape.back();
        if (in[0] > INT32_MAX || in[1] > INT32_MAX) value_error("too many channels in shapes ", shape, " and ", w_a.sizes());
        fit(w_a, "w_a", dtype, in, device);
        fit(w_b, "w_b", dtype, in, device);
        fit(w_o, "w_o", dtype, back, device);
        fit_optional(mask, "mask", at::kFloat, rows, device);
        desc = ff_transition_desc{dtype == at::kFloat ? FF_F32 : FF_BF16, (int32_t)act, (int32_t)in[1], (int32_t)in[0], x.numel() / in[1]};
    }
};
// the given workspace, checked, or a new one
void workspace(at::Tensor& ws, size_t bytes, at::Device device) {
    if (ws.defined()) {
        if (ws.device() != device || !ws.is_contiguous()) value_error("ws is on ", ws.device(), " or not contiguous");
    } else
        ws = at::empty((int64_t)bytes, at::TensorOptions().dtype(at::kByte).device(device));
}

// x, w_a, w_b, w_o, act, residual, mask, out, ws -> y
PyObject* transition_forward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("transition_forward", 9, n, [&]() -> PyObject* {
        const at::Tensor x = tensor(a[0], "x"), w_a = tensor(a[1], "w_a"), w_b = tensor(a[2], "w_b"), w_o = tensor(a[3], "w_o"), residual = optional(a[5], "residual"),
                         mask = optional(a[6], "mask");
        const long act = PyLong_AsLong(a[4]);
        if (PyErr_Occurred()) return nullptr;
        at::Tensor y = optional(a[7], "out"), ws = optional(a[8], "ws");
        const Transition t(x, w_a, w_b, w_o, mask, act);
        fit_optional(residual, "residual", t.dtype, t.shape, t.device);
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(t.device);
            result(y, "out", t.dtype, t.shape, t.device);
            workspace(ws, ff_gated_transition_forward_workspace_bytes(&t.desc), t.device);
            status = ff_gated_transition_forward(&t.desc, in(x), in(w_a), in(w_b), in(w_o), in(residual), (const float*)in(mask), out(y), out(ws), ws.nbytes(),
                                                 c10::hip::getCurrentHIPStream(t.device.index()).stream());
        }
        return status == FF_OK ? THPVariable_Wrap(y) : PyLong_FromLong(status);
    });
}

// x, w_a, w_b, w_o, dy, act, mask, dx, dw_a, dw_b, dw_o, whether their gradients are float32 (-1: as the weights), accumulate, ws -> (dx, dw_a, dw_b, dw_o)
PyObject* transition_backward(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("transition_backward", 14, n, [&]() -> PyObject* {
        const at::Tensor x = tensor(a[0], "x"), w_a = tensor(a[1], "w_a"), w_b = tensor(a[2], "w_b"), w_o = tensor(a[3], "w_o"), dy = tensor(a[4], "dy"),
                         mask = optional(a[6], "mask");
        const long act = PyLong_AsLong(a[5]), wide = PyLong_AsLong(a[11]);
        const int accumulate = PyObject_IsTrue(a[12]);
        if (PyErr_Occurred()) return nullptr;
        at::Tensor dx = optional(a[7], "dx"), dw_a = optional(a[8], "dw_a"), dw_b = optional(a[9], "dw_b"), dw_o = optional(a[10], "dw_o"), ws = optional(a[13], "ws");
        const Transition t(x, w_a, w_b, w_o, mask, act);
        fit(dy, "dy", t.dtype, t.shape, t.device);
        if (accumulate && !(dw_a.defined() && dw_b.defined() && dw_o.defined())) value_error("accumulate needs dw_a, dw_b and dw_o");
        const at::ScalarType grad = wide < 0 ? dw_a.defined() ? dw_a.scalar_type() : t.dtype : wide ? at::kFloat : at::kBFloat16;
        if (grad != at::kFloat && grad != at::kBFloat16) type_error("unsupported dtype ", grad, " of dw_a");
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(t.device);
            result(dx, "dx", t.dtype, t.shape, t.device);
            result(dw_a, "dw_a", grad, t.in, t.device);
            result(dw_b, "dw_b", grad, t.in, t.device);
            result(dw_o, "dw_o", grad, t.back, t.device);
            workspace(ws, ff_gated_transition_backward_workspace_bytes(&t.desc), t.device);
            status = ff_gated_transition_backward(&t.desc, in(x), in(w_a), in(w_b), in(w_o), in(dy), (const float*)in(mask), out(dx), out(dw_a), out(dw_b), out(dw_o),
                                                  grad == at::kFloat ? FF_F32 : FF_BF16, accumulate, out(ws), ws.nbytes(),
                                                  c10::hip::getCurrentHIPStream(t.device.index()).stream());
        }
        return status == FF_OK ? tuple_of(dx, dw_a, dw_b, dw_o) : PyLong_FromLong(status);
    });
}

// x, steps, a, b, c, eps, out, ws -> out
PyObject* orthogonalise(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("orthogonalise", 8, n, [&]() -> PyObject* {
        const at::Tensor x = tensor(a[0], "x");
        const long steps = PyLong_AsLong(a[1]);
        const double p[4] = {PyFloat_AsDouble(a[2]), PyFloat_AsDouble(a[3]), PyFloat_AsDouble(a[4]), PyFloat_AsDouble(a[5])};
        if (PyErr_Occurred()) return nullptr;
        at::Tensor result_ = optional(a[6], "out"), ws = optional(a[7], "ws");
        const at::ScalarType dtype = x.scalar_type();
        const at::Device device = x.device();
        if (!x.is_cuda()) value_error("x is on ", device, ", not on a GPU");
        if (!x.is_contiguous()) value_error("x is not contiguous");
        if (dtype != at::kFloat && dtype != at::kBFloat16) type_error("unsupported dtype ", dtype);
        if (x.dim() < 2 || x.size(-1) < 1 || x.size(-2) < 1) value_error("no matrices in shape ", x.sizes());
        const int64_t rows = x.size(-2), cols = x.size(-1), count = x.numel() / (rows * cols);
        if (rows > INT32_MAX || cols > INT32_MAX || count > INT32_MAX) value_error("too many values in shape ", x.sizes());
        const ff_orthogonalise_desc desc{dtype == at::kFloat ? FF_F32 : FF_BF16, (int32_t)count, (int32_t)rows, (int32_t)cols, (int32_t)std::clamp(steps, 0l, 1000l), p[0], p[1], p[2], p[3]};
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(device);
            result(result_, "out", dtype, x.sizes(), device);
            workspace(ws, ff_orthogonalise_workspace_bytes(&desc), device);
            status = ff_orthogonalise(&desc, in(x), out(result_), out(ws), ws.nbytes(), c10::hip::getCurrentHIPStream(device.index()).stream());
        }
        return status == FF_OK ? THPVariable_Wrap(result_) : PyLong_FromLong(status);
    });
}

// address of the plan's ff_muon_desc, of its host copy, the plan, address of ff_muon_hyper, norm, max_norm, ws, the plan's stream -> status
PyObject* muon_step(PyObject*, PyObject* const* a, Py_ssize_t n) {
    return guarded("muon_step", 8, n, [&]() -> PyObject* {
        const auto* desc = (const ff_muon_desc*)PyLong_AsVoidPtr(a[0]);
        const void* host = PyLong_AsVoidPtr(a[1]);
        const auto* hyper = (const ff_muon_hyper*)PyLong_AsVoidPtr(a[3]);
        void* const own = PyLong_AsVoidPtr(a[7]);
        if (PyErr_Occurred()) return nullptr;
        const at::Tensor plan = tensor(a[2], "plan"), norm = optional(a[4], "norm"), ws = tensor(a[6], "ws");
        if (norm.defined() != (a[5] != Py_None)) value_error("norm and max_norm are given together");
        const at::Device device = plan.device();
        fit_optional(norm, "norm", at::kFloat, {1}, device);
        if (ws.device() != device || !ws.is_contiguous()) value_error("ws is on ", ws.device(), " or not contiguous");
        ff_status status;
        {
            Unlocked unlocked;
            const c10::DeviceGuard guard(device);
            const c10::hip::HIPStream stream = c10::hip::getCurrentHIPStream(device.index());
            status = ff_muon_step(desc, host, in(plan), plan.nbytes(), hyper, (const float*)in(norm), out(ws), ws.nbytes(), stream.stream());
            in_use(plan, stream, own);
            in_use(ws, stream, own);
        }
        return PyLong_FromLong(status);
    });
}

PyMethodDef kMethods[] = {{"layernorm_forward", (PyCFunction)(void (*)(void))layernorm_forward, METH_FASTCALL, nullptr},
                          {"layernorm_backward", (PyCFunction)(void (*)(void))layernorm_backward, METH_FASTCALL, nullptr},
                          {"grad_norm", (PyCFunction)(void (*)(void))grad_norm, METH_FASTCALL, nullptr},
                          {"adamw_step", (PyCFunction)(void (*)(void))adamw_step, METH_FASTCALL, nullptr},
                          {"adamw_moments", (PyCFunction)(void (*)(void))adamw_moments, METH_FASTCALL, nullptr},
                          {"transition_forward", (PyCFunction)(void (*)(void))transition_forward, METH_FASTCALL, nullptr},
                          {"transition_backward", (PyCFunction)(void (*)(void))transition_backward, METH_FASTCALL, nullptr},
                          {"orthogonalise", (PyCFunction)(void (*)(void))orthogonalise, METH_FASTCALL, nullptr},
                          {"muon_step", (PyCFunction)(void (*)(void))muon_step, METH_FASTCALL, nullptr},
                          {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_calls", nullptr, -1, kMethods};

}  // namespace

PyMODINIT_FUNC PyInit__calls() { return PyModule_Create(&kModule); }

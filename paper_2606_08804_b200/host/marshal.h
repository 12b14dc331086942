// What the native entry points share: arguments to device pointers, checks and their messages, errors, the interpreter's lock.
#pragma once
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/cuda/EmptyTensor.h>
#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/DynamicTypes.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/custom_function.h>
#include <torch/csrc/Dtype.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/qdelta.h"

namespace qdhost {

extern PyObject* g_error;                          // binding.QdeltaError

struct Raised {};                                  // a Python exception is set

[[noreturn]] inline void fail(const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    PyErr_FormatV(g_error ? g_error : PyExc_RuntimeError, fmt, ap);
    va_end(ap);
    throw Raised{};
}
inline void check(int rc, const char* what) {
    if (rc != QD_OK) fail("%s failed: %s (%d)", what, qdelta_status_string(rc), rc);
}

// nullptr for None
inline const at::Tensor* tensor(PyObject* o, const char* name) {
    if (o == Py_None || o == nullptr) return nullptr;
    if (!THPVariable_Check(o)) { PyErr_Format(PyExc_TypeError, "%s must be a tensor, got %s", name, Py_TYPE(o)->tp_name); throw Raised{}; }
    return &THPVariable_Unpack(o);
}
inline const at::Tensor& needed(PyObject* o, const char* name) {
    const at::Tensor* t = tensor(o, name);
    if (!t) { PyErr_Format(PyExc_TypeError, "%s must be a tensor, got NoneType", name); throw Raised{}; }
    return *t;
}
inline void want_dims(const at::Tensor& t, int n) {
    if (t.dim() == n) return;
    if (t.dim() > n) PyErr_Format(PyExc_ValueError, "too many values to unpack (expected %d)", n);
    else PyErr_Format(PyExc_ValueError, "not enough values to unpack (expected %d, got %d)", n, (int)t.dim());
    throw Raised{};
}
inline int dtype_code(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return QD_F32;
    if (t.scalar_type() == at::kBFloat16) return QD_BF16;
    fail("unsupported dtype torch.%s", torch::getTHPDtype(t.scalar_type())->name);
}
inline std::string text(c10::IntArrayRef s) {
    std::string r = "(";
    for (size_t i = 0; i < s.size(); ++i) r += (i ? ", " : "") + std::to_string(s[i]);
    return r + (s.size() == 1 ? ",)" : ")");
}
// what a kernel that is given this tensor's address would trip over; empty if nothing
inline std::string complaint(const at::Tensor& t, at::ScalarType dt, c10::IntArrayRef shape, const char* name, bool any_dtype = false) {
    if (!t.is_cuda() || !t.is_contiguous()) return name + std::string(" must be a contiguous CUDA tensor");
    if (!any_dtype && t.scalar_type() != dt)
        return name + std::string(" must have dtype torch.") + torch::getTHPDtype(dt)->name + ", got torch." + torch::getTHPDtype(t.scalar_type())->name;
    if (t.sizes() != shape) return name + std::string(" must have shape ") + text(shape) + ", got " + text(t.sizes());
    return {};
}
// device pointer of a contiguous CUDA tensor of the given type and shape; nullptr for an absent one
inline void* ptr(const at::Tensor* t, at::ScalarType dt, c10::IntArrayRef shape, const char* name, bool any_dtype = false) {
    if (!t) return nullptr;
    const std::string c = complaint(*t, dt, shape, name, any_dtype);
    if (!c.empty()) fail("%s", c.c_str());
    return t->data_ptr();
}
inline at::Tensor empty(c10::IntArrayRef shape, at::ScalarType dt, c10::Device dev) {
    if (!dev.is_cuda()) fail("the inputs must be contiguous CUDA tensors");
    return at::Tensor(at::detail::empty_cuda(shape, dt, dev, std::nullopt));
}
inline qd_stream stream() { return reinterpret_cast<qd_stream>(c10::cuda::getCurrentCUDAStream().stream()); }

struct NoGil {                                     // other threads may run while kernels are enqueued
    PyThreadState* s = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(s); }
};

// What torch throws keeps its Python type: torch.OutOfMemoryError of an allocation, IndexError, TypeError, or the exception that
// a saved-tensor hook raised (non-reentrant checkpointing ends its recomputation with one).
template <class F> PyObject* guarded(F f) {
    try {
        return f();
    } catch (const Raised&) {
    } catch (...) {
        torch::translate_exception_to_python(std::current_exception());
    }
    return nullptr;
}
inline bool arity(Py_ssize_t n, Py_ssize_t want) {
    if (n == want) return true;
    PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", want, n);
    return false;
}
inline PyObject* own(PyObject* o) { Py_INCREF(o); return o; }
inline int to_int(PyObject* o) {
    const long v = PyLong_AsLong(o);
    if (v == -1 && PyErr_Occurred()) throw Raised{};
    return (int)v;
}

// The caller's tensor that a call has written in place: counted as torch counts its own operations in place, so that a graph that saved
// the tensor refuses its backward instead of computing with other values.
inline void written(const at::Tensor* t) {
    if (t && t->defined() && !t->is_inference()) t->unsafeGetTensorImpl()->bump_version();
}

// ---- autograd ---------------------------------------------------------------------------------------------------------
using torch::autograd::AutogradContext;
using torch::autograd::variable_list;

using MaybeTensor = std::optional<at::Tensor>;
inline const at::Tensor* maybe(const MaybeTensor& t) { return t ? &*t : nullptr; }

// a QdeltaError from a thread of the autograd engine, which does not hold the interpreter
[[noreturn]] inline void raise(const std::string& what) {
    pybind11::gil_scoped_acquire gil;
    PyErr_SetString(g_error, what.c_str());
    python_error e;
    e.persist();
    throw std::move(e);
}

extern PyMethodDef layer_methods[];                // the operators around the delta rule (layer.cpp)
extern PyMethodDef linear_methods[];               // those of a linear attention layer (linear.cpp)

}  // namespace qdhost

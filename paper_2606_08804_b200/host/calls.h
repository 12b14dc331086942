// What the entry points of the operators around the delta rule share (layer.cpp, linear.cpp): errors that threads without the interpreter can
// throw, the device of a call, gradients of parameters, results to Python, autograd.
#pragma once
#include "marshal.h"

#include <torch/csrc/autograd/functions/basic_ops.h>

#include <array>
#include <climits>

namespace qdhost {
namespace {

// Thrown by what Python's threads (which hold the interpreter) and autograd's (which do not) share.
struct Bad { std::string what; };
[[noreturn]] void bad(std::string what) { throw Bad{std::move(what)}; }

void rc_check(int rc, const char* what) {
    if (rc != QD_OK) bad(std::string(what) + " failed: " + qdelta_status_string(rc) + " (" + std::to_string(rc) + ")");
}
int i32(int64_t n, const char* name) {
    if (n > INT_MAX) bad(std::string(name) + " is too large");
    return (int)n;
}
int code_of(const at::Tensor& t) {
    if (t.scalar_type() == at::kFloat) return QD_F32;
    if (t.scalar_type() == at::kBFloat16) return QD_BF16;
    bad(std::string("unsupported dtype torch.") + torch::getTHPDtype(t.scalar_type())->name);
}
void dims(const at::Tensor& t, int n, const char* what) {
    if (t.dim() != n) bad(std::string(what) + ", got " + std::to_string(t.dim()) + " dimensions");
}

// The device of a call, made current for its duration.
struct On {
    c10::Device dev;
    c10::cuda::CUDAGuard guard;
    static c10::Device of(const at::Tensor& t, const char* name) {
        if (!t.is_cuda()) bad(std::string(name) + " must be a contiguous CUDA tensor");
        return t.device();
    }
    On(const at::Tensor& t, const char* name) : dev(of(t, name)), guard(dev) {}
    void* p(const at::Tensor* t, at::ScalarType dt, c10::IntArrayRef shape, const char* name) const {
        if (!t || !t->defined()) return nullptr;
        const std::string c = complaint(*t, dt, shape, name);
        if (!c.empty()) bad(c);
        if (t->device() != dev) bad(std::string(name) + " must be on the device of the other tensors");
        return t->data_ptr();
    }
    float* f(const at::Tensor* t, c10::IntArrayRef shape, const char* name) const { return static_cast<float*>(p(t, at::kFloat, shape, name)); }
    at::Tensor make(c10::IntArrayRef shape, at::ScalarType dt) const { return at::Tensor(at::detail::empty_cuda(shape, dt, dev, std::nullopt)); }
};

// Gradients of parameters, fp32, side by side in one allocation: one conversion takes all of them to another type.
struct Params {
    at::Tensor all;
    int64_t at = 0;
    Params(const On& on, std::initializer_list<int64_t> sizes) {
        int64_t n = 0;
        for (const int64_t s : sizes) n += (s + 3) / 4 * 4;
        all = on.make({n}, at::kFloat);
    }
    at::Tensor next(c10::IntArrayRef shape) {              // each 16-byte aligned
        int64_t n = 1;
        for (const int64_t s : shape) n *= s;
        // a view without the dispatcher's two calls for one
        at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::TensorImpl::VIEW, c10::Storage(all.storage()), all.key_set(), all.dtype());
        t.unsafeGetTensorImpl()->set_storage_offset(all.storage_offset() + at);
        t.unsafeGetTensorImpl()->set_sizes_contiguous(shape);
        at += (n + 3) / 4 * 4;
        return t;
    }
};
// ---- calls from Python ----------------------------------------------------------------------------------------------------
template <class F> PyObject* called(F f) {
    return guarded([&]() -> PyObject* {
        try {
            return f();
        } catch (const Bad& b) {
            fail("%s", b.what.c_str());
        }
    });
}
template <class F> auto unlocked(F f) {
    NoGil ng;
    return f();
}
unsigned to_flags(PyObject* o) {
    const unsigned long v = PyLong_AsUnsignedLong(o);
    if (PyErr_Occurred()) throw Raised{};
    return (unsigned)v;
}
PyObject* wrapped(const at::Tensor& t) { return t.defined() ? THPVariable_Wrap(t) : own(Py_None); }
PyObject* tuple(std::initializer_list<at::Tensor> ts) {
    PyObject* r = PyTuple_New((Py_ssize_t)ts.size());
    if (!r) throw Raised{};
    Py_ssize_t i = 0;
    for (const at::Tensor& t : ts) {
        PyObject* w = wrapped(t);
        if (!w) { Py_DECREF(r); throw Raised{}; }
        PyTuple_SET_ITEM(r, i++, w);
    }
    return r;
}
PyObject* dict(std::initializer_list<std::pair<const char*, at::Tensor>> ts) {
    PyObject* r = PyDict_New();
    if (!r) throw Raised{};
    for (const auto& [name, t] : ts) {
        PyObject* w = wrapped(t);
        const int e = w ? PyDict_SetItemString(r, name, w) : -1;
        Py_XDECREF(w);
        if (e) { Py_DECREF(r); throw Raised{}; }
    }
    return r;
}

// ---- autograd ---------------------------------------------------------------------------------------------------------------
// dense, and where the kernels can read 16 bytes at a time (a dense view may begin anywhere)
at::Tensor usable(const at::Tensor& t) {
    at::Tensor c = t.contiguous();
    return c.is_cuda() && (reinterpret_cast<uintptr_t>(c.data_ptr()) & 15) ? c.clone() : c;
}
// the gradient that arrived for an output, in the type the kernels take; undefined stays so
at::Tensor upstream(const at::Tensor& g, at::ScalarType dt) { return g.defined() ? usable(g.to(dt)) : g; }
at::Tensor or_zeros(const at::Tensor& g, const at::Tensor& like) { return g.defined() ? g : at::zeros_like(like); }
const at::Tensor* given(const at::Tensor& t) { return t.defined() ? &t : nullptr; }
at::Tensor or_none(const MaybeTensor& t) { return t ? *t : at::Tensor(); }
// a parameter's gradient in the type of `like`: the same place in the converted allocation
at::Tensor as(const at::Tensor& g, const at::Tensor& like, const at::Tensor& all, at::Tensor& converted) {
    if (!g.defined() || g.scalar_type() == like.scalar_type()) return g;
    if (!converted.defined()) converted = all.to(like.scalar_type());
    return converted.narrow(0, g.storage_offset() - all.storage_offset(), g.numel()).view(g.sizes());
}

// The kernels give first derivatives: with create_graph a second one is refused when it is asked for.
template <class F> variable_list in_backward(F f) {
    variable_list g;
    try {
        at::NoGradGuard off;
        g = f();
    } catch (const Bad& b) {
        raise(b.what);
    }
    if (!at::GradMode::is_enabled()) return g;
    variable_list have;
    for (at::Tensor& t : g)
        if (t.defined()) have.push_back(t.detach().set_requires_grad(true));
    auto refuse = std::make_shared<torch::autograd::DelayedError>("second derivatives of this operator are not available", (int64_t)have.size());
    have = (*refuse)(std::move(have));
    size_t i = 0;
    for (at::Tensor& t : g)
        if (t.defined()) t = have[i++];
    return g;
}
// saved tensors that hooks hand back may be others than were saved: the checks of the call see them again
void present(const at::Tensor& t, const char* name) {
    if (!t.defined()) bad(std::string(name) + " must be a tensor");
}
// Inputs of a node: dense and aligned; whether a gradient is wanted of any.
template <size_t N> bool inputs(PyObject* const* a, const char* const (&names)[N], size_t required, MaybeTensor (&t)[N]) {
    bool need = false;
    for (size_t i = 0; i < N; ++i) {
        const at::Tensor* x = i < required ? &needed(a[i], names[i]) : tensor(a[i], names[i]);
        if (!x) continue;
        need = need || x->requires_grad();
        t[i] = usable(*x);
    }
    return need && at::GradMode::is_enabled();
}

}  // namespace
}  // namespace qdhost

// Host path of the operators around the delta rule: convolution, selective scan, layer norm; single calls and autograd nodes.
// As in host.cpp: checks, output allocation and the C-ABI call, every number from libqdelta.so.  A call works on the device of its
// tensors, in the current stream of that device, whichever device is current.
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

// ---- convolution --------------------------------------------------------------------------------------------------------
struct Conv {
    On on;
    int64_t B, T, D, W;
    at::ScalarType dt;
    int code, b, t, d, w;
    const void *xp, *wp, *bp;
    Conv(const at::Tensor& x, const at::Tensor& wt, const at::Tensor* bias) : on(x, "x") {
        dims(x, 3, "x must be [B, T, D]");
        dims(wt, 2, "w must be [D, W]");
        B = x.size(0); T = x.size(1); D = x.size(2); W = wt.size(1);
        dt = x.scalar_type();
        code = code_of(x);
        b = i32(B, "B"); t = i32(T, "T"); d = i32(D, "D"); w = i32(W, "W");
        xp = on.p(&x, dt, {B, T, D}, "x");
        wp = on.p(&wt, dt, {D, W}, "w");
        bp = on.p(bias, dt, {D}, "bias");
    }
    // of a state; a width that no kernel serves is refused by the call, not by a negative size
    std::array<int64_t, 3> state() const { return {B, W > 1 ? W - 1 : 1, D}; }
};
std::pair<at::Tensor, at::Tensor> conv_forward(const at::Tensor& x, const at::Tensor& w, const at::Tensor* bias, const at::Tensor* state,
                                               bool want_last, unsigned flags) {
    const Conv c(x, w, bias);
    const void* sp = c.on.p(state, c.dt, c.state(), "state");
    at::Tensor y = c.on.make({c.B, c.T, c.D}, c.dt), last;
    if (want_last) last = c.on.make(c.state(), c.dt);
    rc_check(qdelta_conv_fwd(c.b, c.t, c.d, c.w, c.code, c.xp, c.wp, c.bp, sp, y.data_ptr(), want_last ? last.data_ptr() : nullptr, flags, stream()),
             "qdelta_conv_fwd");
    return {y, last};
}
struct ConvGrads { at::Tensor dx, dw, dbias, dstate, params; };
ConvGrads conv_backward(const at::Tensor& x, const at::Tensor& w, const at::Tensor* bias, const at::Tensor* state, const at::Tensor& dy,
                        const at::Tensor* dlast, bool want_dstate, unsigned flags) {
    const Conv c(x, w, bias);
    const void *sp = c.on.p(state, c.dt, c.state(), "state"), *gp = c.on.p(&dy, c.dt, {c.B, c.T, c.D}, "dy");
    const void* lp = c.on.p(dlast, c.dt, c.state(), "dstate");
    const size_t n = qdelta_conv_workspace_bytes(c.b, c.t, c.d, c.w, c.code);
    if (n == 0) bad("unsupported or invalid shape for the convolution");
    const at::Tensor ws = c.on.make({(int64_t)n}, at::kByte);
    ConvGrads g;
    g.dx = c.on.make({c.B, c.T, c.D}, c.dt);
    Params params(c.on, {c.D * c.W, bias ? c.D : 0});
    g.params = params.all;
    g.dw = params.next({c.D, c.W});
    if (bias) g.dbias = params.next({c.D});
    if (want_dstate) g.dstate = c.on.make(c.state(), c.dt);
    rc_check(qdelta_conv_bwd(c.b, c.t, c.d, c.w, c.code, c.xp, c.wp, c.bp, sp, gp, lp, g.dx.data_ptr(), g.dw.data_ptr<float>(),
                             bias ? g.dbias.data_ptr<float>() : nullptr, want_dstate ? g.dstate.data_ptr() : nullptr, ws.data_ptr(), n, flags,
                             stream()),
             "qdelta_conv_bwd");
    return g;
}

// ---- scan -----------------------------------------------------------------------------------------------------------------
struct Scan {
    On on;
    qd_scan_shape s;
    int64_t B, T, D, N, G;
    at::ScalarType dt;
    const void *u, *dtp, *Bm, *Cm, *z;
    const float *A, *skip, *bias;
    // t: u, dt, A, Bm, Cm, D, z, dt_bias; the last three may be absent
    explicit Scan(const at::Tensor* const* t) : on(*t[0], "u") {
        dims(*t[0], 3, "u must be [B, T, D]");
        dims(*t[2], 2, "A must be [D, N]");
        dims(*t[3], 4, "Bm must be [B, T, G, N]");
        B = t[0]->size(0); T = t[0]->size(1); D = t[0]->size(2); N = t[2]->size(1); G = t[3]->size(2);
        dt = t[0]->scalar_type();
        s = qd_scan_shape{i32(B, "B"), i32(T, "T"), i32(D, "D"), i32(N, "N"), i32(G, "G"), code_of(*t[0])};
        u = on.p(t[0], dt, {B, T, D}, "u");
        dtp = on.p(t[1], dt, {B, T, D}, "dt");
        A = on.f(t[2], {D, N}, "A");
        Bm = on.p(t[3], dt, {B, T, G, N}, "Bm");
        Cm = on.p(t[4], dt, {B, T, G, N}, "Cm");
        skip = on.f(t[5], {D}, "D");
        z = on.p(t[6], dt, {B, T, D}, "z");
        bias = on.f(t[7], {D}, "dt_bias");
    }
    float* state(const at::Tensor* t, const char* name) const { return on.f(t, {B, D, N}, name); }
    at::Tensor workspace(int for_backward) const {
        const size_t n = qdelta_scan_workspace_bytes(&s, for_backward);
        if (for_backward && n == 0) bad("unsupported or invalid shape for the scan");
        return n ? on.make({(int64_t)n}, at::kByte) : at::Tensor();
    }
};
struct ScanOut { at::Tensor y, hT, ws; };
ScanOut scan_forward(const at::Tensor* const* t, const at::Tensor* h0, const at::Tensor* workspace, bool want_hT, unsigned flags) {
    const Scan c(t);
    const float* hp = c.state(h0, "h0");
    ScanOut r;
    r.ws = workspace ? *workspace : c.workspace(flags & QD_FWD_SAVE_FOR_BWD ? 1 : 0);
    if (r.ws.defined()) c.on.p(&r.ws, at::kByte, {r.ws.numel()}, "workspace");
    r.y = c.on.make({c.B, c.T, c.D}, c.dt);
    if (want_hT) r.hT = c.on.make({c.B, c.D, c.N}, at::kFloat);
    rc_check(qdelta_scan_fwd(&c.s, c.u, c.dtp, c.A, c.Bm, c.Cm, c.skip, c.z, c.bias, hp, r.y.data_ptr(),
                             want_hT ? r.hT.data_ptr<float>() : nullptr, r.ws.defined() ? r.ws.data_ptr() : nullptr,
                             r.ws.defined() ? (size_t)r.ws.numel() : 0, flags, stream()),
             "qdelta_scan_fwd");
    return r;
}
struct ScanGrads { at::Tensor du, ddt, dA, dBm, dCm, dD, dz, dbias, dh0; };
ScanGrads scan_backward(const at::Tensor* const* t, const at::Tensor* h0, const at::Tensor& dy, const at::Tensor* dhT,
                        const at::Tensor* workspace, bool want_dh0, unsigned flags) {
    const Scan c(t);
    const float *hp = c.state(h0, "h0"), *gh = c.state(dhT, "dhT");
    const void* gy = c.on.p(&dy, c.dt, {c.B, c.T, c.D}, "dy");
    const at::Tensor ws = workspace ? *workspace : c.workspace(1);
    c.on.p(&ws, at::kByte, {ws.numel()}, "workspace");
    ScanGrads g;
    g.du = c.on.make({c.B, c.T, c.D}, c.dt);
    g.ddt = c.on.make({c.B, c.T, c.D}, c.dt);
    g.dA = c.on.make({c.D, c.N}, at::kFloat);
    g.dBm = c.on.make({c.B, c.T, c.G, c.N}, c.dt);
    g.dCm = c.on.make({c.B, c.T, c.G, c.N}, c.dt);
    if (c.skip) g.dD = c.on.make({c.D}, at::kFloat);
    if (c.z) g.dz = c.on.make({c.B, c.T, c.D}, c.dt);
    if (c.bias) g.dbias = c.on.make({c.D}, at::kFloat);
    if (want_dh0) g.dh0 = c.on.make({c.B, c.D, c.N}, at::kFloat);
    const auto f = [](const at::Tensor& x) { return x.defined() ? x.data_ptr<float>() : nullptr; };
    rc_check(qdelta_scan_bwd(&c.s, c.u, c.dtp, c.A, c.Bm, c.Cm, c.skip, c.z, c.bias, hp, gy, gh, g.du.data_ptr(), g.ddt.data_ptr(), f(g.dA),
                             g.dBm.data_ptr(), g.dCm.data_ptr(), f(g.dD), c.z ? g.dz.data_ptr() : nullptr, f(g.dbias), f(g.dh0),
                             ws.data_ptr(), (size_t)ws.numel(), flags, stream()),
             "qdelta_scan_bwd");
    return g;
}

// ---- norm -----------------------------------------------------------------------------------------------------------------
struct Norm {
    On on;
    int64_t rows, width;
    at::ScalarType dt;
    int code, w;
    const void *xp, *wp;
    Norm(const at::Tensor& x, const at::Tensor* weight) : on(x, "x") {
        if (x.dim() < 1) bad("x must have a last dimension to normalise");
        width = x.size(-1);
        rows = width ? x.numel() / width : 0;
        dt = x.scalar_type();
        code = code_of(x);
        w = i32(width, "the width");
        xp = on.p(&x, dt, x.sizes(), "x");
        wp = on.p(weight, dt, {width}, "weight");
    }
};
std::pair<at::Tensor, at::Tensor> norm_forward(const at::Tensor& x, const at::Tensor* weight, const at::Tensor* bias, double eps,
                                               bool want_stats, unsigned flags) {
    const Norm c(x, weight);
    const void* bp = c.on.p(bias, c.dt, {c.width}, "bias");
    at::Tensor y = c.on.make(x.sizes(), c.dt), stats;
    if (want_stats) stats = c.on.make({2, c.rows}, at::kFloat);
    rc_check(qdelta_norm_fwd(c.rows, c.w, c.code, c.xp, c.wp, bp, y.data_ptr(), want_stats ? stats.data_ptr<float>() : nullptr, (float)eps,
                             flags, stream()),
             "qdelta_norm_fwd");
    return {y, stats};
}
struct NormGrads { at::Tensor dx, dweight, dbias, params; };
NormGrads norm_backward(const at::Tensor& x, const at::Tensor* weight, const at::Tensor& dy, const at::Tensor& stats, bool want_dweight,
                        bool want_dbias, unsigned flags) {
    const Norm c(x, weight);
    const void* gp = c.on.p(&dy, c.dt, x.sizes(), "dy");
    const float* sp = c.on.f(&stats, {2, c.rows}, "stats");
    NormGrads g;
    g.dx = c.on.make(x.sizes(), c.dt);
    at::Tensor ws;
    if (want_dweight || want_dbias) {
        const size_t n = qdelta_norm_workspace_bytes(c.rows, c.w, c.code);
        if (n == 0) bad("unsupported or invalid shape for the norm");
        ws = c.on.make({(int64_t)n}, at::kByte);
    }
    Params params(c.on, {want_dweight ? c.width : 0, want_dbias ? c.width : 0});
    g.params = params.all;
    if (want_dweight) g.dweight = params.next({c.width});
    if (want_dbias) g.dbias = params.next({c.width});
    rc_check(qdelta_norm_bwd(c.rows, c.w, c.code, c.xp, c.wp, gp, sp, g.dx.data_ptr(), want_dweight ? g.dweight.data_ptr<float>() : nullptr,
                             want_dbias ? g.dbias.data_ptr<float>() : nullptr, ws.defined() ? ws.data_ptr() : nullptr,
                             ws.defined() ? (size_t)ws.numel() : 0, flags, stream()),
             "qdelta_norm_bwd");
    return g;
}

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

// conv_fwd(x, w, bias, state, want_last, flags) -> (y, last)
PyObject* conv_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &w = needed(a[1], "w");
        const at::Tensor *bias = tensor(a[2], "bias"), *state = tensor(a[3], "state");
        const unsigned flags = to_flags(a[5]);
        const auto r = unlocked([&] { return conv_forward(x, w, bias, state, a[4] == Py_True, flags); });
        return tuple({r.first, r.second});
    });
}
// conv_bwd(x, w, bias, state, dy, dlast, want_dstate, flags) -> {dx, dw, dbias, dstate}
PyObject* conv_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 8)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &w = needed(a[1], "w"), &dy = needed(a[4], "dy");
        const at::Tensor *bias = tensor(a[2], "bias"), *state = tensor(a[3], "state"), *dlast = tensor(a[5], "dstate");
        const unsigned flags = to_flags(a[7]);
        const ConvGrads g = unlocked([&] { return conv_backward(x, w, bias, state, dy, dlast, a[6] == Py_True, flags); });
        return dict({{"dx", g.dx}, {"dw", g.dw}, {"dbias", g.dbias}, {"dstate", g.dstate}});
    });
}
// conv_steps(x, w, bias, state, y, flags) -> y
PyObject* conv_steps(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &w = needed(a[1], "w"), &state = needed(a[3], "state");
        const at::Tensor *bias = tensor(a[2], "bias"), *given = tensor(a[4], "y");
        const unsigned flags = to_flags(a[5]);
        const at::Tensor y = unlocked([&] {
            const Conv c(x, w, bias);
            void* sp = c.on.p(&state, c.dt, c.state(), "state");
            const at::Tensor o = given ? *given : c.on.make({c.B, c.T, c.D}, c.dt);
            rc_check(qdelta_conv_steps(c.b, c.t, c.d, c.w, c.code, c.xp, c.wp, c.bp, sp, c.on.p(&o, c.dt, {c.B, c.T, c.D}, "y"), flags, stream()),
                     "qdelta_conv_steps");
            written(&state);
            written(given);
            return o;
        });
        return given ? own(a[4]) : wrapped(y);
    });
}

struct ScanTensors {
    const at::Tensor* t[8];
    explicit ScanTensors(PyObject* const* a) {
        static const char* names[8] = {"u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias"};
        for (int i = 0; i < 8; ++i) t[i] = i < 5 ? &needed(a[i], names[i]) : tensor(a[i], names[i]);
    }
};
// scan_fwd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, workspace, want_hT, flags) -> (y, hT, workspace)
PyObject* scan_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 12)) return nullptr;
    return called([&] {
        const ScanTensors t(a);
        const at::Tensor *h0 = tensor(a[8], "h0"), *ws = tensor(a[9], "workspace");
        const unsigned flags = to_flags(a[11]);
        const ScanOut r = unlocked([&] { return scan_forward(t.t, h0, ws, a[10] == Py_True, flags); });
        return tuple({r.y, r.hT, r.ws});
    });
}
// scan_bwd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, dy, dhT, workspace, want_dh0, flags) -> {du, ddt, dA, dBm, dCm, dD, dz, ddt_bias, dh0}
PyObject* scan_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 14)) return nullptr;
    return called([&] {
        const ScanTensors t(a);
        const at::Tensor *h0 = tensor(a[8], "h0"), *dhT = tensor(a[10], "dhT"), *ws = tensor(a[11], "workspace");
        const at::Tensor& dy = needed(a[9], "dy");
        const unsigned flags = to_flags(a[13]);
        const ScanGrads g = unlocked([&] { return scan_backward(t.t, h0, dy, dhT, ws, a[12] == Py_True, flags); });
        return dict({{"du", g.du}, {"ddt", g.ddt}, {"dA", g.dA}, {"dBm", g.dBm}, {"dCm", g.dCm}, {"dD", g.dD}, {"dz", g.dz},
                     {"ddt_bias", g.dbias}, {"dh0", g.dh0}});
    });
}
// scan_steps(u, dt, A, Bm, Cm, D, z, dt_bias, state, y, flags) -> y
PyObject* scan_steps(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 11)) return nullptr;
    return called([&] {
        const ScanTensors t(a);
        const at::Tensor& state = needed(a[8], "state");
        const at::Tensor* given = tensor(a[9], "y");
        const unsigned flags = to_flags(a[10]);
        const at::Tensor y = unlocked([&] {
            const Scan c(t.t);
            float* sp = c.state(&state, "state");
            const at::Tensor o = given ? *given : c.on.make({c.B, c.T, c.D}, c.dt);
            rc_check(qdelta_scan_steps(&c.s, c.u, c.dtp, c.A, c.Bm, c.Cm, c.skip, c.z, c.bias, sp, c.on.p(&o, c.dt, {c.B, c.T, c.D}, "y"), flags,
                                       stream()),
                     "qdelta_scan_steps");
            written(&state);
            written(given);
            return o;
        });
        return given ? own(a[9]) : wrapped(y);
    });
}

// norm_fwd(x, weight, bias, eps, want_stats, flags) -> (y, stats)
PyObject* norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    return called([&] {
        const at::Tensor& x = needed(a[0], "x");
        const at::Tensor *weight = tensor(a[1], "weight"), *bias = tensor(a[2], "bias");
        const double eps = PyFloat_AsDouble(a[3]);
        if (PyErr_Occurred()) throw Raised{};
        const unsigned flags = to_flags(a[5]);
        const auto r = unlocked([&] { return norm_forward(x, weight, bias, eps, a[4] == Py_True, flags); });
        return tuple({r.first, r.second});
    });
}
// norm_bwd(x, weight, dy, stats, want_dweight, want_dbias, flags) -> {dx, dweight, dbias}
PyObject* norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &dy = needed(a[2], "dy"), &stats = needed(a[3], "stats");
        const at::Tensor* weight = tensor(a[1], "weight");
        const unsigned flags = to_flags(a[6]);
        const NormGrads g = unlocked([&] { return norm_backward(x, weight, dy, stats, a[4] == Py_True, a[5] == Py_True, flags); });
        return dict({{"dx", g.dx}, {"dweight", g.dweight}, {"dbias", g.dbias}});
    });
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

struct ConvNode : torch::autograd::Function<ConvNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const at::Tensor& w, const MaybeTensor& bias,
                                 const MaybeTensor& state, int64_t flags, bool need_grad) {
        const auto r = conv_forward(x, w, maybe(bias), maybe(state), true, (unsigned)flags);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            ctx->save_for_backward({x, w, or_none(bias), or_none(state)});
            ctx->saved_data["flags"] = flags;
        }
        return {r.first, r.second};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            const at::Tensor &x = in[0], &w = in[1], &bias = in[2], &state = in[3];
            present(x, "x");
            present(w, "w");
            const at::Tensor dy = or_zeros(upstream(g[0], x.scalar_type()), x), dlast = upstream(g[1], x.scalar_type());
            const ConvGrads r = conv_backward(x, w, given(bias), given(state), dy, given(dlast), state.defined(),
                                              (unsigned)ctx->saved_data["flags"].toInt());
            at::Tensor converted;
            return {r.dx, as(r.dw, w, r.params, converted), as(r.dbias, w, r.params, converted), r.dstate, at::Tensor(), at::Tensor()};
        });
    }
};

struct ScanNode : torch::autograd::Function<ScanNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& u, const at::Tensor& dt, const at::Tensor& A, const at::Tensor& Bm,
                                 const at::Tensor& Cm, const MaybeTensor& D, const MaybeTensor& z, const MaybeTensor& bias,
                                 const MaybeTensor& h0, int64_t flags, bool need_grad) {
        const at::Tensor* t[8] = {&u, &dt, &A, &Bm, &Cm, maybe(D), maybe(z), maybe(bias)};
        const ScanOut r = scan_forward(t, maybe(h0), nullptr, true, (unsigned)flags | (need_grad ? QD_FWD_SAVE_FOR_BWD : 0));
        ctx->set_materialize_grads(false);
        if (need_grad) {
            // not h0, which the workspace stands for: its owner may go on with it in place
            ctx->save_for_backward({u, dt, A, Bm, Cm, or_none(D), or_none(z), or_none(bias), r.ws});
            ctx->saved_data["flags"] = flags;
            ctx->saved_data["h0"] = h0.has_value();
        }
        return {r.y, r.hT};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            static const char* names[5] = {"u", "dt", "A", "Bm", "Cm"};
            const at::Tensor* t[8];
            for (int i = 0; i < 8; ++i) {
                if (i < 5) present(in[i], names[i]);
                t[i] = given(in[i]);
            }
            present(in[8], "the saved workspace");
            const at::Tensor& u = in[0];
            const at::Tensor dy = or_zeros(upstream(g[0], u.scalar_type()), u), dhT = upstream(g[1], at::kFloat);
            const ScanGrads r = scan_backward(t, nullptr, dy, given(dhT), &in[8], ctx->saved_data["h0"].toBool(),
                                              (unsigned)ctx->saved_data["flags"].toInt() | QD_BWD_REUSE_FWD);
            return {r.du, r.ddt, r.dA, r.dBm, r.dCm, r.dD, r.dz, r.dbias, r.dh0, at::Tensor(), at::Tensor()};
        });
    }
};

struct NormNode : torch::autograd::Function<NormNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const MaybeTensor& weight, const MaybeTensor& bias, double eps,
                                 int64_t flags, bool need_grad) {
        const auto r = norm_forward(x, maybe(weight), maybe(bias), eps, need_grad, (unsigned)flags);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            ctx->save_for_backward({x, or_none(weight), or_none(bias), r.second});
            ctx->saved_data["flags"] = flags;
            ctx->saved_data["dweight"] = weight && weight->requires_grad();
            ctx->saved_data["dbias"] = bias && bias->requires_grad();
        }
        return {r.first};
    }
    static variable_list backward(AutogradContext* ctx, variable_list g) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            const at::Tensor &x = in[0], &weight = in[1], &bias = in[2], &stats = in[3];
            present(x, "x");
            present(stats, "the saved statistics");
            const at::Tensor dy = or_zeros(upstream(g[0], x.scalar_type()), x);
            const NormGrads r = norm_backward(x, given(weight), dy, stats, weight.defined() && ctx->saved_data["dweight"].toBool(),
                                              bias.defined() && ctx->saved_data["dbias"].toBool(), (unsigned)ctx->saved_data["flags"].toInt());
            at::Tensor converted;
            return {r.dx, as(r.dweight, x, r.params, converted), as(r.dbias, x, r.params, converted), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};

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

// conv_autograd(x, w, bias, state, flags) -> (y, last)
PyObject* conv_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 5)) return nullptr;
    return called([&] {
        MaybeTensor t[4];
        const bool need = inputs(a, {"x", "w", "bias", "state"}, 2, t);
        const variable_list r = ConvNode::apply(*t[0], *t[1], t[2], t[3], (int64_t)to_flags(a[4]), need);
        return tuple({r[0], r[1]});
    });
}
// scan_autograd(u, dt, A, Bm, Cm, D, z, dt_bias, h0, flags) -> (y, hT)
PyObject* scan_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 10)) return nullptr;
    return called([&] {
        MaybeTensor t[9];
        const bool need = inputs(a, {"u", "dt", "A", "Bm", "Cm", "D", "z", "dt_bias", "h0"}, 5, t);
        const variable_list r = ScanNode::apply(*t[0], *t[1], *t[2], *t[3], *t[4], t[5], t[6], t[7], t[8], (int64_t)to_flags(a[9]), need);
        return tuple({r[0], r[1]});
    });
}
// norm_autograd(x, weight, bias, eps, flags) -> y
PyObject* norm_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 5)) return nullptr;
    return called([&] {
        MaybeTensor t[3];
        const bool need = inputs(a, {"x", "weight", "bias"}, 1, t);
        const double eps = PyFloat_AsDouble(a[3]);
        if (PyErr_Occurred()) throw Raised{};
        const variable_list r = NormNode::apply(*t[0], t[1], t[2], eps, (int64_t)to_flags(a[4]), need);
        return wrapped(r[0]);
    });
}

}  // namespace

#define QD_METHOD(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef layer_methods[] = {
    QD_METHOD(conv_fwd), QD_METHOD(conv_bwd), QD_METHOD(conv_steps), QD_METHOD(scan_fwd), QD_METHOD(scan_bwd), QD_METHOD(scan_steps),
    QD_METHOD(norm_fwd), QD_METHOD(norm_bwd), QD_METHOD(conv_autograd), QD_METHOD(scan_autograd), QD_METHOD(norm_autograd),
    {nullptr, nullptr, 0, nullptr},
};

}  // namespace qdhost

// Host path of the operators of a linear attention layer: the attention, its gated norm, the norm behind the residual sum, rotary positions.
// As in layer.cpp.
#include "calls.h"

namespace qdhost {
namespace {

void* at_of(const at::Tensor& t) { return t.defined() ? t.data_ptr() : nullptr; }
float* floats(const at::Tensor& t) { return t.defined() ? t.data_ptr<float>() : nullptr; }

// ---- linear attention -------------------------------------------------------------------------------------------------------
struct Linear {
    On on;
    int64_t B, T, H, dk, dv;
    at::ScalarType dt;
    qd_linear_shape s;
    const void *q, *k, *v;
    const float* g;
    Linear(const at::Tensor& qt, const at::Tensor& kt, const at::Tensor& vt, const at::Tensor& decay) : on(qt, "q") {
        dims(qt, 4, "q must be [B, T, H, dk]");
        dims(vt, 4, "v must be [B, T, H, dv]");
        B = qt.size(0); T = qt.size(1); H = qt.size(2); dk = qt.size(3); dv = vt.size(3);
        dt = qt.scalar_type();
        s = qd_linear_shape{i32(B, "B"), i32(T, "T"), i32(H, "H"), i32(dk, "dk"), i32(dv, "dv"), code_of(qt)};
        q = on.p(&qt, dt, {B, T, H, dk}, "q");
        k = on.p(&kt, dt, {B, T, H, dk}, "k");
        v = on.p(&vt, dt, {B, T, H, dv}, "v");
        g = on.f(&decay, {H}, "log_decay");
    }
    float* state(const at::Tensor* t, const char* name) const { return on.f(t, {B, H, dk, dv}, name); }
    at::Tensor workspace(const at::Tensor* given, int for_backward) const {
        if (given) {
            on.p(given, at::kByte, {given->numel()}, "workspace");
            return *given;
        }
        const size_t n = qdelta_linear_workspace_bytes(&s, for_backward);
        if (n == 0) bad("unsupported or invalid shape for linear attention");
        return on.make({(int64_t)n}, at::kByte);
    }
};
struct LinearOut { at::Tensor o, hT, ws; };
LinearOut linear_forward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& decay, const at::Tensor* h0,
                         const at::Tensor* workspace, bool want_hT, double scale) {
    const Linear c(q, k, v, decay);
    const float* hp = c.state(h0, "h0");
    LinearOut r;
    r.ws = c.workspace(workspace, 0);
    r.o = c.on.make({c.B, c.T, c.H, c.dv}, c.dt);
    if (want_hT) r.hT = c.on.make({c.B, c.H, c.dk, c.dv}, at::kFloat);
    rc_check(qdelta_linear_fwd(&c.s, c.q, c.k, c.v, c.g, hp, r.o.data_ptr(), floats(r.hT), (float)scale, r.ws.data_ptr(), (size_t)r.ws.numel(), 0,
                               stream()),
             "qdelta_linear_fwd");
    return r;
}
struct LinearGrads { at::Tensor dq, dk, dv, dh0; };
LinearGrads linear_backward(const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& decay, const at::Tensor* h0,
                            const at::Tensor& dO, const at::Tensor* dhT, const at::Tensor* workspace, bool want_dh0, double scale) {
    const Linear c(q, k, v, decay);
    const float *hp = c.state(h0, "h0"), *gh = c.state(dhT, "dhT");
    const void* go = c.on.p(&dO, c.dt, {c.B, c.T, c.H, c.dv}, "dO");
    const at::Tensor ws = c.workspace(workspace, 1);
    LinearGrads r;
    r.dq = c.on.make({c.B, c.T, c.H, c.dk}, c.dt);
    r.dk = c.on.make({c.B, c.T, c.H, c.dk}, c.dt);
    r.dv = c.on.make({c.B, c.T, c.H, c.dv}, c.dt);
    if (want_dh0) r.dh0 = c.on.make({c.B, c.H, c.dk, c.dv}, at::kFloat);
    rc_check(qdelta_linear_bwd(&c.s, c.q, c.k, c.v, c.g, hp, go, gh, r.dq.data_ptr(), r.dk.data_ptr(), r.dv.data_ptr(), floats(r.dh0),
                               (float)scale, ws.data_ptr(), (size_t)ws.numel(), 0, stream()),
             "qdelta_linear_bwd");
    return r;
}

// ---- layer norm with a gate, and behind a residual sum ----------------------------------------------------------------------
constexpr int64_t kNarrow = 1024;            // columns up to which a backward without sums over rows needs no workspace
struct Fused {
    On on;
    int64_t rows, width;
    at::ScalarType dt;
    int code, w;
    const void* xp;
    Fused(const at::Tensor& x, const char* name) : on(x, name) {
        if (x.dim() < 1) bad(std::string(name) + " must have a last dimension to normalise");
        width = x.size(-1);
        rows = width ? x.numel() / width : 0;
        dt = x.scalar_type();
        code = code_of(x);
        w = i32(width, "the width");
        xp = on.p(&x, dt, x.sizes(), name);
    }
    const void* like(const at::Tensor* t, const at::Tensor& x, const char* name) const { return on.p(t, dt, x.sizes(), name); }
    const void* param(const at::Tensor* t, const char* name) const { return on.p(t, dt, {width}, name); }
    at::Tensor workspace() const {
        const size_t n = qdelta_fused_norm_workspace_bytes(rows, w, code);
        if (n == 0) bad("unsupported or invalid shape for the norm");
        return on.make({(int64_t)n}, at::kByte);
    }
};
std::pair<at::Tensor, at::Tensor> gated_forward(const at::Tensor& x, const at::Tensor& gate, const at::Tensor* weight, const at::Tensor* bias,
                                                double eps, bool want_stats, unsigned flags) {
    const Fused c(x, "x");
    const void *gp = c.like(&gate, x, "gate"), *wp = c.param(weight, "weight"), *bp = c.param(bias, "bias");
    at::Tensor y = c.on.make(x.sizes(), c.dt), stats;
    if (want_stats) stats = c.on.make({2, c.rows}, at::kFloat);
    rc_check(qdelta_gated_norm_fwd(c.rows, c.w, c.code, c.xp, gp, wp, bp, y.data_ptr(), floats(stats), (float)eps, flags, stream()),
             "qdelta_gated_norm_fwd");
    return {y, stats};
}
struct GatedGrads { at::Tensor dx, dgate, dweight, dbias, params; };
GatedGrads gated_backward(const at::Tensor& x, const at::Tensor& gate, const at::Tensor* weight, const at::Tensor* bias, const at::Tensor& dy,
                          const at::Tensor& stats, bool want_dweight, bool want_dbias, unsigned flags) {
    const Fused c(x, "x");
    const void *zp = c.like(&gate, x, "gate"), *wp = c.param(weight, "weight"), *bp = c.param(bias, "bias"), *gp = c.like(&dy, x, "dy");
    const float* sp = c.on.f(&stats, {2, c.rows}, "stats");
    GatedGrads g;
    g.dx = c.on.make(x.sizes(), c.dt);
    g.dgate = c.on.make(x.sizes(), c.dt);
    at::Tensor ws;
    if (want_dweight || want_dbias || c.width > kNarrow) ws = c.workspace();
    Params params(c.on, {want_dweight ? c.width : 0, want_dbias ? c.width : 0});
    g.params = params.all;
    if (want_dweight) g.dweight = params.next({c.width});
    if (want_dbias) g.dbias = params.next({c.width});
    rc_check(qdelta_gated_norm_bwd(c.rows, c.w, c.code, c.xp, zp, wp, bp, gp, sp, g.dx.data_ptr(), g.dgate.data_ptr(), floats(g.dweight),
                                   floats(g.dbias), at_of(ws), ws.defined() ? (size_t)ws.numel() : 0, flags, stream()),
             "qdelta_gated_norm_bwd");
    return g;
}
struct AddedOut { at::Tensor y, total, stats; };
AddedOut added_forward(const at::Tensor& x, const at::Tensor& residual, const at::Tensor* scale, const at::Tensor* weight, const at::Tensor* bias,
                       double eps, bool want_stats, unsigned flags) {
    const Fused c(x, "x");
    const void *rp = c.like(&residual, x, "residual"), *cp = c.param(scale, "scale"), *wp = c.param(weight, "weight"), *bp = c.param(bias, "bias");
    AddedOut r;
    r.y = c.on.make(x.sizes(), c.dt);
    r.total = c.on.make(x.sizes(), c.dt);
    if (want_stats) r.stats = c.on.make({2, c.rows}, at::kFloat);
    rc_check(qdelta_add_norm_fwd(c.rows, c.w, c.code, c.xp, rp, cp, wp, bp, r.total.data_ptr(), r.y.data_ptr(), floats(r.stats), (float)eps, flags,
                                 stream()),
             "qdelta_add_norm_fwd");
    return r;
}
struct AddedGrads { at::Tensor dx, dresidual, dscale, dweight, dbias, params; };
AddedGrads added_backward(const at::Tensor& x, const at::Tensor& residual, const at::Tensor* scale, const at::Tensor* weight, const at::Tensor& dy,
                          const at::Tensor* dtotal, const at::Tensor& stats, bool want_dscale, bool want_dweight, bool want_dbias, unsigned flags) {
    const Fused c(x, "x");
    const void *rp = c.like(&residual, x, "residual"), *cp = c.param(scale, "scale"), *wp = c.param(weight, "weight"), *gp = c.like(&dy, x, "dy"),
               *tp = c.like(dtotal, x, "dtotal");
    const float* sp = c.on.f(&stats, {2, c.rows}, "stats");
    AddedGrads g;
    g.dresidual = c.on.make(x.sizes(), c.dt);
    g.dx = scale ? c.on.make(x.sizes(), c.dt) : g.dresidual;
    at::Tensor ws;
    if (want_dscale || want_dweight || want_dbias || c.width > kNarrow) ws = c.workspace();
    Params params(c.on, {want_dscale ? c.width : 0, want_dweight ? c.width : 0, want_dbias ? c.width : 0});
    g.params = params.all;
    if (want_dscale) g.dscale = params.next({c.width});
    if (want_dweight) g.dweight = params.next({c.width});
    if (want_dbias) g.dbias = params.next({c.width});
    rc_check(qdelta_add_norm_bwd(c.rows, c.w, c.code, c.xp, rp, cp, wp, gp, tp, sp, scale ? g.dx.data_ptr() : nullptr, g.dresidual.data_ptr(),
                                 floats(g.dscale), floats(g.dweight), floats(g.dbias), at_of(ws), ws.defined() ? (size_t)ws.numel() : 0, flags,
                                 stream()),
             "qdelta_add_norm_bwd");
    return g;
}

// ---- rotary positions -------------------------------------------------------------------------------------------------------
// out: NULL, or two tensors to write to (q and k themselves for a call in place)
std::pair<at::Tensor, at::Tensor> rotate(const at::Tensor& q, const at::Tensor* k, const at::Tensor& turns, const at::Tensor* positions,
                                         int64_t start, double scale, unsigned flags, const at::Tensor* q_out, const at::Tensor* k_out) {
    const On on(q, "q");
    dims(q, 4, "q must be [B, T, H, d]");
    dims(turns, 1, "turns must be [pairs]");
    const int64_t B = q.size(0), T = q.size(1), Hq = q.size(2), d = q.size(3), pairs = turns.size(0);
    const at::ScalarType dt = q.scalar_type();
    const int code = code_of(q);
    int64_t Hk = 0;
    if (k) {
        dims(*k, 4, "k must be [B, T, H, d]");
        Hk = k->size(2);
        if (Hk == 0) bad("k must have heads");
    } else if (k_out) {
        bad("an output for k needs k");
    }
    const void *qp = on.p(&q, dt, {B, T, Hq, d}, "q"), *kp = on.p(k, dt, {B, T, Hk, d}, "k");
    const void *tp = on.p(&turns, at::kLong, {pairs}, "turns"), *pp = on.p(positions, at::kLong, {B, T}, "positions");
    const at::Tensor qo = q_out ? *q_out : on.make(q.sizes(), dt);
    at::Tensor ko;
    if (k) ko = k_out ? *k_out : on.make(k->sizes(), dt);
    rc_check(qdelta_rotary(i32(B, "B"), i32(T, "T"), i32(Hq, "heads"), i32(Hk, "heads"), i32(d, "d"), i32(pairs, "pairs"), code, qp, kp,
                           static_cast<const long long*>(tp), static_cast<const long long*>(pp), (long long)start,
                           on.p(&qo, dt, {B, T, Hq, d}, "the output for q"), on.p(k ? &ko : nullptr, dt, {B, T, Hk, d}, "the output for k"),
                           (float)scale, flags, stream()),
             "qdelta_rotary");
    written(q_out);
    written(k_out);
    return {qo, ko};
}

// ---- calls from Python ----------------------------------------------------------------------------------------------------
double to_double(PyObject* o) {
    const double v = PyFloat_AsDouble(o);
    if (PyErr_Occurred()) throw Raised{};
    return v;
}
int64_t to_int64(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (PyErr_Occurred()) throw Raised{};
    return v;
}
// linear_fwd(q, k, v, log_decay, h0, workspace, want_hT, scale) -> (o, hT, workspace)
PyObject* linear_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 8)) return nullptr;
    return called([&] {
        const at::Tensor &q = needed(a[0], "q"), &k = needed(a[1], "k"), &v = needed(a[2], "v"), &g = needed(a[3], "log_decay");
        const at::Tensor *h0 = tensor(a[4], "h0"), *ws = tensor(a[5], "workspace");
        const double scale = to_double(a[7]);
        const LinearOut r = unlocked([&] { return linear_forward(q, k, v, g, h0, ws, a[6] == Py_True, scale); });
        return tuple({r.o, r.hT, r.ws});
    });
}
// linear_bwd(q, k, v, log_decay, h0, dO, dhT, workspace, want_dh0, scale) -> {dq, dk, dv, dh0}
PyObject* linear_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 10)) return nullptr;
    return called([&] {
        const at::Tensor &q = needed(a[0], "q"), &k = needed(a[1], "k"), &v = needed(a[2], "v"), &g = needed(a[3], "log_decay"),
                         &dO = needed(a[5], "dO");
        const at::Tensor *h0 = tensor(a[4], "h0"), *dhT = tensor(a[6], "dhT"), *ws = tensor(a[7], "workspace");
        const double scale = to_double(a[9]);
        const LinearGrads r = unlocked([&] { return linear_backward(q, k, v, g, h0, dO, dhT, ws, a[8] == Py_True, scale); });
        return dict({{"dq", r.dq}, {"dk", r.dk}, {"dv", r.dv}, {"dh0", r.dh0}});
    });
}
// linear_steps(q, k, v, log_decay, state, o, scale) -> o
PyObject* linear_steps(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    return called([&] {
        const at::Tensor &q = needed(a[0], "q"), &k = needed(a[1], "k"), &v = needed(a[2], "v"), &g = needed(a[3], "log_decay"),
                         &state = needed(a[4], "state");
        const at::Tensor* given = tensor(a[5], "o");
        const double scale = to_double(a[6]);
        const at::Tensor o = unlocked([&] {
            const Linear c(q, k, v, g);
            float* sp = c.state(&state, "state");
            const at::Tensor r = given ? *given : c.on.make({c.B, c.T, c.H, c.dv}, c.dt);
            rc_check(qdelta_linear_steps(&c.s, c.q, c.k, c.v, c.g, sp, c.on.p(&r, c.dt, {c.B, c.T, c.H, c.dv}, "o"), (float)scale, 0, stream()),
                     "qdelta_linear_steps");
            written(&state);
            written(given);
            return r;
        });
        return given ? own(a[5]) : wrapped(o);
    });
}
// gated_norm_fwd(x, gate, weight, bias, eps, want_stats, flags) -> (y, stats)
PyObject* gated_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &gate = needed(a[1], "gate");
        const at::Tensor *weight = tensor(a[2], "weight"), *bias = tensor(a[3], "bias");
        const double eps = to_double(a[4]);
        const unsigned flags = to_flags(a[6]);
        const auto r = unlocked([&] { return gated_forward(x, gate, weight, bias, eps, a[5] == Py_True, flags); });
        return tuple({r.first, r.second});
    });
}
// gated_norm_bwd(x, gate, weight, bias, dy, stats, want_dweight, want_dbias, flags) -> {dx, dgate, dweight, dbias}
PyObject* gated_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 9)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &gate = needed(a[1], "gate"), &dy = needed(a[4], "dy"), &stats = needed(a[5], "stats");
        const at::Tensor *weight = tensor(a[2], "weight"), *bias = tensor(a[3], "bias");
        const unsigned flags = to_flags(a[8]);
        const GatedGrads g = unlocked([&] { return gated_backward(x, gate, weight, bias, dy, stats, a[6] == Py_True, a[7] == Py_True, flags); });
        return dict({{"dx", g.dx}, {"dgate", g.dgate}, {"dweight", g.dweight}, {"dbias", g.dbias}});
    });
}
// add_norm_fwd(x, residual, scale, weight, bias, eps, want_stats, flags) -> (y, total, stats)
PyObject* add_norm_fwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 8)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &residual = needed(a[1], "residual");
        const at::Tensor *scale = tensor(a[2], "scale"), *weight = tensor(a[3], "weight"), *bias = tensor(a[4], "bias");
        const double eps = to_double(a[5]);
        const unsigned flags = to_flags(a[7]);
        const AddedOut r = unlocked([&] { return added_forward(x, residual, scale, weight, bias, eps, a[6] == Py_True, flags); });
        return tuple({r.y, r.total, r.stats});
    });
}
// add_norm_bwd(x, residual, scale, weight, dy, dtotal, stats, want_dscale, want_dweight, want_dbias, flags) -> {dx, dresidual, dscale, dweight, dbias}
PyObject* add_norm_bwd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 11)) return nullptr;
    return called([&] {
        const at::Tensor &x = needed(a[0], "x"), &residual = needed(a[1], "residual"), &dy = needed(a[4], "dy"), &stats = needed(a[6], "stats");
        const at::Tensor *scale = tensor(a[2], "scale"), *weight = tensor(a[3], "weight"), *dtotal = tensor(a[5], "dtotal");
        const unsigned flags = to_flags(a[10]);
        const AddedGrads g = unlocked([&] {
            return added_backward(x, residual, scale, weight, dy, dtotal, stats, a[7] == Py_True, a[8] == Py_True, a[9] == Py_True, flags);
        });
        return dict({{"dx", g.dx}, {"dresidual", g.dresidual}, {"dscale", g.dscale}, {"dweight", g.dweight}, {"dbias", g.dbias}});
    });
}
// rotary(q, k, turns, positions, start, scale, flags, q_out, k_out) -> (q', k')
PyObject* rotary(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 9)) return nullptr;
    return called([&] {
        const at::Tensor &q = needed(a[0], "q"), &turns = needed(a[2], "turns");
        const at::Tensor *k = tensor(a[1], "k"), *positions = tensor(a[3], "positions"), *qo = tensor(a[7], "q_out"), *ko = tensor(a[8], "k_out");
        const int64_t start = to_int64(a[4]);
        const double scale = to_double(a[5]);
        const unsigned flags = to_flags(a[6]);
        const auto r = unlocked([&] { return rotate(q, k, turns, positions, start, scale, flags, qo, ko); });
        return tuple({r.first, r.second});
    });
}

// ---- autograd ---------------------------------------------------------------------------------------------------------------
struct LinearNode : torch::autograd::Function<LinearNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& q, const at::Tensor& k, const at::Tensor& v, const at::Tensor& g,
                                 const MaybeTensor& h0, double scale, bool need_grad) {
        const LinearOut r = linear_forward(q, k, v, g, maybe(h0), nullptr, true, scale);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            ctx->save_for_backward({q, k, v, g, or_none(h0)});
            ctx->saved_data["scale"] = scale;
            ctx->saved_data["dh0"] = h0 && h0->requires_grad();
        }
        return {r.o, r.hT};
    }
    static variable_list backward(AutogradContext* ctx, variable_list up) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            static const char* names[4] = {"q", "k", "v", "log_decay"};
            for (int i = 0; i < 4; ++i) present(in[i], names[i]);
            const at::Tensor &v = in[2], &h0 = in[4];
            const at::Tensor dO = or_zeros(upstream(up[0], v.scalar_type()), v), dhT = upstream(up[1], at::kFloat);
            const LinearGrads r = linear_backward(in[0], in[1], v, in[3], given(h0), dO, given(dhT), nullptr,
                                                  h0.defined() && ctx->saved_data["dh0"].toBool(), ctx->saved_data["scale"].toDouble());
            return {r.dq, r.dk, r.dv, at::Tensor(), r.dh0, at::Tensor(), at::Tensor()};
        });
    }
};

struct GatedNode : torch::autograd::Function<GatedNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const at::Tensor& gate, const MaybeTensor& weight,
                                 const MaybeTensor& bias, double eps, int64_t flags, bool need_grad) {
        const auto r = gated_forward(x, gate, maybe(weight), maybe(bias), eps, need_grad, (unsigned)flags);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            ctx->save_for_backward({x, gate, or_none(weight), or_none(bias), r.second});
            ctx->saved_data["flags"] = flags;
            ctx->saved_data["dweight"] = weight && weight->requires_grad();
            ctx->saved_data["dbias"] = bias && bias->requires_grad();
        }
        return {r.first};
    }
    static variable_list backward(AutogradContext* ctx, variable_list up) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            const at::Tensor &x = in[0], &gate = in[1], &weight = in[2], &bias = in[3], &stats = in[4];
            present(x, "x");
            present(gate, "gate");
            present(stats, "the saved statistics");
            const at::Tensor dy = or_zeros(upstream(up[0], x.scalar_type()), x);
            const GatedGrads r = gated_backward(x, gate, given(weight), given(bias), dy, stats, weight.defined() && ctx->saved_data["dweight"].toBool(),
                                                bias.defined() && ctx->saved_data["dbias"].toBool(), (unsigned)ctx->saved_data["flags"].toInt());
            at::Tensor converted;
            return {r.dx, r.dgate, as(r.dweight, x, r.params, converted), as(r.dbias, x, r.params, converted), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};

struct AddedNode : torch::autograd::Function<AddedNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& x, const at::Tensor& residual, const MaybeTensor& scale,
                                 const MaybeTensor& weight, const MaybeTensor& bias, double eps, int64_t flags, bool need_grad) {
        const AddedOut r = added_forward(x, residual, maybe(scale), maybe(weight), maybe(bias), eps, need_grad, (unsigned)flags);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            const bool dscale = scale && scale->requires_grad();
            ctx->save_for_backward({x, residual, or_none(scale), or_none(weight), r.stats});
            ctx->saved_data["flags"] = flags;
            ctx->saved_data["dscale"] = dscale;
            ctx->saved_data["dweight"] = weight && weight->requires_grad();
            ctx->saved_data["dbias"] = bias && bias->requires_grad();
        }
        return {r.y, r.total};
    }
    static variable_list backward(AutogradContext* ctx, variable_list up) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            const at::Tensor &x = in[0], &residual = in[1], &scale = in[2], &weight = in[3], &stats = in[4];
            present(x, "x");
            present(residual, "residual");
            present(stats, "the saved statistics");
            const at::Tensor dy = or_zeros(upstream(up[0], x.scalar_type()), x), dtotal = upstream(up[1], x.scalar_type());
            const bool dscale = scale.defined() && ctx->saved_data["dscale"].toBool();
            const AddedGrads r = added_backward(x, residual, given(scale), given(weight), dy, given(dtotal), stats, dscale,
                                                weight.defined() && ctx->saved_data["dweight"].toBool(), ctx->saved_data["dbias"].toBool(),
                                                (unsigned)ctx->saved_data["flags"].toInt());
            at::Tensor converted;
            return {r.dx, r.dresidual, as(r.dscale, x, r.params, converted), as(r.dweight, x, r.params, converted),
                    as(r.dbias, x, r.params, converted), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};

struct RotaryNode : torch::autograd::Function<RotaryNode> {
    static variable_list forward(AutogradContext* ctx, const at::Tensor& q, const MaybeTensor& k, const at::Tensor& turns,
                                 const MaybeTensor& positions, int64_t start, double scale, int64_t flags, bool need_grad) {
        const auto r = rotate(q, maybe(k), turns, maybe(positions), start, scale, (unsigned)flags, nullptr, nullptr);
        ctx->set_materialize_grads(false);
        if (need_grad) {
            ctx->save_for_backward({turns, or_none(positions)});
            ctx->saved_data["start"] = start;
            ctx->saved_data["scale"] = scale;
            ctx->saved_data["flags"] = flags;
            ctx->saved_data["type"] = (int64_t)q.scalar_type();
        }
        return r.second.defined() ? variable_list{r.first, r.second} : variable_list{r.first};
    }
    static variable_list backward(AutogradContext* ctx, variable_list up) {
        return in_backward([&]() -> variable_list {
            const variable_list in = ctx->get_saved_variables();
            const at::Tensor &turns = in[0], &positions = in[1];
            present(turns, "turns");
            const auto type = (at::ScalarType)ctx->saved_data["type"].toInt();
            at::Tensor dq = upstream(up[0], type), dk = up.size() > 1 ? upstream(up[1], type) : at::Tensor();
            const auto back = [&](const at::Tensor& a, const at::Tensor* b) {
                return rotate(a, b, turns, given(positions), ctx->saved_data["start"].toInt(), ctx->saved_data["scale"].toDouble(),
                              (unsigned)ctx->saved_data["flags"].toInt() ^ QD_INVERSE, nullptr, nullptr);
            };
            if (dq.defined()) std::tie(dq, dk) = back(dq, given(dk));
            else if (dk.defined()) dk = back(dk, nullptr).first;
            return {dq, dk, at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor(), at::Tensor()};
        });
    }
};

// linear_autograd(q, k, v, log_decay, h0, scale) -> (o, hT)
PyObject* linear_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    return called([&] {
        MaybeTensor t[5];
        if (at::GradMode::is_enabled() && needed(a[3], "log_decay").requires_grad())
            bad("log_decay is a constant of the layer and has no gradient: pass log_decay.detach()");
        const bool need = inputs(a, {"q", "k", "v", "log_decay", "h0"}, 4, t);
        const double scale = to_double(a[5]);
        const variable_list r = LinearNode::apply(*t[0], *t[1], *t[2], *t[3], t[4], scale, need);
        return tuple({r[0], r[1]});
    });
}
// gated_norm_autograd(x, gate, weight, bias, eps, flags) -> y
PyObject* gated_norm_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 6)) return nullptr;
    return called([&] {
        MaybeTensor t[4];
        const bool need = inputs(a, {"x", "gate", "weight", "bias"}, 2, t);
        const double eps = to_double(a[4]);
        return wrapped(GatedNode::apply(*t[0], *t[1], t[2], t[3], eps, (int64_t)to_flags(a[5]), need)[0]);
    });
}
// add_norm_autograd(x, residual, scale, weight, bias, eps, flags) -> (y, total)
PyObject* add_norm_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    return called([&] {
        MaybeTensor t[5];
        const bool need = inputs(a, {"x", "residual", "scale", "weight", "bias"}, 2, t);
        const double eps = to_double(a[5]);
        const variable_list r = AddedNode::apply(*t[0], *t[1], t[2], t[3], t[4], eps, (int64_t)to_flags(a[6]), need);
        return tuple({r[0], r[1]});
    });
}
// rotary_autograd(q, k, turns, positions, start, scale, flags) -> (q', k')
PyObject* rotary_autograd(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (!arity(n, 7)) return nullptr;
    return called([&] {
        MaybeTensor q[1], k[1];
        bool need = inputs(a, {"q"}, 1, q);
        need = inputs(a + 1, {"k"}, 0, k) || need;
        const at::Tensor turns = usable(needed(a[2], "turns"));
        MaybeTensor positions;
        if (const at::Tensor* p = tensor(a[3], "positions")) positions = usable(*p);
        const int64_t start = to_int64(a[4]);
        const double scale = to_double(a[5]);
        const variable_list r = RotaryNode::apply(*q[0], k[0], turns, positions, start, scale, (int64_t)to_flags(a[6]), need);
        return tuple({r[0], r.size() > 1 ? r[1] : at::Tensor()});
    });
}

}  // namespace

#define QD_METHOD(name) {#name, (PyCFunction)(void*)name, METH_FASTCALL, nullptr}
PyMethodDef linear_methods[] = {
    QD_METHOD(linear_fwd), QD_METHOD(linear_bwd), QD_METHOD(linear_steps), QD_METHOD(gated_norm_fwd), QD_METHOD(gated_norm_bwd),
    QD_METHOD(add_norm_fwd), QD_METHOD(add_norm_bwd), QD_METHOD(rotary), QD_METHOD(linear_autograd), QD_METHOD(gated_norm_autograd),
    QD_METHOD(add_norm_autograd), QD_METHOD(rotary_autograd),
    {nullptr, nullptr, 0, nullptr},
};

}  // namespace qdhost

// C-ABI entry points: argument validation, workspace carving, kernel sequencing.
#include "internal.h"

#include <vector>

namespace qd {

static size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

WsLayout ws_layout(const qd_shape& s) {
    WsLayout L{};
    const size_t BH = (size_t)s.B * s.H, T = (size_t)split_padded_T(s), N = T / kChunk;
    const size_t io = s.dtype == QD_BF16 ? 2 : 4;
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off = align256(off + bytes); return o; };
    L.status = take(256);
    L.g = take(BH * T * 4);
    L.P = take(BH * T * kChunk * io);
    L.W = take(BH * T * s.dk * io);
    L.U = take(BH * T * s.dv * io);
    L.rqk = take(2 * BH * T * 4);
    L.fwd_end = off;
    L.slice = split_slice(s);
    L.M = take(BH * N * kChunk * kChunk * 4);
    L.hs = take(BH * N * s.dk * s.dv * 4);
    L.D = take(BH * T * s.dv * io);
    L.dhs = take(BH * N * s.dk * s.dv * 4);
    L.dD = take(BH * T * s.dv * io);
    L.kdhd = take((size_t)(s.dv / L.slice) * BH * T * 4);
    L.dhh = take((size_t)(s.dv / L.slice) * BH * N * 4);
    L.bwd_end = off;
    return L;
}

int check_shape(const qd_shape* s) {
    if (!s) return QD_ERR_INVALID_ARG;
    if (s->B <= 0 || s->T <= 0 || s->H <= 0 || s->dk <= 0 || s->dv <= 0 || s->chunk <= 0) return QD_ERR_INVALID_ARG;
    if (s->dtype != QD_F32 && s->dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if (s->chunk != kChunk) return QD_ERR_UNSUPPORTED;
    if ((s->dk != 64 && s->dk != 128) || (s->dv != 64 && s->dv != 128)) return QD_ERR_UNSUPPORTED;
    if (s->T > 0x7fffffff - 127) return QD_ERR_UNSUPPORTED;          // T is rounded up to 64 or 128 in 32 bits
    if ((long long)s->B * s->H * ((s->T + 127) / 128 * 2) > 0x7fffffffLL / 4) return QD_ERR_UNSUPPORTED;
    // bf16 128 x 128 has the tcgen05 kernels alone: split_bf16.cu has none for it
    if (s->dtype == QD_BF16 && s->dk == 128 && s->dv == 128 && !tc_supported(*s)) return QD_ERR_UNSUPPORTED;
    return QD_OK;
}

static bool misaligned(const void* p) { return ((uintptr_t)p & 15) != 0; }

// ---- optional per-stage timing with CUDA events on the launching stream ------------------------
enum Stage { ST_PREP = 0, ST_CHAIN_FWD, ST_CHAIN_BWD, ST_CHUNK_BWD, ST_DECODE, ST_CONV, ST_SCAN, ST_NORM, ST_LINEAR, ST_ROTARY, ST_COUNT };
static const char* kStageNames[ST_COUNT] = {"prep", "chain_fwd", "chain_bwd", "chunk_bwd", "decode", "conv", "scan", "norm", "linear", "rotary"};
struct Pending { cudaEvent_t a, b; int stage; };
static bool g_profile = false;
static std::vector<Pending> g_pending;
static std::vector<cudaEvent_t> g_pool;
static double g_ms[ST_COUNT];
static long long g_launches[ST_COUNT];

static cudaEvent_t get_event() {
    cudaEvent_t e = nullptr;
    if (!g_pool.empty()) { e = g_pool.back(); g_pool.pop_back(); return e; }
    if (cudaEventCreate(&e) != cudaSuccess) return nullptr;
    return e;
}

// Brackets one kernel launch (of the operators around the delta rule: one call) with two events when profiling is on.
struct StageTimer {
    cudaEvent_t a = nullptr, b = nullptr;
    int stage; cudaStream_t s;
    StageTimer(int stage_, cudaStream_t s_) : stage(stage_), s(s_) {
        if (!g_profile) return;
        a = get_event(); b = get_event();
        if (a && b) cudaEventRecord(a, s);
    }
    ~StageTimer() {
        if (!g_profile || !a || !b) return;
        cudaEventRecord(b, s);
        g_pending.push_back({a, b, stage});
    }
};

template <class F> static cudaError_t timed(int stage, cudaStream_t s, F f) {
    StageTimer t(stage, s);
    return f();
}

// Kernels are timed one by one, so in one part.
static int fwd_parts(const ChunkArgs& a) { return g_profile ? 1 : tc_fwd_parts(a); }
static int bwd_parts(const ChunkArgs& a) { return g_profile ? 1 : tc_bwd_parts(a); }

// The two kernels of the forward, beside each other in parts where that is faster.
static cudaError_t tc_forward(const ChunkArgs& a) {
    const int parts = fwd_parts(a);
    if (parts > 1) return tc_fwd(a, parts);
    const cudaError_t e = timed(ST_PREP, a.stream, [&] { return tc_prep(a); });
    return e != cudaSuccess ? e : timed(ST_CHAIN_FWD, a.stream, [&] { return tc_chain_fwd(a); });
}
// The two of the backward, likewise.
static cudaError_t tc_backward(const ChunkArgs& a) {
    const int parts = bwd_parts(a);
    if (parts > 1) return tc_bwd(a, parts);
    const cudaError_t e = timed(ST_CHAIN_BWD, a.stream, [&] { return tc_chain_bwd(a); });
    return e != cudaSuccess ? e : timed(ST_CHUNK_BWD, a.stream, [&] { return tc_chunk_bwd(a); });
}

// ---- operators around the delta rule: what a shape has to satisfy ---------------------------------------------------
constexpr long long kMostElements = 1LL << 37;             // of a tensor; what fits the GPU's memory is below it, and grids fit 31 bits
static int check_conv(int B, int T, int D, int W, int dtype) {
    if (B <= 0 || T <= 0 || D <= 0 || W <= 0) return QD_ERR_INVALID_ARG;
    if (dtype != QD_F32 && dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if (W < 2 || W > 4 || T > 1 << 30 || D > 1 << 20) return QD_ERR_UNSUPPORTED;
    if ((long long)B * T > kMostElements / D) return QD_ERR_UNSUPPORTED;
    return QD_OK;
}
static int check_scan(const qd_scan_shape* s) {
    if (!s || s->B <= 0 || s->T <= 0 || s->D <= 0 || s->N <= 0 || s->G <= 0) return QD_ERR_INVALID_ARG;
    if (s->dtype != QD_F32 && s->dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if (s->N > 64 || s->T > 1 << 30 || s->D > 1 << 20 || s->D % s->G) return QD_ERR_UNSUPPORTED;
    if ((long long)s->B * s->D > 1LL << 30 || (long long)s->B * s->T > kMostElements / ((long long)s->G * s->N) ||
        (long long)s->B * s->T > kMostElements / s->D)
        return QD_ERR_UNSUPPORTED;
    return QD_OK;
}
static int check_norm(long long rows, int width, int dtype) {
    if (rows <= 0 || width <= 0) return QD_ERR_INVALID_ARG;
    if (dtype != QD_F32 && dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if (width > 16384 || rows > kMostElements / 4 || rows > kMostElements / width) return QD_ERR_UNSUPPORTED;
    return QD_OK;
}
static int check_linear(const qd_linear_shape* s) {
    if (!s || s->B <= 0 || s->T <= 0 || s->H <= 0 || s->dk <= 0 || s->dv <= 0) return QD_ERR_INVALID_ARG;
    if (s->dtype != QD_F32 && s->dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if ((s->dk != 64 && s->dk != 128) || (s->dv != 64 && s->dv != 128)) return QD_ERR_UNSUPPORTED;
    // states, and with them CTAs of a walk, fit 31 bits whatever they are split into
    if (s->T > 1 << 30 || s->H > 1 << 20 || (long long)s->B * s->H > 1 << 23 || (long long)s->B * s->T > kMostElements / 128 / s->H)
        return QD_ERR_UNSUPPORTED;
    return QD_OK;
}
static bool finite(float x) { return x - x == 0.f; }
static int check_rotary(int B, int T, int Hq, int Hk, int d, int pairs, int dtype) {
    if (B <= 0 || T <= 0 || Hq <= 0 || Hk < 0 || d <= 0 || pairs <= 0) return QD_ERR_INVALID_ARG;
    if (dtype != QD_F32 && dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if (d > 1024 || pairs > d / 2 || Hq > 1 << 16 || Hk > 1 << 16) return QD_ERR_UNSUPPORTED;
    // tokens: CTAs fit 31 bits with one token each
    if ((long long)B * T > 0x7fffffffLL || (long long)B * T > kMostElements / d / (Hq > Hk ? Hq : Hk)) return QD_ERR_UNSUPPORTED;
    return QD_OK;
}
template <size_t N> static bool any_misaligned(const void* const (&ptrs)[N]) {
    for (const void* p : ptrs)
        if (p && misaligned(p)) return true;
    return false;
}

}  // namespace qd

using namespace qd;

extern "C" {

size_t qdelta_chunk_workspace_bytes(const qd_shape* shape, int for_backward) {
    if (check_shape(shape) != QD_OK) return 0;
    // the tensor-core path and the fp32 path lay the workspace out differently; a shape takes exactly one of them
    if (tc_supported(*shape)) {
        TcLayout TL = tc_layout(*shape);
        return for_backward ? TL.bwd_end : TL.fwd_end;
    }
    WsLayout L = ws_layout(*shape);
    return for_backward ? L.bwd_end : L.fwd_end;
}

int qdelta_chunk_path(const qd_shape* shape) {
    if (check_shape(shape) != QD_OK) return -1;
    return tc_supported(*shape) ? 1 : 0;
}

int qdelta_chunk_parts(const qd_shape* shape, int backward) {
    if (check_shape(shape) != QD_OK) return -1;
    if (!tc_supported(*shape)) return 1;
    ChunkArgs a{};
    a.s = *shape;
    a.save = true;
    return backward ? bwd_parts(a) : fwd_parts(a);
}

int qdelta_chunk_fwd(const qd_shape* shape, const void* q, const void* k, const void* v, const void* beta,
                     const void* alpha, const void* lambda, const float* h0, void* o, float* hT,
                     void* workspace, size_t workspace_bytes, unsigned flags, qd_stream stream) {
    int rc = check_shape(shape);
    if (rc != QD_OK) return rc;
    if (!q || !k || !v || !beta || !o) return QD_ERR_INVALID_ARG;
    const void* ptrs[] = {q, k, v, h0, o, hT, workspace};
    for (const void* p : ptrs)
        if (p && misaligned(p)) return QD_ERR_INVALID_ARG;
    const void* coef[] = {beta, alpha, lambda};
    for (const void* p : coef)
        if (p && ((uintptr_t)p & (shape->dtype == QD_BF16 ? 1 : 3))) return QD_ERR_INVALID_ARG;
    if (flags & ~(unsigned)(QD_FWD_SAVE_FOR_BWD | QD_COEF_LOGITS | QD_NORM_QK)) return QD_ERR_INVALID_ARG;
    ChunkArgs a{};
    a.s = *shape;
    a.L = ws_layout(*shape);
    a.save = (flags & QD_FWD_SAVE_FOR_BWD) != 0;
    a.logits = (flags & QD_COEF_LOGITS) != 0;
    a.norm = (flags & QD_NORM_QK) != 0;
    if (!workspace || workspace_bytes < qdelta_chunk_workspace_bytes(shape, a.save ? 1 : 0)) return QD_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.beta = beta; a.alpha = alpha; a.lam = lambda; a.h0 = h0; a.o = o; a.hT = hT;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    if (tc_supported(*shape)) {
        a.TL = tc_layout(*shape);
        if (tc_forward(a) != cudaSuccess) return QD_ERR_CUDA;
        return QD_OK;
    }
    if (timed(ST_PREP, a.stream, [&] { return split_prep(a); }) != cudaSuccess) return QD_ERR_CUDA;
    if (timed(ST_CHAIN_FWD, a.stream, [&] { return split_chain_fwd(a); }) != cudaSuccess) return QD_ERR_CUDA;
    return QD_OK;
}

int qdelta_chunk_bwd(const qd_shape* shape, const void* q, const void* k, const void* v, const void* beta,
                     const void* alpha, const void* lambda, const float* h0, const void* dO, const float* dhT,
                     void* dq, void* dk, void* dv, float* dbeta, float* dalpha, float* dlambda, float* dh0,
                     void* workspace, size_t workspace_bytes, unsigned flags, qd_stream stream) {
    int rc = check_shape(shape);
    if (rc != QD_OK) return rc;
    if (!q || !k || !v || !beta || !dO || !dq || !dk || !dv || !dbeta) return QD_ERR_INVALID_ARG;
    if ((alpha && !dalpha) || (lambda && !dlambda)) return QD_ERR_INVALID_ARG;
    const void* ptrs[] = {q, k, v, h0, dO, dhT, dq, dk, dv, dh0, workspace};
    for (const void* p : ptrs)
        if (p && misaligned(p)) return QD_ERR_INVALID_ARG;
    const void* coef[] = {beta, alpha, lambda};
    for (const void* p : coef)
        if (p && ((uintptr_t)p & (shape->dtype == QD_BF16 ? 1 : 3))) return QD_ERR_INVALID_ARG;
    const void* gcoef[] = {dbeta, dalpha, dlambda};
    for (const void* p : gcoef)
        if (p && ((uintptr_t)p & 3)) return QD_ERR_INVALID_ARG;
    if (flags & ~(unsigned)(QD_BWD_REUSE_FWD | QD_COEF_LOGITS | QD_NORM_QK)) return QD_ERR_INVALID_ARG;
    ChunkArgs a{};
    a.s = *shape;
    a.L = ws_layout(*shape);
    a.save = true;
    a.logits = (flags & QD_COEF_LOGITS) != 0;
    a.norm = (flags & QD_NORM_QK) != 0;
    if (!workspace || workspace_bytes < qdelta_chunk_workspace_bytes(shape, 1)) return QD_ERR_WORKSPACE;
    a.q = q; a.k = k; a.v = v; a.beta = beta; a.alpha = alpha; a.lam = lambda; a.h0 = h0;
    a.dO = dO; a.dhT = dhT; a.dq = dq; a.dk = dk; a.dv = dv;
    a.dbeta = dbeta; a.dalpha = dalpha; a.dlam = dlambda; a.dh0 = dh0;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    if (tc_supported(*shape)) {
        a.TL = tc_layout(*shape);
        if (!(flags & QD_BWD_REUSE_FWD)) {
            // recompute what a saving forward leaves behind; its o goes to the dDelta section, which
            // the reverse chain overwrites afterwards
            a.o = a.ws + a.TL.dDt;
            a.hT = nullptr;
            if (tc_forward(a) != cudaSuccess) return QD_ERR_CUDA;
            a.own_predecessor = true;      // the reverse chain follows this library's forward chain in the stream
        }
        return tc_backward(a) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
    }
    if (!(flags & QD_BWD_REUSE_FWD)) {
        // recompute the forward intermediates (outputs of the forward itself are not rewritten:
        // o goes to the dD section, which the reverse chain overwrites afterwards)
        a.o = a.ws + a.L.dD;
        a.hT = nullptr;
        if (timed(ST_PREP, a.stream, [&] { return split_prep(a); }) != cudaSuccess) return QD_ERR_CUDA;
        if (timed(ST_CHAIN_FWD, a.stream, [&] { return split_chain_fwd(a); }) != cudaSuccess) return QD_ERR_CUDA;
    }
    if (timed(ST_CHAIN_BWD, a.stream, [&] { return split_chain_bwd(a); }) != cudaSuccess) return QD_ERR_CUDA;
    if (timed(ST_CHUNK_BWD, a.stream, [&] { return split_chunk_bwd(a); }) != cudaSuccess) return QD_ERR_CUDA;
    return QD_OK;
}

int qdelta_recurrent_step(int B, int H, int dk, int dv, int dtype, const void* q, const void* k, const void* v,
                          const void* beta, const void* alpha, const void* lambda, float* state, void* o,
                          qd_stream stream) {
    if (B <= 0 || H <= 0) return QD_ERR_INVALID_ARG;
    if (dtype != QD_F32 && dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if ((dk != 64 && dk != 128) || (dv != 64 && dv != 128)) return QD_ERR_UNSUPPORTED;
    if (!q || !k || !v || !beta || !state || !o) return QD_ERR_INVALID_ARG;
    if ((long long)B * H > 0x3fffffffLL) return QD_ERR_UNSUPPORTED;
    const void* ptrs[] = {q, k, v, state};
    for (const void* p : ptrs)
        if (p && misaligned(p)) return QD_ERR_INVALID_ARG;
    const void* coef[] = {beta, alpha, lambda, o};
    for (const void* p : coef)
        if (p && ((uintptr_t)p & (dtype == QD_BF16 ? 1 : 3))) return QD_ERR_INVALID_ARG;
    if (timed(ST_DECODE, (cudaStream_t)stream, [&] {
            return decode_steps(B, 1, H, dk, dv, dtype, q, k, v, beta, alpha, lambda, state, o, false, false, false, (cudaStream_t)stream);
        }) != cudaSuccess)
        return QD_ERR_CUDA;
    return QD_OK;
}

int qdelta_recurrent_steps(int B, int S, int H, int dk, int dv, int dtype, const void* q, const void* k, const void* v,
                           const void* beta, const void* alpha, const void* lambda, void* state, void* o,
                           unsigned flags, qd_stream stream) {
    if (B <= 0 || H <= 0 || S <= 0) return QD_ERR_INVALID_ARG;
    if (flags & ~(unsigned)(QD_COEF_LOGITS | QD_NORM_QK | QD_STATE_BF16)) return QD_ERR_INVALID_ARG;
    if (dtype != QD_F32 && dtype != QD_BF16) return QD_ERR_UNSUPPORTED;
    if ((dk != 64 && dk != 128) || (dv != 64 && dv != 128)) return QD_ERR_UNSUPPORTED;
    if (!q || !k || !v || !beta || !state || !o) return QD_ERR_INVALID_ARG;
    if ((long long)B * H > 0x3fffffffLL || (long long)B * S * H > 0x7fffffffLL / 128) return QD_ERR_UNSUPPORTED;
    const void* ptrs[] = {q, k, v, state};
    for (const void* p : ptrs)
        if (p && misaligned(p)) return QD_ERR_INVALID_ARG;
    const void* coef[] = {beta, alpha, lambda, o};
    for (const void* p : coef)
        if (p && ((uintptr_t)p & (dtype == QD_BF16 ? 1 : 3))) return QD_ERR_INVALID_ARG;
    if (timed(ST_DECODE, (cudaStream_t)stream, [&] {
            return decode_steps(B, S, H, dk, dv, dtype, q, k, v, beta, alpha, lambda, state, o,
                                (flags & QD_COEF_LOGITS) != 0, (flags & QD_NORM_QK) != 0, (flags & QD_STATE_BF16) != 0,
                                (cudaStream_t)stream);
        }) != cudaSuccess)
        return QD_ERR_CUDA;
    return QD_OK;
}

int qdelta_conv_fwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state,
                    void* y, void* last, unsigned flags, qd_stream stream) {
    const int rc = check_conv(B, T, D, W, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !w || !y || y == x || (last && last == state)) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, w, bias, state, y, last};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_SILU)) return QD_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = timed(ST_CONV, s, [&] { return conv_fwd(B, T, D, W, dtype, x, w, bias, state, y, last, (flags & QD_SILU) != 0, s); });
    return e == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_conv_steps(int B, int S, int D, int W, int dtype, const void* x, const void* w, const void* bias, void* state, void* y,
                      unsigned flags, qd_stream stream) {
    const int rc = check_conv(B, S, D, W, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !w || !state || !y || y == x) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, w, bias, state, y};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_SILU)) return QD_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = timed(ST_CONV, s, [&] { return conv_fwd(B, S, D, W, dtype, x, w, bias, state, y, state, (flags & QD_SILU) != 0, s); });
    return e == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

size_t qdelta_conv_workspace_bytes(int B, int T, int D, int W, int dtype) {
    return check_conv(B, T, D, W, dtype) == QD_OK ? conv_bwd_workspace(B, T, D, W) : 0;
}

int qdelta_conv_bwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state,
                    const void* dy, const void* dlast, void* dx, float* dw, float* dbias, void* dstate, void* workspace,
                    size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_conv(B, T, D, W, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !w || !dy || !dx || !dw || (bias && !dbias) || dx == x || dx == dy || (dstate && dstate == dlast)) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, w, bias, state, dy, dlast, dx, dw, dbias, dstate, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_SILU)) return QD_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < conv_bwd_workspace(B, T, D, W)) return QD_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = timed(ST_CONV, s, [&] {
        return conv_bwd(B, T, D, W, dtype, x, w, bias, state, dy, dlast, dx, dw, dbias, dstate, (float*)workspace, (flags & QD_SILU) != 0, s);
    });
    return e == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

size_t qdelta_scan_workspace_bytes(const qd_scan_shape* shape, int for_backward) {
    if (check_scan(shape) != QD_OK) return 0;
    return for_backward ? scan_bwd_workspace(*shape) : scan_fwd_workspace(*shape, false);
}

int qdelta_scan_fwd(const qd_scan_shape* shape, const void* u, const void* dt, const float* A, const void* Bm, const void* Cm,
                    const float* D, const void* z, const float* dt_bias, const float* h0, void* y, float* hT, void* workspace,
                    size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_scan(shape);
    if (rc != QD_OK) return rc;
    if (!u || !dt || !A || !Bm || !Cm || !y || (hT && hT == h0)) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {u, dt, A, Bm, Cm, D, z, dt_bias, h0, y, hT, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)(QD_SOFTPLUS | QD_FWD_SAVE_FOR_BWD))) return QD_ERR_INVALID_ARG;
    ScanArgs a{};
    a.s = *shape;
    a.save = (flags & QD_FWD_SAVE_FOR_BWD) != 0;
    a.softplus = (flags & QD_SOFTPLUS) != 0;
    const size_t need = qdelta_scan_workspace_bytes(shape, a.save ? 1 : 0);
    if (need && (!workspace || workspace_bytes < need)) return QD_ERR_WORKSPACE;
    a.u = u; a.dt = dt; a.A = A; a.Bm = Bm; a.Cm = Cm; a.D = D; a.z = z; a.dt_bias = dt_bias; a.h0 = h0; a.y = y; a.hT = hT;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    return timed(ST_SCAN, a.stream, [&] { return scan_fwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_scan_bwd(const qd_scan_shape* shape, const void* u, const void* dt, const float* A, const void* Bm, const void* Cm,
                    const float* D, const void* z, const float* dt_bias, const float* h0, const void* dy, const float* dhT, void* du,
                    void* ddt, float* dA, void* dBm, void* dCm, float* dD, void* dz, float* ddt_bias, float* dh0, void* workspace,
                    size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_scan(shape);
    if (rc != QD_OK) return rc;
    if (!u || !dt || !A || !Bm || !Cm || !dy || !du || !ddt || !dA || !dBm || !dCm) return QD_ERR_INVALID_ARG;
    if ((D && !dD) || (z && !dz) || (dt_bias && !ddt_bias) || (dh0 && dh0 == dhT)) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {u, dt, A, Bm, Cm, D, z, dt_bias, h0, dy, dhT, du, ddt, dA, dBm, dCm, dD, dz, ddt_bias, dh0, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)(QD_SOFTPLUS | QD_BWD_REUSE_FWD))) return QD_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < scan_bwd_workspace(*shape)) return QD_ERR_WORKSPACE;
    ScanArgs a{};
    a.s = *shape;
    a.softplus = (flags & QD_SOFTPLUS) != 0;
    a.u = u; a.dt = dt; a.A = A; a.Bm = Bm; a.Cm = Cm; a.D = D; a.z = z; a.dt_bias = dt_bias; a.h0 = h0;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    if (!(flags & QD_BWD_REUSE_FWD)) {                     // the states that a saving forward leaves, without its outputs
        a.save = true;
        if (timed(ST_SCAN, a.stream, [&] { return scan_fwd(a); }) != cudaSuccess) return QD_ERR_CUDA;
    }
    a.dy = dy; a.dhT = dhT; a.du = du; a.ddt = ddt; a.dA = dA; a.dBm = dBm; a.dCm = dCm;
    a.dD = D ? dD : nullptr; a.dz = dz; a.ddt_bias = dt_bias ? ddt_bias : nullptr; a.dh0 = dh0;
    return timed(ST_SCAN, a.stream, [&] { return scan_bwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_scan_steps(const qd_scan_shape* shape, const void* u, const void* dt, const float* A, const void* Bm, const void* Cm,
                      const float* D, const void* z, const float* dt_bias, float* state, void* y, unsigned flags, qd_stream stream) {
    const int rc = check_scan(shape);
    if (rc != QD_OK) return rc;
    if (!u || !dt || !A || !Bm || !Cm || !state || !y) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {u, dt, A, Bm, Cm, D, z, dt_bias, state, y};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_SOFTPLUS)) return QD_ERR_INVALID_ARG;
    ScanArgs a{};
    a.s = *shape;
    a.softplus = (flags & QD_SOFTPLUS) != 0;
    a.u = u; a.dt = dt; a.A = A; a.Bm = Bm; a.Cm = Cm; a.D = D; a.z = z; a.dt_bias = dt_bias; a.hT = state; a.y = y;
    a.stream = (cudaStream_t)stream;
    return timed(ST_SCAN, a.stream, [&] { return scan_steps(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_norm_fwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* bias, void* y, float* stats,
                    float eps, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !y || !(eps >= 0.f) || eps > 3e38f) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, weight, bias, y, stats};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_RMS)) return QD_ERR_INVALID_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = timed(ST_NORM, s, [&] { return norm_fwd(rows, width, dtype, x, weight, bias, y, stats, eps, (flags & QD_RMS) != 0, s); });
    return e == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

size_t qdelta_norm_workspace_bytes(long long rows, int width, int dtype) {
    return check_norm(rows, width, dtype) == QD_OK ? norm_bwd_workspace(rows, width, dtype) : 0;
}

int qdelta_norm_bwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* dy, const float* stats, void* dx,
                    float* dweight, float* dbias, void* workspace, size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !dy || !stats || !dx) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, weight, dy, stats, dx, dweight, dbias, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_RMS)) return QD_ERR_INVALID_ARG;
    if ((dweight || dbias) && (!workspace || workspace_bytes < norm_bwd_workspace(rows, width, dtype))) return QD_ERR_WORKSPACE;
    const cudaStream_t s = (cudaStream_t)stream;
    const cudaError_t e = timed(ST_NORM, s, [&] {
        return norm_bwd(rows, width, dtype, x, weight, dy, stats, dx, dweight, dbias, (float*)workspace, (flags & QD_RMS) != 0, s);
    });
    return e == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

size_t qdelta_linear_workspace_bytes(const qd_linear_shape* shape, int for_backward) {
    return check_linear(shape) == QD_OK ? linear_workspace(*shape, for_backward != 0) : 0;
}

int qdelta_linear_fwd(const qd_linear_shape* shape, const void* q, const void* k, const void* v, const float* log_decay, const float* h0,
                      void* o, float* hT, float scale, void* workspace, size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_linear(shape);
    if (rc != QD_OK) return rc;
    if (!q || !k || !v || !log_decay || !o || o == q || o == k || o == v || (hT && hT == h0) || !finite(scale) || flags) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {q, k, v, h0, o, hT, workspace};
    if (any_misaligned(ptrs) || ((uintptr_t)log_decay & 3)) return QD_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < linear_workspace(*shape, false)) return QD_ERR_WORKSPACE;
    LinearArgs a{};
    a.s = *shape;
    a.q = q; a.k = k; a.v = v; a.g = log_decay; a.h0 = h0; a.o = o; a.hT = hT; a.scale = scale;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    return timed(ST_LINEAR, a.stream, [&] { return linear_fwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_linear_bwd(const qd_linear_shape* shape, const void* q, const void* k, const void* v, const float* log_decay, const float* h0,
                      const void* dO, const float* dhT, void* dq, void* dk, void* dv, float* dh0, float scale, void* workspace,
                      size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_linear(shape);
    if (rc != QD_OK) return rc;
    // the walk that writes dh0 runs beside those that read h0
    if (!q || !k || !v || !log_decay || !dO || !dq || !dk || !dv || (dh0 && (dh0 == dhT || dh0 == h0)) || !finite(scale) || flags) return QD_ERR_INVALID_ARG;
    const void* const outs[] = {dq, dk, dv};
    const void* const ins[] = {q, k, v, dO};
    for (const void* x : outs)
        for (const void* y : ins)
            if (x == y) return QD_ERR_INVALID_ARG;          // other walks still read it
    if (dq == dk || dq == dv || dk == dv) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {q, k, v, h0, dO, dhT, dq, dk, dv, dh0, workspace};
    if (any_misaligned(ptrs) || ((uintptr_t)log_decay & 3)) return QD_ERR_INVALID_ARG;
    if (!workspace || workspace_bytes < linear_workspace(*shape, true)) return QD_ERR_WORKSPACE;
    LinearArgs a{};
    a.s = *shape;
    a.q = q; a.k = k; a.v = v; a.g = log_decay; a.h0 = h0; a.dO = dO; a.dhT = dhT; a.dq = dq; a.dk = dk; a.dv = dv; a.dh0 = dh0; a.scale = scale;
    a.ws = (char*)workspace;
    a.stream = (cudaStream_t)stream;
    return timed(ST_LINEAR, a.stream, [&] { return linear_bwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_linear_steps(const qd_linear_shape* shape, const void* q, const void* k, const void* v, const float* log_decay, float* state,
                        void* o, float scale, unsigned flags, qd_stream stream) {
    const int rc = check_linear(shape);
    if (rc != QD_OK) return rc;
    // o would be written before other CTAs have read these
    if (!q || !k || !v || !log_decay || !state || !o || o == q || o == k || o == v || !finite(scale) || flags) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {q, k, v, state, o};
    if (any_misaligned(ptrs) || ((uintptr_t)log_decay & 3)) return QD_ERR_INVALID_ARG;
    LinearArgs a{};
    a.s = *shape;
    a.q = q; a.k = k; a.v = v; a.g = log_decay; a.hT = state; a.o = o; a.scale = scale;
    a.stream = (cudaStream_t)stream;
    return timed(ST_LINEAR, a.stream, [&] { return linear_steps(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

size_t qdelta_fused_norm_workspace_bytes(long long rows, int width, int dtype) {
    return check_norm(rows, width, dtype) == QD_OK ? fused_norm_workspace(rows, width, dtype) : 0;
}

int qdelta_gated_norm_fwd(long long rows, int width, int dtype, const void* x, const void* gate, const void* weight, const void* bias, void* y,
                          float* stats, float eps, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !gate || !y || !(eps >= 0.f) || eps > 3e38f) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, gate, weight, bias, y, stats};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)(QD_RMS | QD_SILU))) return QD_ERR_INVALID_ARG;
    FusedNormArgs a{};
    a.rows = rows; a.width = width; a.dtype = dtype; a.rms = (flags & QD_RMS) != 0; a.silu = (flags & QD_SILU) != 0;
    a.x = x; a.gate = gate; a.weight = weight; a.bias = bias; a.y = y; a.stats = stats; a.eps = eps;
    a.stream = (cudaStream_t)stream;
    return timed(ST_NORM, a.stream, [&] { return fused_norm_fwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_gated_norm_bwd(long long rows, int width, int dtype, const void* x, const void* gate, const void* weight, const void* bias,
                          const void* dy, const float* stats, void* dx, void* dgate, float* dweight, float* dbias, void* workspace,
                          size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !gate || !dy || !stats || !dx || !dgate || dx == dgate) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, gate, weight, bias, dy, stats, dx, dgate, dweight, dbias, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)(QD_RMS | QD_SILU))) return QD_ERR_INVALID_ARG;
    if ((dweight || dbias || fused_norm_needs_workspace(rows, width, dtype)) &&
        (!workspace || workspace_bytes < fused_norm_workspace(rows, width, dtype)))
        return QD_ERR_WORKSPACE;
    FusedNormArgs a{};
    a.rows = rows; a.width = width; a.dtype = dtype; a.rms = (flags & QD_RMS) != 0; a.silu = (flags & QD_SILU) != 0;
    a.x = x; a.gate = gate; a.weight = weight; a.bias = bias; a.dy = dy; a.stats = const_cast<float*>(stats);
    a.dx = dx; a.dgate = dgate; a.dweight = dweight; a.dbias = dbias; a.part = (float*)workspace;
    a.stream = (cudaStream_t)stream;
    return timed(ST_NORM, a.stream, [&] { return fused_norm_bwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_add_norm_fwd(long long rows, int width, int dtype, const void* x, const void* residual, const void* scale, const void* weight,
                        const void* bias, void* total, void* y, float* stats, float eps, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !residual || !total || !y || total == y || !(eps >= 0.f) || eps > 3e38f) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, residual, scale, weight, bias, total, y, stats};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_RMS)) return QD_ERR_INVALID_ARG;
    FusedNormArgs a{};
    a.rows = rows; a.width = width; a.dtype = dtype; a.added = true; a.rms = (flags & QD_RMS) != 0;
    a.x = x; a.residual = residual; a.scale = scale; a.weight = weight; a.bias = bias; a.total = total; a.y = y; a.stats = stats; a.eps = eps;
    a.stream = (cudaStream_t)stream;
    return timed(ST_NORM, a.stream, [&] { return fused_norm_fwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_add_norm_bwd(long long rows, int width, int dtype, const void* x, const void* residual, const void* scale, const void* weight,
                        const void* dy, const void* dtotal, const float* stats, void* dx, void* dresidual, float* dscale, float* dweight,
                        float* dbias, void* workspace, size_t workspace_bytes, unsigned flags, qd_stream stream) {
    const int rc = check_norm(rows, width, dtype);
    if (rc != QD_OK) return rc;
    if (!x || !residual || !dy || !stats || !dresidual || (scale && !dx) || dx == dresidual) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {x, residual, scale, weight, dy, dtotal, stats, dx, dresidual, dscale, dweight, dbias, workspace};
    if (any_misaligned(ptrs) || (flags & ~(unsigned)QD_RMS)) return QD_ERR_INVALID_ARG;
    if ((dscale || dweight || dbias || fused_norm_needs_workspace(rows, width, dtype)) &&
        (!workspace || workspace_bytes < fused_norm_workspace(rows, width, dtype)))
        return QD_ERR_WORKSPACE;
    FusedNormArgs a{};
    a.rows = rows; a.width = width; a.dtype = dtype; a.added = true; a.rms = (flags & QD_RMS) != 0;
    a.x = x; a.residual = residual; a.scale = scale; a.weight = weight; a.dy = dy; a.dtotal = dtotal; a.stats = const_cast<float*>(stats);
    a.dx = dx; a.dresidual = dresidual; a.dscale = dscale; a.dweight = dweight; a.dbias = dbias; a.part = (float*)workspace;
    a.stream = (cudaStream_t)stream;
    return timed(ST_NORM, a.stream, [&] { return fused_norm_bwd(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_rotary(int B, int T, int Hq, int Hk, int d, int pairs, int dtype, const void* q, const void* k, const long long* turns,
                  const long long* positions, long long start, void* q_out, void* k_out, float scale, unsigned flags, qd_stream stream) {
    const int rc = check_rotary(B, T, Hq, Hk, d, pairs, dtype);
    if (rc != QD_OK) return rc;
    if (!q || !q_out || !turns || (Hk && (!k || !k_out)) || !finite(scale)) return QD_ERR_INVALID_ARG;
    if (Hk && (q_out == k || k_out == q || q_out == k_out)) return QD_ERR_INVALID_ARG;
    const void* const ptrs[] = {q, k, q_out, k_out};
    if (any_misaligned(ptrs) || ((uintptr_t)turns & 7) || ((uintptr_t)positions & 7)) return QD_ERR_INVALID_ARG;
    if (flags & ~(unsigned)(QD_INTERLEAVED | QD_INVERSE)) return QD_ERR_INVALID_ARG;
    RotaryArgs a{};
    a.B = B; a.T = T; a.Hq = Hq; a.Hk = Hk; a.d = d; a.pairs = pairs; a.dtype = dtype;
    a.q = q; a.k = k; a.turns = turns; a.positions = positions; a.start = start; a.q_out = q_out; a.k_out = k_out; a.scale = scale;
    a.interleaved = (flags & QD_INTERLEAVED) != 0; a.inverse = (flags & QD_INVERSE) != 0;
    a.stream = (cudaStream_t)stream;
    return timed(ST_ROTARY, a.stream, [&] { return rotary(a); }) == cudaSuccess ? QD_OK : QD_ERR_CUDA;
}

int qdelta_workspace_status(const void* workspace, int* status_out, qd_stream stream) {
    if (!workspace || !status_out) return QD_ERR_INVALID_ARG;
    unsigned w = 0;
    if (cudaMemcpyAsync(&w, workspace, 4, cudaMemcpyDeviceToHost, (cudaStream_t)stream) != cudaSuccess) return QD_ERR_CUDA;
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return QD_ERR_CUDA;
    *status_out = (int)w;
    return QD_OK;
}

int qdelta_profile_enable(int on) {
    g_profile = on != 0;
    return QD_OK;
}

int qdelta_profile_stage_count(void) { return ST_COUNT; }

const char* qdelta_profile_stage_name(int stage) {
    return (stage >= 0 && stage < ST_COUNT) ? kStageNames[stage] : "";
}

int qdelta_profile_read(int stage, double* total_ms, long long* launches, int reset) {
    if (stage < 0 || stage >= ST_COUNT || !total_ms || !launches) return QD_ERR_INVALID_ARG;
    for (const Pending& p : g_pending) {
        float ms = 0.f;
        if (cudaEventSynchronize(p.b) != cudaSuccess || cudaEventElapsedTime(&ms, p.a, p.b) != cudaSuccess)
            return QD_ERR_CUDA;
        g_ms[p.stage] += ms;
        g_launches[p.stage] += 1;
        g_pool.push_back(p.a);
        g_pool.push_back(p.b);
    }
    g_pending.clear();
    *total_ms = g_ms[stage];
    *launches = g_launches[stage];
    if (reset) { g_ms[stage] = 0.0; g_launches[stage] = 0; }
    return QD_OK;
}

const char* qdelta_status_string(int status) {
    switch (status) {
        case QD_OK: return "QD_OK";
        case QD_ERR_INVALID_ARG: return "QD_ERR_INVALID_ARG";
        case QD_ERR_UNSUPPORTED: return "QD_ERR_UNSUPPORTED";
        case QD_ERR_WORKSPACE: return "QD_ERR_WORKSPACE";
        case QD_ERR_CUDA: return "QD_ERR_CUDA";
        case QD_ERR_TIMEOUT: return "QD_ERR_TIMEOUT";
        case QD_ERR_STATIC_SCRATCH: return "QD_ERR_STATIC_SCRATCH (shape needs more than the built-in scratch array)";
        default: return "QD_ERR_UNKNOWN";
    }
}

}  // extern "C"

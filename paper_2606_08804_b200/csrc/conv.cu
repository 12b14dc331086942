// Short causal depthwise convolution: per sequence and channel, with W = 2, 3 or 4 taps,
//   pre_t = b + sum_j w_j x_{t-W+1+j} ,   y_t = SiLU(pre_t) or pre_t ;
// the W - 1 tokens before the first are the state (zeros if absent), the last W - 1 of state and tokens are the state afterwards.
// Backward, with dpre = dy f'(pre) (f' from pre, which is computed anew: W products instead of a saved tensor):
//   dx_s = sum_j w_j dpre_{s+W-1-j} (tokens and state rows alike, plus the gradient of the state afterwards),
//   dw_j = sum_t dpre_t x_{t-W+1+j},   db = sum_t dpre_t.
//
// Bound by HBM: 4 + 2 W operations and one exponential per element read and written.  A thread owns a group of neighbouring channels
// (16 bytes) and walks a run of tokens with the last W - 1 inputs (and, backward, the last W dpre) in registers, so an input is
// read once but for the W - 1 tokens in front of a run (W - 1 on either side backward).  A warp reads 32 neighbouring groups of a token.
#include "rows.cuh"

namespace qd {
namespace {

struct ConvP {
    int B, T, D, groups, cx, gx, run, runs;  // groups of channels; neighbouring groups per CTA, CTAs to cover them; tokens per run, runs per sequence
    const void *x, *w, *bias, *state, *dy, *dlast;
    void *y, *last, *dx, *dstate;
    float* part;                             // backward: [gy][W + 1][D]
    bool silu, vec;
};

template <typename IO, int V, int W>
__device__ __forceinline__ void load_taps(const ConvP& p, int c0, int left, float (&w)[W][V], float (&b)[V]) {
    const IO* wp = static_cast<const IO*>(p.w) + (size_t)c0 * W;
    const Pack<IO, V * W> t = load_pack<IO, V * W>(wp, left * W, p.vec);
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][i] = pick(t, i * W + j);
    if (p.bias) widen(load_pack<IO, V>(static_cast<const IO*>(p.bias) + c0, left, p.vec), b);
    else
#pragma unroll
        for (float& f : b) f = 0.f;
}

// Row of token t of sequence b, or of the state for t < 0; zeros where there is none.
template <typename IO, int V, int W>
__device__ __forceinline__ Pack<IO, V> load_row(const ConvP& p, const IO* x, const IO* state, int t, int left) {
    if (t >= 0) return load_pack<IO, V>(x + (size_t)t * p.D, left, p.vec);
    if (state) return load_pack<IO, V>(state + (size_t)(t + W - 1) * p.D, left, p.vec);
    return zero_pack<IO, V>();
}

// Forward and decode steps (one run for each sequence: the state may then be the one that is written).
template <typename IO, int V, int W>
__global__ void __launch_bounds__(256) k_conv_fwd(const ConvP p) {
    constexpr int U = 4;                                   // tokens on their way at a time
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int bx = blockIdx.x % p.gx, by = blockIdx.x / p.gx;
    const int g = bx * p.cx + threadIdx.x % p.cx;
    const long long item = (long long)by * (256 / p.cx) + threadIdx.x / p.cx;
    if (g >= p.groups || item >= (long long)p.B * p.runs) return;
    const int b = (int)(item / p.runs), t0 = (int)(item % p.runs) * p.run, t1 = min(p.T, t0 + p.run);
    const int c0 = g * V, left = p.D - c0;
    const IO* x = static_cast<const IO*>(p.x) + (size_t)b * p.T * p.D + c0;
    const IO* state = p.state ? static_cast<const IO*>(p.state) + (size_t)b * (W - 1) * p.D + c0 : nullptr;
    IO* y = static_cast<IO*>(p.y) + (size_t)b * p.T * p.D + c0;
    float w[W][V], bias[V];
    Pack<IO, V> win[W];                                    // the last W - 1 rows and the present one
#pragma unroll
    for (int j = 0; j < W - 1; ++j) win[j] = load_row<IO, V, W>(p, x, state, t0 - (W - 1) + j, left);
    Pack<IO, V> next[U];
#pragma unroll
    for (int i = 0; i < U; ++i) next[i] = t0 + i < t1 ? load_pack<IO, V>(x + (size_t)(t0 + i) * p.D, left, p.vec) : zero_pack<IO, V>();
    load_taps<IO, V, W>(p, c0, left, w, bias);
    for (int t = t0; t < t1; t += U) {
        Pack<IO, V> cur[U];
#pragma unroll
        for (int i = 0; i < U; ++i) cur[i] = next[i];
#pragma unroll
        for (int i = 0; i < U; ++i)
            if (t + U + i < t1) next[i] = load_pack<IO, V>(x + (size_t)(t + U + i) * p.D, left, p.vec);
#pragma unroll
        for (int i = 0; i < U; ++i) {
            if (t + i >= t1) break;
            win[W - 1] = cur[i];
            float o[V];
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float s = bias[c];
#pragma unroll
                for (int j = 0; j < W; ++j) s = fmaf(w[j][c], pick(win[j], c), s);
                o[c] = p.silu ? s * sigmoid(s) : s;
            }
            store_pack(y + (size_t)(t + i) * p.D, narrow<IO, V>(o), left, p.vec);
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        }
    }
    if (p.last && t1 == p.T) {                             // what this thread holds are the last W - 1 rows
        IO* last = static_cast<IO*>(p.last) + (size_t)b * (W - 1) * p.D + c0;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) store_pack(last + (size_t)j * p.D, win[j], left, p.vec);
    }
}

// Backward of a run [t0, t1): dpre of its tokens and of the W - 1 behind them.  Token s emits dx of token s - W + 1.
template <typename IO, int V, int W>
__global__ void __launch_bounds__(256) k_conv_bwd(const ConvP p) {
    __shared__ float red[256][V + 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int bx = blockIdx.x % p.gx, by = blockIdx.x / p.gx;
    const int g = bx * p.cx + threadIdx.x % p.cx;
    const long long item = (long long)by * (256 / p.cx) + threadIdx.x / p.cx;
    const bool live = g < p.groups && item < (long long)p.B * p.runs;
    const int c0 = g * V, left = p.D - c0;
    float dw[W][V], db[V];
#pragma unroll
    for (int c = 0; c < V; ++c) {
        db[c] = 0.f;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][c] = 0.f;
    }
    if (live) {
        const int b = (int)(item / p.runs), t0 = (int)(item % p.runs) * p.run, t1 = min(p.T, t0 + p.run);
        const size_t base = (size_t)b * p.T * p.D + c0, sbase = (size_t)b * (W - 1) * p.D + c0;
        const IO *x = static_cast<const IO*>(p.x) + base, *dy = static_cast<const IO*>(p.dy) + base;
        const IO* state = p.state ? static_cast<const IO*>(p.state) + sbase : nullptr;
        const IO* dlast = p.dlast ? static_cast<const IO*>(p.dlast) + sbase : nullptr;
        IO* dx = static_cast<IO*>(p.dx) + base;
        IO* dstate = p.dstate ? static_cast<IO*>(p.dstate) + sbase : nullptr;
        float w[W][V], bias[V], dp[W][V];
        Pack<IO, V> win[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) win[j] = load_row<IO, V, W>(p, x, state, t0 - (W - 1) + j, left);
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int c = 0; c < V; ++c) dp[j][c] = 0.f;
        load_taps<IO, V, W>(p, c0, left, w, bias);
        auto xrow = [&](int t) { return t < p.T ? load_pack<IO, V>(x + (size_t)t * p.D, left, p.vec) : zero_pack<IO, V>(); };
        auto yrow = [&](int t) { return t < p.T ? load_pack<IO, V>(dy + (size_t)t * p.D, left, p.vec) : zero_pack<IO, V>(); };
        const int end = t1 + W - 1;
        Pack<IO, V> nx = xrow(t0), ny = yrow(t0);
#pragma unroll 2
        for (int s = t0; s < end; ++s) {
            win[W - 1] = nx;
            float gy[V];
            widen(ny, gy);
            if (s + 1 < end) { nx = xrow(s + 1); ny = yrow(s + 1); }
            const bool own = s < t1;
#pragma unroll
            for (int c = 0; c < V; ++c) {
                float d = gy[c];
                if (p.silu) {
                    float a = bias[c];
#pragma unroll
                    for (int j = 0; j < W; ++j) a = fmaf(w[j][c], pick(win[j], c), a);
                    const float sg = sigmoid(a);
                    d *= sg * fmaf(a, 1.f - sg, 1.f);
                }
                if (s >= p.T) d = 0.f;                     // behind the last token: nothing, whatever the window holds
#pragma unroll
                for (int j = 0; j < W - 1; ++j) dp[j][c] = dp[j + 1][c];
                dp[W - 1][c] = d;
                if (own) {
                    db[c] += d;
#pragma unroll
                    for (int j = 0; j < W; ++j) dw[j][c] = fmaf(d, pick(win[j], c), dw[j][c]);
                }
            }
            const int t = s - (W - 1);                     // its gradient is complete
            if (t >= t0 || (t < 0 && dstate)) {            // t < 0 in a sequence's first run only
                float o[V];
#pragma unroll
                for (int c = 0; c < V; ++c) {
                    o[c] = 0.f;
#pragma unroll
                    for (int j = 0; j < W; ++j) o[c] = fmaf(w[W - 1 - j][c], dp[j][c], o[c]);
                }
                if (dlast && t >= p.T - (W - 1)) {
                    float e[V];
                    widen(load_pack<IO, V>(dlast + (size_t)(t - (p.T - (W - 1))) * p.D, left, p.vec), e);
#pragma unroll
                    for (int c = 0; c < V; ++c) o[c] += e[c];
                }
                IO* to = t >= 0 ? dx + (size_t)t * p.D : dstate + (size_t)(t + W - 1) * p.D;
                store_pack(to, narrow<IO, V>(o), left, p.vec);
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) win[j] = win[j + 1];
        }
    }
    // one partial of dw and db for the CTA: the threads of a group of channels in order
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        __syncthreads();
#pragma unroll
        for (int c = 0; c < V; ++c) red[threadIdx.x][c] = j < W ? dw[j < W ? j : 0][c] : db[c];
        __syncthreads();
        for (int i = threadIdx.x; i < p.cx * V; i += 256) {
            const int x = i / V, c = i % V, ch = (bx * p.cx + x) * V + c;
            if (ch >= p.D) continue;
            float t = 0.f;
            for (int r = x; r < 256; r += p.cx) t += red[r][c];
            p.part[((size_t)by * (W + 1) + j) * p.D + ch] = t;
        }
    }
}

struct ConvPlan { int V, groups, cx, run, runs, gx; long long gy; };
// Runs as long as leaves `threads` of them: a run reads W - 1 tokens again.  Neighbouring groups per CTA: a warp's worth, fewer where
// there are fewer channels.
ConvPlan conv_plan(int B, int T, int D, int V, long long threads, int shortest, bool whole) {
    ConvPlan q{};
    q.V = V;
    q.groups = (D + V - 1) / V;
    q.cx = 32;
    while (q.cx > 1 && q.cx / 2 >= q.groups) q.cx /= 2;
    const long long rows = (threads + q.groups - 1) / q.groups;             // runs wanted
    const long long per = (rows + B - 1) / B;
    long long run = whole ? T : ((long long)T + per - 1) / per;
    if (run < shortest) run = shortest;
    if (run > T) run = T;
    q.run = (int)run;
    q.runs = (int)(((long long)T + run - 1) / run);
    q.gx = (q.groups + q.cx - 1) / q.cx;
    const long long per_cta = 256 / q.cx;
    q.gy = ((long long)B * q.runs + per_cta - 1) / per_cta;
    return q;
}
int vector_of(int dtype) { return dtype == QD_BF16 ? 8 : 4; }               // 16 bytes
ConvPlan conv_fwd_plan(int B, int T, int D, int dtype, bool whole) {
    return conv_plan(B, T, D, vector_of(dtype), (long long)kSMs * 2048, 4, whole);
}
ConvPlan conv_bwd_plan(int B, int T, int D, int dtype) { return conv_plan(B, T, D, vector_of(dtype), (long long)kSMs * 1024, 16, false); }

template <typename IO, int V>
cudaError_t launch_fwd(int W, const ConvPlan& q, const ConvP& p, cudaStream_t stream) {
    const auto k = W == 2 ? k_conv_fwd<IO, V, 2> : W == 3 ? k_conv_fwd<IO, V, 3> : k_conv_fwd<IO, V, 4>;
    return launch_overlapped(k, dim3((unsigned)(q.gx * q.gy)), dim3(256), 0, stream, p);
}
template <typename IO, int V>
cudaError_t launch_bwd(int W, const ConvPlan& q, const ConvP& p, cudaStream_t stream) {
    const auto k = W == 2 ? k_conv_bwd<IO, V, 2> : W == 3 ? k_conv_bwd<IO, V, 3> : k_conv_bwd<IO, V, 4>;
    return launch_overlapped(k, dim3((unsigned)(q.gx * q.gy)), dim3(256), 0, stream, p);
}

}  // namespace

size_t conv_bwd_workspace(int B, int T, int D, int W, int dtype) {
    return (size_t)conv_bwd_plan(B, T, D, dtype).gy * (W + 1) * D * sizeof(float);
}

cudaError_t conv_fwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state, void* y,
                     void* last, bool silu, cudaStream_t stream) {
    const ConvPlan q = conv_fwd_plan(B, T, D, dtype, state && state == last);
    ConvP p{};
    p.B = B; p.T = T; p.D = D; p.groups = q.groups; p.cx = q.cx; p.gx = q.gx; p.run = q.run; p.runs = q.runs;
    p.x = x; p.w = w; p.bias = bias; p.state = state; p.y = y; p.last = last;
    p.silu = silu; p.vec = D % q.V == 0;
    return dtype == QD_BF16 ? launch_fwd<__nv_bfloat16, 8>(W, q, p, stream) : launch_fwd<float, 4>(W, q, p, stream);
}

cudaError_t conv_bwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state,
                     const void* dy, const void* dlast, void* dx, float* dw, float* dbias, void* dstate, float* part, bool silu,
                     cudaStream_t stream) {
    const ConvPlan q = conv_bwd_plan(B, T, D, dtype);
    ConvP p{};
    p.B = B; p.T = T; p.D = D; p.groups = q.groups; p.cx = q.cx; p.gx = q.gx; p.run = q.run; p.runs = q.runs;
    p.x = x; p.w = w; p.bias = bias; p.state = state; p.dy = dy; p.dlast = dlast; p.dx = dx; p.dstate = dstate;
    p.part = part; p.silu = silu; p.vec = D % q.V == 0;
    const cudaError_t e = dtype == QD_BF16 ? launch_bwd<__nv_bfloat16, 8>(W, q, p, stream) : launch_bwd<float, 4>(W, q, p, stream);
    if (e != cudaSuccess) return e;
    return sum_parts(part, (int)q.gy, (long long)(W + 1) * D, (long long)W * D, D, W, dw, dbias, stream);
}

}  // namespace qd

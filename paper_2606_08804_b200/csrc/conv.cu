// Short causal depthwise convolution: per sequence and channel, with W = 2, 3 or 4 taps,
//   pre_t = b + sum_j w_j x_{t-W+1+j} ,   y_t = SiLU(pre_t) or pre_t ;
// the W - 1 tokens before the first are the state (zeros if absent), the last W - 1 of state and tokens are the state afterwards.
// Backward, with dpre = dy f'(pre) (f' from pre, which is computed anew: W products instead of a saved tensor):
//   dx_s = sum_j w_j dpre_{s+W-1-j} (tokens and state rows alike, plus the gradient of the state afterwards),
//   dw_j = sum_t dpre_t x_{t-W+1+j},   db = sum_t dpre_t.
//
// Bound by HBM: 16384 tokens of 6144 bf16 channels take 74 us forward (5.4 TB/s) and 128 backward (4.7 TB/s, where the registers of the
// gradients leave 16 warps to an SM), 256 decode steps 5.8 us (4.3 TB/s).  A thread owns a group of neighbouring channels and walks a run
// of tokens with the last W - 1 inputs (and, backward, the last W - 1 dpre) in registers, so an input is read once but for the W - 1 tokens
// in front of a run (W - 1 on either side backward); a warp reads 32 neighbouring groups of a token.  So that the arithmetic stays below
// HBM's time, channels are taken two at a time in the packed fp32 instructions of sm_100, an input is widened once, and bf16 gates use the
// special function unit directly.
// Where rows are not whole groups, the channels of a thread are `cx` apart instead, so that a warp's single loads are neighbours.
#include "rows.cuh"

namespace qd {
namespace {

constexpr int kConvThreads = 128;

struct ConvP {
    int B, T, D, cx, gx, run, runs;          // groups per row of a CTA's threads, CTAs across the channels; tokens per run, runs per sequence
    const void *x, *w, *bias, *state, *dy, *dlast;
    void *y, *last, *dx, *dstate;
    float* part;                             // backward: [gy][W + 1][D]
    bool silu, vec;
};

// The channels of a thread: c0, c0 + step, .. (V of them, those below D).  VEC: neighbours, all of them or none.
template <int V, bool VEC> struct Cols {
    int c0, step, left;
    __device__ __forceinline__ Cols(const ConvP& p, int bx, int x) {
        step = VEC ? 1 : p.cx;
        c0 = bx * p.cx * V + (VEC ? x * V : x);
        left = VEC ? (c0 < p.D ? V : 0) : (p.D - c0 + step - 1) / step;
    }
};
template <typename IO, int V, bool VEC>
__device__ __forceinline__ Pack<IO, V> load_cols(const IO* p, const Cols<V, VEC>& c) {
    if constexpr (VEC) {
        return load_pack<IO, V>(p, V, true);
    } else {
        Pack<IO, V> r = zero_pack<IO, V>();
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < c.left) {
                if constexpr (sizeof(IO) == 4) r.w[i] = __float_as_uint(p[(size_t)i * c.step]);
                else r.w[i >> 1] |= (uint32_t)reinterpret_cast<const unsigned short*>(p)[(size_t)i * c.step] << (i & 1) * 16;
            }
        return r;
    }
}
template <typename IO, int V, bool VEC>
__device__ __forceinline__ void store_cols(IO* p, const Pack<IO, V>& r, const Cols<V, VEC>& c) {
    if constexpr (VEC) {
        store_pack(p, r, V, true);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i < c.left) {
                if constexpr (sizeof(IO) == 4) p[(size_t)i * c.step] = __uint_as_float(r.w[i]);
                else reinterpret_cast<unsigned short*>(p)[(size_t)i * c.step] = (unsigned short)(i & 1 ? r.w[i >> 1] >> 16 : r.w[i >> 1]);
            }
    }
}
template <typename IO, int V>
__device__ __forceinline__ void widen2(const Pack<IO, V>& r, f2 (&f)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) f[i] = pack2(pick(r, 2 * i), pick(r, 2 * i + 1));
}
template <typename IO, int V>
__device__ __forceinline__ Pack<IO, V> narrow2(const f2 (&f)[V / 2]) {
    float o[V];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        const float2 t = unpack2(f[i]);
        o[2 * i] = t.x;
        o[2 * i + 1] = t.y;
    }
    return narrow<IO, V>(o);
}

template <typename IO, int V, int W, bool VEC>
__device__ __forceinline__ void load_taps(const ConvP& p, const Cols<V, VEC>& c, f2 (&w)[W][V / 2], f2 (&b)[V / 2]) {
    const IO* wp = static_cast<const IO*>(p.w) + (size_t)c.c0 * W;
    float f[V][W];
    if constexpr (VEC) {
        const Pack<IO, V * W> t = load_pack<IO, V * W>(wp, V * W, true);
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) f[i][j] = pick(t, i * W + j);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i)
#pragma unroll
            for (int j = 0; j < W; ++j) f[i][j] = i < c.left ? ld(wp, (size_t)i * c.step * W + j) : 0.f;
    }
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        b[i] = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) w[j][i] = pack2(f[2 * i][j], f[2 * i + 1][j]);
    }
    if (p.bias) widen2(load_cols(static_cast<const IO*>(p.bias) + c.c0, c), b);
}

// sigmoid of two numbers.  bf16 results are rounded to 2^-9, so that e^-x may have a relative error of 2^-24 |x|.
template <typename IO>
__device__ __forceinline__ f2 sigmoid2(f2 v) {
    if constexpr (sizeof(IO) == 2) {
        const float2 t = unpack2(add2(exp2_pair(mul2(v, both(-kLog2e))), both(1.f)));
        return pack2(reciprocal(t.x), reciprocal(t.y));
    } else {
        const float2 t = unpack2(v);
        return pack2(sigmoid(t.x), sigmoid(t.y));
    }
}
// The last rows in a ring of four: a token's row goes where its number mod 4 says, which unrolled by four is a register, and nothing moves.
constexpr int kRing = 4;
template <int V, int W>
__device__ __forceinline__ void convolve(const f2 (&w)[W][V / 2], const f2 (&b)[V / 2], const f2 (&win)[kRing][V / 2], int u, f2 (&pre)[V / 2]) {
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        f2 s = b[i];
#pragma unroll
        for (int j = 0; j < W; ++j) s = fma2(w[j][i], win[(u + kRing - (W - 1) + j) % kRing][i], s);
        pre[i] = s;
    }
}
template <typename IO, int V, bool SILU>
__device__ __forceinline__ Pack<IO, V> finish(const f2 (&pre)[V / 2]) {
    f2 o[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) o[i] = SILU ? mul2(pre[i], sigmoid2<IO>(pre[i])) : pre[i];
    return narrow2<IO, V>(o);
}
// The W - 1 rows before token t0 of a sequence, from its tokens or its state; t0 is number 0 of the ring.
template <typename IO, int V, int W, bool VEC>
__device__ __forceinline__ void load_window(const ConvP& p, const Cols<V, VEC>& c, const IO* x, const IO* state, int t0, f2 (&win)[kRing][V / 2]) {
#pragma unroll
    for (int j = 1; j < W; ++j) {
        const int t = t0 - j;
        widen2(t >= 0 ? load_cols(x + (size_t)t * p.D, c) : state ? load_cols(state + (size_t)(t + W - 1) * p.D, c) : zero_pack<IO, V>(), win[kRing - j]);
    }
}
// The W - 1 rows up to the one whose number is u.
template <typename IO, int V, int W, bool VEC>
__device__ __forceinline__ void store_window(const ConvP& p, const Cols<V, VEC>& c, int b, const f2 (&win)[kRing][V / 2], int u) {
    IO* last = static_cast<IO*>(p.last) + (size_t)b * (W - 1) * p.D + c.c0;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) store_cols(last + (size_t)j * p.D, narrow2<IO, V>(win[(u + kRing - (W - 2) + j) % kRing]), c);
}
struct Inside { static constexpr bool value = true; };     // a group of four tokens none of which is at an edge
struct Edge { static constexpr bool value = false; };

template <typename IO, int V, int W, bool VEC, bool SILU>
__global__ void __launch_bounds__(kConvThreads, sizeof(IO) == 2 ? 8 : 4) k_conv_fwd(const ConvP p) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int bx = blockIdx.x % p.gx;
    const long long item = (long long)(blockIdx.x / p.gx) * (kConvThreads / p.cx) + threadIdx.x / p.cx;
    const Cols<V, VEC> c(p, bx, threadIdx.x % p.cx);
    if (c.left <= 0 || item >= (long long)p.B * p.runs) return;
    const int b = (int)(item / p.runs), t0 = (int)(item % p.runs) * p.run, t1 = min(p.T, t0 + p.run);
    const IO* x = static_cast<const IO*>(p.x) + (size_t)b * p.T * p.D + c.c0;
    const IO* state = p.state ? static_cast<const IO*>(p.state) + (size_t)b * (W - 1) * p.D + c.c0 : nullptr;
    const size_t D = p.D;
    const IO* at = x + (size_t)t0 * D;                     // of the group's first token
    IO* y = static_cast<IO*>(p.y) + (size_t)b * p.T * D + c.c0 + (size_t)t0 * D;
    Pack<IO, V> next[kRing];                               // tokens on their way
#pragma unroll
    for (int u = 0; u < kRing; ++u) next[u] = t0 + u < t1 ? load_cols(at + u * D, c) : zero_pack<IO, V>();
    f2 w[W][V / 2], bias[V / 2], win[kRing][V / 2];
    load_window<IO, V, W, VEC>(p, c, x, state, t0, win);
    load_taps<IO, V, W, VEC>(p, c, w, bias);
    auto group = [&](auto where, int t) {
        constexpr bool INSIDE = decltype(where)::value;    // and so is the group after it
        const IO* ahead = at + kRing * D;
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            if (!INSIDE && t + u >= t1) break;
            f2 pre[V / 2];
            widen2(next[u], win[u]);
            if (INSIDE || t + u + kRing < t1) next[u] = load_cols(ahead + u * D, c);
            convolve<V, W>(w, bias, win, u, pre);
            store_cols(y + u * D, finish<IO, V, SILU>(pre), c);
            // what this thread holds at the end are the last W - 1 rows
            if (!INSIDE && t + u + 1 == p.T && p.last) store_window<IO, V, W, VEC>(p, c, b, win, u);
        }
        at = ahead;
        y += kRing * D;
    };
    int t = t0;
    for (; t + 2 * kRing <= t1; t += kRing) group(Inside{}, t);
    for (; t < t1; t += kRing) group(Edge{}, t);
}

// Decode steps: every sequence in one run, the state written where it was read.
template <typename IO, int V, int W, bool VEC, bool SILU>
__global__ void __launch_bounds__(kConvThreads) k_conv_steps(const ConvP p) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int bx = blockIdx.x % p.gx;
    const long long b = (long long)(blockIdx.x / p.gx) * (kConvThreads / p.cx) + threadIdx.x / p.cx;
    const Cols<V, VEC> c(p, bx, threadIdx.x % p.cx);
    if (c.left <= 0 || b >= p.B) return;
    const IO* x = static_cast<const IO*>(p.x) + (size_t)b * p.T * p.D + c.c0;
    const IO* state = static_cast<const IO*>(p.state) + (size_t)b * (W - 1) * p.D + c.c0;
    IO* y = static_cast<IO*>(p.y) + (size_t)b * p.T * p.D + c.c0;
    Pack<IO, V> next = load_cols(x, c);
    f2 w[W][V / 2], bias[V / 2], win[kRing][V / 2];
    load_window<IO, V, W, VEC>(p, c, x, state, 0, win);
    load_taps<IO, V, W, VEC>(p, c, w, bias);
    for (int t = 0; t < p.T; t += kRing) {
#pragma unroll
        for (int u = 0; u < kRing; ++u) {
            if (t + u >= p.T) break;
            f2 pre[V / 2];
            widen2(next, win[u]);
            if (t + u + 1 < p.T) next = load_cols(x + (size_t)(t + u + 1) * p.D, c);
            convolve<V, W>(w, bias, win, u, pre);
            store_cols(y + (size_t)(t + u) * p.D, finish<IO, V, SILU>(pre), c);
            if (t + u + 1 == p.T) store_window<IO, V, W, VEC>(p, c, (int)b, win, u);
        }
    }
}

// Backward of a run [t0, t1): dpre of its tokens and of the W - 1 behind them.  Token s emits dx of token s - W + 1.
// What is read is copied to shared memory three groups of four tokens ahead, each thread its own: in registers it would be one (171 us instead
// of 128 for 16384 tokens of 6144 channels).
template <typename IO, int V, int W, bool VEC, bool SILU>
__global__ void __launch_bounds__(kConvThreads, 4) k_conv_bwd(const ConvP p) {
    constexpr int AHEAD = 3;
    __shared__ float red[kConvThreads][V + 1];
    extern __shared__ __align__(16) unsigned char ahead_smem[];            // [AHEAD][kRing][x, dy][threads] groups of channels
    Pack<IO, V>* ahead = reinterpret_cast<Pack<IO, V>*>(ahead_smem) + threadIdx.x;
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int bx = blockIdx.x % p.gx;
    const long long by = blockIdx.x / p.gx, item = by * (kConvThreads / p.cx) + threadIdx.x / p.cx;
    const Cols<V, VEC> c(p, bx, threadIdx.x % p.cx);
    f2 dw[W][V / 2], db[V / 2];
#pragma unroll
    for (int i = 0; i < V / 2; ++i) {
        db[i] = 0;
#pragma unroll
        for (int j = 0; j < W; ++j) dw[j][i] = 0;
    }
    if (c.left > 0 && item < (long long)p.B * p.runs) {
        const int b = (int)(item / p.runs), t0 = (int)(item % p.runs) * p.run, t1 = min(p.T, t0 + p.run), end = t1 + W - 1;
        const size_t D = p.D, base = (size_t)b * p.T * D + c.c0, sbase = (size_t)b * (W - 1) * D + c.c0;
        const IO* x = static_cast<const IO*>(p.x) + base;
        const IO* state = p.state ? static_cast<const IO*>(p.state) + sbase : nullptr;
        const IO* dlast = p.dlast ? static_cast<const IO*>(p.dlast) + sbase : nullptr;
        IO* dstate = p.dstate ? static_cast<IO*>(p.dstate) + sbase : nullptr;
        const IO *xp = x + (size_t)t0 * D, *yp = static_cast<const IO*>(p.dy) + base + (size_t)t0 * D;     // of the group's first token
        IO* dx = static_cast<IO*>(p.dx) + base;
        // group of four tokens from s, which are `rows` ahead of xp, yp
        auto fetch = [&](auto where, int slot, int s, int rows) {
            constexpr bool INSIDE = decltype(where)::value;
#pragma unroll
            for (int u = 0; u < kRing; ++u) {
                const bool in = INSIDE || (s + u < end && s + u < p.T);
                Pack<IO, V>* to = ahead + (slot * kRing + u) * 2 * kConvThreads;
                const size_t off = in ? (size_t)(rows + u) * D : 0;
                if constexpr (VEC) {
                    copy_bytes<V * sizeof(IO)>(to, xp + off, in ? V * sizeof(IO) : 0);
                    copy_bytes<V * sizeof(IO)>(to + kConvThreads, yp + off, in ? V * sizeof(IO) : 0);
                } else if constexpr (sizeof(IO) == 4) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const bool has = in && i < c.left;
                        copy_bytes<4>(&to[0].w[i], xp + (has ? off + i * c.step : 0), has ? 4 : 0);
                        copy_bytes<4>(&to[kConvThreads].w[i], yp + (has ? off + i * c.step : 0), has ? 4 : 0);
                    }
                } else {                                   // single bf16 are no size that can be copied so: waited for
                    to[0] = in ? load_cols(xp + off, c) : zero_pack<IO, V>();
                    to[kConvThreads] = in ? load_cols(yp + off, c) : zero_pack<IO, V>();
                }
            }
            copy_commit();
        };
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) fetch(Edge{}, g, t0 + g * kRing, g * kRing);
        f2 w[W][V / 2], bias[V / 2], win[kRing][V / 2], dp[kRing][V / 2];
        load_window<IO, V, W, VEC>(p, c, x, state, t0, win);
        load_taps<IO, V, W, VEC>(p, c, w, bias);
#pragma unroll
        for (int j = 0; j < kRing; ++j)
#pragma unroll
            for (int i = 0; i < V / 2; ++i) dp[j][i] = 0;
        int slot = 0;
        auto group = [&](auto where, int s0) {
            constexpr bool INSIDE = decltype(where)::value;                // tokens of the run whose W - 1 before them are too; the groups ahead exist
            copy_wait<AHEAD - 1>();
            Pack<IO, V>* have = ahead + slot * kRing * 2 * kConvThreads;
            IO* to = dx + (size_t)(INSIDE ? s0 - (W - 1) : 0) * D;
#pragma unroll
            for (int u = 0; u < kRing; ++u) {
                const int s = s0 + u;
                if (!INSIDE && s >= end) break;
                f2(&d)[V / 2] = dp[u];
                widen2(have[u * 2 * kConvThreads], win[u]);
                widen2(have[(u * 2 + 1) * kConvThreads], d);
                if (!INSIDE && s >= p.T) {                 // behind the last token: nothing, whatever the window holds
#pragma unroll
                    for (f2& v : d) v = 0;
                } else if (SILU) {
                    f2 pre[V / 2];
                    convolve<V, W>(w, bias, win, u, pre);
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        const f2 sg = sigmoid2<IO>(pre[i]), rest = fma2(sg, both(-1.f), both(1.f));
                        d[i] = mul2(d[i], mul2(sg, fma2(pre[i], rest, both(1.f))));
                    }
                }
                if (INSIDE || s < t1) {
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        db[i] = add2(db[i], d[i]);
#pragma unroll
                        for (int j = 0; j < W; ++j) dw[j][i] = fma2(d[i], win[(u + kRing - (W - 1) + j) % kRing][i], dw[j][i]);
                    }
                }
                const int t = s - (W - 1);                 // its gradient is complete
                if (INSIDE || t >= t0 || (t < 0 && dstate)) {              // t < 0 in a sequence's first run only
                    f2 o[V / 2];
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        f2 v = mul2(w[0][i], d[i]);
#pragma unroll
                        for (int j = 1; j < W; ++j) v = fma2(w[j][i], dp[(u + kRing - j) % kRing][i], v);
                        o[i] = v;
                    }
                    if (!INSIDE && dlast && t >= p.T - (W - 1)) {
                        f2 e[V / 2];
                        widen2(load_cols(dlast + (size_t)(t - (p.T - (W - 1))) * D, c), e);
#pragma unroll
                        for (int i = 0; i < V / 2; ++i) o[i] = add2(o[i], e[i]);
                    }
                    IO* out = INSIDE ? to + u * D : t >= 0 ? dx + (size_t)t * D : dstate + (size_t)(t + W - 1) * D;
                    store_cols(out, narrow2<IO, V>(o), c);
                }
            }
            fetch(where, slot, s0 + AHEAD * kRing, AHEAD * kRing);
            slot = slot == AHEAD - 1 ? 0 : slot + 1;
            xp += kRing * D;
            yp += kRing * D;
        };
        int s = t0;
        group(Edge{}, s);
        s += kRing;
        for (; s + (AHEAD + 1) * kRing <= t1; s += kRing) group(Inside{}, s);
        for (; s < end; s += kRing) group(Edge{}, s);
    }
    // one partial of dw and db for the CTA: the threads of a group of channels in order
#pragma unroll
    for (int j = 0; j <= W; ++j) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            const float2 t = unpack2(j < W ? dw[j < W ? j : 0][i] : db[i]);
            red[threadIdx.x][2 * i] = t.x;
            red[threadIdx.x][2 * i + 1] = t.y;
        }
        __syncthreads();
        for (int e = threadIdx.x; e < p.cx * V; e += kConvThreads) {
            const int gr = VEC ? e / V : e % p.cx, i = VEC ? e % V : e / p.cx, ch = bx * p.cx * V + e;      // channels in order
            if (ch >= p.D) continue;
            float t = 0.f;
            for (int r = gr; r < kConvThreads; r += p.cx) t += red[r][i];
            p.part[((size_t)by * (W + 1) + j) * p.D + ch] = t;
        }
    }
}

struct ConvPlan { int cx, gx, run, runs; long long gy; };
// Runs such that `threads` of them, which are resident at once, take all tokens, of `shortest` tokens at least: a run reads W - 1 tokens
// again.  Neighbouring groups in a row of threads: a warp's worth, fewer where there are fewer channels.
ConvPlan conv_plan(int B, int T, int D, int V, long long threads, int shortest) {
    ConvPlan q{};
    const int groups = (D + V - 1) / V;
    q.cx = 32;
    while (q.cx > 1 && q.cx / 2 >= groups) q.cx /= 2;
    q.gx = (groups + q.cx - 1) / q.cx;
    const long long per = threads / ((long long)q.gx * q.cx) / B;           // runs of a sequence
    long long run = per > 1 ? ((long long)T + per - 1) / per : T;
    if (run < shortest) run = shortest;
    if (run > T) run = T;
    q.run = (int)run;
    q.runs = (int)(((long long)T + run - 1) / run);
    const long long per_cta = kConvThreads / q.cx;
    q.gy = ((long long)B * q.runs + per_cta - 1) / per_cta;
    return q;
}
constexpr int kFwdGroup = 4;                               // of eight bf16 channels fewer threads have loads on their way (82 us for 75)
constexpr int kBwdGroup = 4;                               // half the registers of eight, so that more threads have loads on their way
ConvPlan conv_bwd_plan(int B, int T, int D) { return conv_plan(B, T, D, kBwdGroup, kSMs * 4LL * kConvThreads, 8); }

ConvP params(int B, int T, int D, const ConvPlan& q, bool silu, bool vec) {
    ConvP p{};
    p.B = B; p.T = T; p.D = D; p.cx = q.cx; p.gx = q.gx; p.run = q.run; p.runs = q.runs; p.silu = silu; p.vec = vec;
    return p;
}
enum Kind { FWD, STEPS, BWD };
template <Kind KIND, typename IO, int V, int W, bool VEC, bool SILU>
cudaError_t launch(const ConvPlan& q, const ConvP& p, cudaStream_t stream) {
    const dim3 grid((unsigned)(q.gx * q.gy));
    if constexpr (KIND == FWD) return launch_overlapped(k_conv_fwd<IO, V, W, VEC, SILU>, grid, dim3(kConvThreads), 0, stream, p);
    else if constexpr (KIND == STEPS) return launch_overlapped(k_conv_steps<IO, V, W, VEC, SILU>, grid, dim3(kConvThreads), 0, stream, p);
    else {
        constexpr size_t smem = 3 * kRing * 2 * kConvThreads * V * sizeof(IO);
        const cudaError_t e = set_max_smem_once((const void*)k_conv_bwd<IO, V, W, VEC, SILU>, smem);
        return e != cudaSuccess ? e : launch_overlapped(k_conv_bwd<IO, V, W, VEC, SILU>, grid, dim3(kConvThreads), smem, stream, p);
    }
}
template <Kind KIND, typename IO, int V, int W>
cudaError_t launch(const ConvPlan& q, const ConvP& p, cudaStream_t s) {
    if (p.vec) return p.silu ? launch<KIND, IO, V, W, true, true>(q, p, s) : launch<KIND, IO, V, W, true, false>(q, p, s);
    return p.silu ? launch<KIND, IO, V, W, false, true>(q, p, s) : launch<KIND, IO, V, W, false, false>(q, p, s);
}
template <Kind KIND, typename IO, int V>
cudaError_t launch(int W, const ConvPlan& q, const ConvP& p, cudaStream_t s) {
    return W == 2 ? launch<KIND, IO, V, 2>(q, p, s) : W == 3 ? launch<KIND, IO, V, 3>(q, p, s) : launch<KIND, IO, V, 4>(q, p, s);
}

}  // namespace

size_t conv_bwd_workspace(int B, int T, int D, int W) { return (size_t)conv_bwd_plan(B, T, D).gy * (W + 1) * D * sizeof(float); }

cudaError_t conv_fwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state, void* y,
                     void* last, bool silu, cudaStream_t stream) {
    constexpr int V = kFwdGroup;
    const bool steps = state && state == last;
    const ConvPlan q = steps ? conv_plan(B, T, D, V, 0, T) : conv_plan(B, T, D, V, kSMs * (dtype == QD_BF16 ? 8LL : 4LL) * kConvThreads, 4);
    ConvP p = params(B, T, D, q, silu, D % V == 0);
    p.x = x; p.w = w; p.bias = bias; p.state = state; p.y = y; p.last = last;
    if (steps) return dtype == QD_BF16 ? launch<STEPS, __nv_bfloat16, kFwdGroup>(W, q, p, stream) : launch<STEPS, float, kFwdGroup>(W, q, p, stream);
    return dtype == QD_BF16 ? launch<FWD, __nv_bfloat16, kFwdGroup>(W, q, p, stream) : launch<FWD, float, kFwdGroup>(W, q, p, stream);
}

cudaError_t conv_bwd(int B, int T, int D, int W, int dtype, const void* x, const void* w, const void* bias, const void* state,
                     const void* dy, const void* dlast, void* dx, float* dw, float* dbias, void* dstate, float* part, bool silu,
                     cudaStream_t stream) {
    const ConvPlan q = conv_bwd_plan(B, T, D);
    ConvP p = params(B, T, D, q, silu, D % kBwdGroup == 0);
    p.x = x; p.w = w; p.bias = bias; p.state = state; p.dy = dy; p.dlast = dlast; p.dx = dx; p.dstate = dstate; p.part = part;
    const cudaError_t e = dtype == QD_BF16 ? launch<BWD, __nv_bfloat16, kBwdGroup>(W, q, p, stream) : launch<BWD, float, kBwdGroup>(W, q, p, stream);
    if (e != cudaSuccess) return e;
    return sum_parts(part, (int)q.gy, (long long)(W + 1) * D, (long long)W * D, D, W, dw, dbias, stream);
}

}  // namespace qd

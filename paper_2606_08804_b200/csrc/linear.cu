// Linear attention: which walks (linear.cuh) a forward and a backward are, in how many segments, and the recurrent form.
#include "linear.cuh"
#include "rows.cuh"

#include <initializer_list>

namespace qd {
namespace {

constexpr size_t kStatusBytes = 256;

int linear_chunk(const qd_linear_shape& s) { return s.dtype == QD_BF16 ? 128 : 64; }          // tokens
// CTAs of one walk over whole sequences, for columns of c (fp32: 32 columns of the state to a CTA)
long long linear_ctas(const qd_linear_shape& s, int dc) { return (long long)s.B * s.H * (s.dtype == QD_BF16 ? 1 : dc / 32); }

// Segments of a sequence: as many as make the CTAs' longest run of chunks shortest, launch by launch.  A segment costs its chunks and what a CTA
// needs before its first one; where there are several, the sums of all but the last come first, which take half as long as a walk.
// (32768 tokens of 16 heads in bf16, four of which form every factor: forward 813 us in one segment, 184 in the chosen nine, 224 in ten, 193 in
// eight; backward 883, 427 in the chosen nine, 457 in ten, 434 in five.  Of 14 numbers up to 32 at 14 shapes in bf16 and 19 at eight in fp32 the
// best was at most 6 % faster than the chosen one, but for 777 tokens of 16 heads of 128 x 128 in fp32: 77 for 98, backward 178 for 194.)
int segments_of(const qd_linear_shape& s, bool backward) {
    const int chunk = linear_chunk(s), chunks = (s.T + chunk - 1) / chunk;
    // walks of each launch: o; dq, dk and dv together, or the first two, whose state is transposed, and dv
    const bool together = !backward || s.dk == s.dv;
    const long long first = backward ? linear_ctas(s, s.dk) * (together ? kLinearWalks : 2) : linear_ctas(s, s.dv), second = together ? 0 : linear_ctas(s, s.dv),
                    sums = linear_ctas(s, s.dv) * (backward ? 2 : 1);
    if (first + second > 4 * kSMs) return 1;
    const auto waves = [](long long ctas) { return (double)((ctas + kSMs - 1) / kSMs); };
    int best = 1;
    double least = 1e30;
    for (int n = 1; n <= 32 && n <= chunks; ++n) {
        const int length = (chunks + n - 1) / n;
        if ((chunks + length - 1) / length != n) continue;
        const double cost = (waves(first * n) + waves(second * n)) * (length + 2) + (n > 1 ? 0.5 * waves(sums * (n - 1)) * (length + 2) + 3 : 0);
        if (cost < least) { least = cost; best = n; }
    }
    return best;
}

// The sums of the segments alone, in `ends`, become the states that they begin with: s0, then what is before each, decayed.  A thread has four
// elements of a state; the loads of all segments are under way together.
struct LinearJoin { const float* s0; float* ends; int reverse; };
struct LinearJoins { LinearJoin j[2]; };
constexpr int kJoinThreads = 128;
__global__ void __launch_bounds__(kJoinThreads) k_linear_join(const LinearJoins js, const float* g, int H, int T, int segments, int length, int quads) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const LinearJoin& j = js.j[blockIdx.z];
    const int e = blockIdx.x * kJoinThreads + threadIdx.x;
    const size_t bh = blockIdx.y;
    if (e >= quads) return;
    const float decay = g[bh % H];
    float4* ends = reinterpret_cast<float4*>(j.ends) + bh * segments * quads + e;
    float4 s = j.s0 ? __ldcg(reinterpret_cast<const float4*>(j.s0) + bh * quads + e) : make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int kGroup = 8;
    for (int n0 = 0; n0 < segments; n0 += kGroup) {
        float4 v[kGroup];
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int n = n0 + i, at = j.reverse ? segments - 1 - n : n;
            if (n + 1 < segments) v[i] = __ldcg(ends + (size_t)at * quads);                // nobody begins with the sums of the last one
        }
#pragma unroll
        for (int i = 0; i < kGroup; ++i) {
            const int n = n0 + i, at = j.reverse ? segments - 1 - n : n;
            if (n >= segments) break;
            ends[(size_t)at * quads] = s;
            const Keep keep = keep_power(decay, min(length, T - at * length));
            // a state of 0 stays 0, also across a segment over which a head's factor is beyond fp32 (a batch padded in front)
            auto on = [&](float h, float add) { return h == 0.f ? add : kept(keep, h, add); };
            if (n + 1 < segments) s = make_float4(on(s.x, v[i].x), on(s.y, v[i].y), on(s.z, v[i].z), on(s.w, v[i].w));
        }
    }
}

struct Plan {
    LinearP p;
    float* ends[2];
};
Plan plan(const LinearArgs& a, bool backward) {
    Plan r{};
    const int chunk = linear_chunk(a.s), chunks = (a.s.T + chunk - 1) / chunk, n = segments_of(a.s, backward);
    r.p.T = a.s.T; r.p.H = a.s.H; r.p.BH = a.s.B * a.s.H;
    r.p.segments = n;
    r.p.length = (chunks + n - 1) / n * chunk;
    r.p.g = a.g;
    r.p.scale = a.scale;
    r.p.status = reinterpret_cast<unsigned*>(a.ws);
    const size_t state = (size_t)r.p.BH * n * a.s.dk * a.s.dv;
    for (int i = 0; i < 2; ++i) r.ends[i] = reinterpret_cast<float*>(a.ws + kStatusBytes) + i * state;
    return r;
}
// walks of one shape of state, at most kLinearWalks
cudaError_t walk(LinearP p, std::initializer_list<LinearWalk> ws, int db, int dc, const LinearArgs& a, bool clear) {
    int n = 0;
    for (const LinearWalk& w : ws) p.w[n++] = w;
    p.walks = n;
    p.clear = clear;
    return a.s.dtype == QD_BF16 ? linear_tc(p, db, dc, a.stream) : linear_planes(p, db, dc, a.stream);
}
cudaError_t join(const LinearP& p, std::initializer_list<LinearJoin> js, const LinearArgs& a) {
    LinearJoins all{};
    int n = 0;
    for (const LinearJoin& j : js) all.j[n++] = j;
    const int quads = a.s.dk * a.s.dv / 4;
    return launch_overlapped(k_linear_join, dim3((unsigned)(quads / kJoinThreads), (unsigned)p.BH, (unsigned)n), dim3(kJoinThreads), 0, a.stream, all, p.g,
                             p.H, p.T, p.segments, p.length, quads);
}

}  // namespace

size_t linear_workspace(const qd_linear_shape& s, bool backward) {
    const int n = segments_of(s, backward);
    return kStatusBytes + (n > 1 ? (size_t)(backward ? 2 : 1) * s.B * s.H * n * s.dk * s.dv * 4 : 0);
}

cudaError_t linear_fwd(const LinearArgs& a) {
    const Plan l = plan(a, false);
    const int dk = a.s.dk, dv = a.s.dv;
    const bool cut = l.p.segments > 1;
    if (cut) {
        cudaError_t e = walk(l.p, {LinearWalk{nullptr, a.k, a.v, nullptr, nullptr, nullptr, l.ends[0], 0, a.hT != nullptr, 0}}, dk, dv, a, true);
        if (e == cudaSuccess) e = join(l.p, {LinearJoin{a.h0, l.ends[0], 0}}, a);
        if (e != cudaSuccess) return e;
    }
    return walk(l.p, {LinearWalk{a.q, a.k, a.v, a.o, cut ? l.ends[0] : a.h0, a.hT, nullptr, 0, a.hT != nullptr, 0}}, dk, dv, a, !cut);
}

cudaError_t linear_bwd(const LinearArgs& a) {
    const Plan l = plan(a, true);
    const int dk = a.s.dk, dv = a.s.dv;
    const bool cut = l.p.segments > 1;
    if (cut) {
        cudaError_t e = walk(l.p, {LinearWalk{nullptr, a.k, a.v, nullptr, nullptr, nullptr, l.ends[0], 0, 0, 0},
                                   LinearWalk{nullptr, a.q, a.dO, nullptr, nullptr, nullptr, l.ends[1], 1, a.dh0 != nullptr, 0}}, dk, dv, a, true);
        if (e == cudaSuccess) e = join(l.p, {LinearJoin{a.h0, l.ends[0], 0}, LinearJoin{a.dhT, l.ends[1], 1}}, a);
        if (e != cudaSuccess) return e;
    }
    const float *h = cut ? l.ends[0] : a.h0, *dh = cut ? l.ends[1] : a.dhT;
    const LinearWalk wq{a.dO, a.v, a.k, a.dq, h, nullptr, nullptr, 0, 0, 1}, wk{a.v, a.dO, a.q, a.dk, dh, nullptr, nullptr, 1, 0, 1},
        wv{a.k, a.q, a.dO, a.dv, dh, a.dh0, nullptr, 1, a.dh0 != nullptr, 0};
    if (dk == dv) return walk(l.p, {wq, wk, wv}, dk, dv, a, !cut);
    const cudaError_t e = walk(l.p, {wq, wk}, dv, dk, a, !cut);
    return e == cudaSuccess ? walk(l.p, {wv}, dk, dv, a, false) : e;
}

// ---- single tokens --------------------------------------------------------------------------------------------------------
// S tokens of every sequence, state in place: h <- e^g h + k v^T, o = scale h^T q.  Bound by HBM, one read and one write of the state: a
// CTA has COLS columns of one state, each thread 16 bytes of every RP-th row in registers for all tokens; the read-out's sums over rows go
// through shared memory, a barrier a token.  256 sequences of 16 heads of 128 x 128: 82 us, 6.5 TB/s.
namespace {

constexpr int kStepThreads = 256, kStepTokens = 8;

template <typename IO, int DK, int COLS>
__global__ void __launch_bounds__(kStepThreads) k_linear_steps(int S, int H, int dv, const IO* __restrict__ q, const IO* __restrict__ k,
                                                               const IO* __restrict__ v, const float* __restrict__ g, float* state,
                                                               IO* __restrict__ o, float scale) {
    constexpr int CT = COLS / 4, RP = kStepThreads / CT, NP = DK / RP;
    static_assert(NP >= 1 && DK % RP == 0, "every thread has rows");
    __shared__ float sq[kStepTokens][DK], sk[kStepTokens][DK];
    __shared__ __align__(16) float sv[kStepTokens][COLS], red[2][RP][COLS];
    const int nsl = dv / COLS, bh = blockIdx.x / nsl, j0 = blockIdx.x % nsl * COLS, b = bh / H, h = bh % H;
    const int tid = threadIdx.x, ct = tid % CT, rg = tid / CT;
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    float4* base = reinterpret_cast<float4*>(state + ((size_t)bh * DK + rg) * dv + j0) + ct;
    const size_t step = (size_t)RP * dv / 4;
    float4 st[NP];
#pragma unroll
    for (int i = 0; i < NP; ++i) st[i] = __ldcs(base + i * step);
    const Keep keep = keep_power(g[h], 1);
    for (int s0 = 0; s0 < S; s0 += kStepTokens) {
        const int n = min(kStepTokens, S - s0);
        const size_t row = ((size_t)b * S + s0) * H + h;
        if (s0) __syncthreads();
        for (int i = tid; i < n * DK; i += kStepThreads) {
            const size_t at = (row + (size_t)(i / DK) * H) * DK + i % DK;
            sq[i / DK][i % DK] = scale * ld(q, at);
            sk[i / DK][i % DK] = ld(k, at);
        }
        for (int i = tid; i < n * COLS; i += kStepThreads) sv[i / COLS][i % COLS] = ld(v, (row + (size_t)(i / COLS) * H) * dv + j0 + i % COLS);
        __syncthreads();
        for (int t = 0; t < n; ++t) {
            const float4 vv = *reinterpret_cast<const float4*>(&sv[t][4 * ct]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const float kk = sk[t][i * RP + rg], qq = sq[t][i * RP + rg];
                st[i].x = kept(keep, st[i].x, kk * vv.x); acc.x = fmaf(qq, st[i].x, acc.x);
                st[i].y = kept(keep, st[i].y, kk * vv.y); acc.y = fmaf(qq, st[i].y, acc.y);
                st[i].z = kept(keep, st[i].z, kk * vv.z); acc.z = fmaf(qq, st[i].z, acc.z);
                st[i].w = kept(keep, st[i].w, kk * vv.w); acc.w = fmaf(qq, st[i].w, acc.w);
            }
            float (*part)[COLS] = red[t & 1];
            *reinterpret_cast<float4*>(&part[rg][4 * ct]) = acc;
            __syncthreads();
            if (tid < COLS) {
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < RP; ++i) sum += part[i][tid];
                qd::st(o, (row + (size_t)t * H) * dv + j0 + tid, sum);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < NP; ++i) __stcs(base + i * step, st[i]);
}

template <typename IO, int DK, int COLS>
cudaError_t steps(const LinearArgs& a) {
    return launch_overlapped(k_linear_steps<IO, DK, COLS>, dim3((unsigned)(a.s.B * a.s.H * (a.s.dv / COLS))), dim3(kStepThreads), 0, a.stream, a.s.T,
                             a.s.H, a.s.dv, static_cast<const IO*>(a.q), static_cast<const IO*>(a.k), static_cast<const IO*>(a.v), a.g, a.hT,
                             static_cast<IO*>(a.o), a.scale);
}
template <typename IO>
cudaError_t steps(const LinearArgs& a) {
    // few states: a quarter of a state to a CTA, so that more SMs read
    const bool few = (long long)a.s.B * a.s.H * (a.s.dv / 64) < 2 * kSMs;
    if (a.s.dk == 128) return few ? steps<IO, 128, 32>(a) : steps<IO, 128, 64>(a);
    return few ? steps<IO, 64, 32>(a) : steps<IO, 64, 64>(a);
}

}  // namespace

cudaError_t linear_steps(const LinearArgs& a) { return a.s.dtype == QD_F32 ? steps<float>(a) : steps<__nv_bfloat16>(a); }

}  // namespace qd

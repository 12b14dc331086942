// Forward of the selective scan (scan.cuh).  Per token, channel and state: one exponential and the products dt A, dt u B, a h + ., <C, h>.
// The special function unit gives 4 exponentials per clock and sub-partition, so a warp's 16 x 16 states need 64 clocks of it and 32 of the
// fp32 pipe, softplus and gate another 16: bound by the exponentials, not by HBM, when there are warps enough.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

template <int NB> struct FwdSmem {
    static constexpr int CC = kWalkers / NB * kWarpChannels, NS = NB * kWarpStates;
    float4 dt[2][kTile][CC / 2], x[2][kTile][CC / 2];      // dt, dt u: every pair of channels in both orders
    f2x2 B[2][kTile][NS / 2], C[2][kTile][NS / 2];         // each state's value twice, for both channels of a pair
    float y[2][NB][kTile][CC];
    float bias[CC], skip[CC];
};

template <typename IO, int NB, bool LOCAL>
__global__ void __launch_bounds__(kThreads, 2) k_scan_fwd(const P p) {
    using S = FwdSmem<NB>;
    constexpr int CW = kWalkers / NB, CC = S::CC, NS = S::NS;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    S& sm = *reinterpret_cast<S*>(raw_smem);
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int walked = LOCAL ? p.segs - 1 : p.segs;        // LOCAL: the last segment is not launched
    const int seg = idx % walked, b = idx / walked;
    const int t0 = seg * p.seglen, t1 = min(d.T, t0 + p.seglen), n = (t1 - t0 + kTile - 1) / kTile;

    if (warp < kWalkers) {
        // ---- walk ----------------------------------------------------------------------------------------------------------
        const Map m(lane);
        const int wc = warp % CW, n0 = warp / CW * kWarpStates, ch = ct * CC + wc * kWarpChannels;
        const size_t mine = (((size_t)g * d.ctas + ct) * kWalkers + warp) * kWarpTile + lane * 8;
        f2 A2[4], h[4] = {0, 0, 0, 0}, sum = 0;
        load_decay(p, m, g, ch, n0, A2);
        if (seg == 0) {
            if (p.h0) load_state(p, m, p.h0, b, g, ch, n0, h);
        } else if (!LOCAL) load_end(p, 0, 1, seg, b, mine, h);
        float* saved = p.saved ? p.saved + ((size_t)b * ((d.T + kSave - 1) / kSave) + t0 / kSave) * d.states + mine : nullptr;
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            const int k = i & 1;
            const f2 *dt = reinterpret_cast<const f2*>(sm.dt[k]) + wc * kWarpChannels + m.at, *x = reinterpret_cast<const f2*>(sm.x[k]) + wc * kWarpChannels + m.at;
            const f2x2 *B = &sm.B[k][0][n0 / 2], *C = &sm.C[k][0][n0 / 2];
            float out[kTile / 2];                          // stored when the tile is done: nothing stands in the way of the loads till then
#pragma unroll
            for (int t = 0; t < kTile; t += 2) {
                if (!LOCAL && saved && t % kSave == 0 && t0 + i * kTile + t < t1) {
                    store_tile(saved, h);
                    saved += d.states;
                }
                f2 y[2];
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const f2 vd = dt[(t + s) * CC], vx = x[(t + s) * CC];
                    const f2x2 b0 = B[(t + s) * (NS / 2) + m.pair[0]], b1 = B[(t + s) * (NS / 2) + m.pair[1]];
                    const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b};
#pragma unroll
                    for (int j = 0; j < 4; ++j) h[j] = fma2(exp2_pair(mul2(vd, A2[j])), h[j], mul2(vx, vb[j]));
                    if (LOCAL) sum = add2(sum, vd);
                    else {
                        const f2x2 c0 = C[(t + s) * (NS / 2) + m.pair[0]], c1 = C[(t + s) * (NS / 2) + m.pair[1]];
                        y[s] = fma2(h[3], c1.b, fma2(h[2], c1.a, fma2(h[1], c0.b, mul2(h[0], c0.a))));
                    }
                }
                if (!LOCAL) {
                    // over the four lanes: a lane keeps its first channel, then of the two tokens that of its q / 2
                    const float2 e0 = unpack2(y[0]), e1 = unpack2(y[1]);
                    const float k0 = e0.x + __shfl_xor_sync(0xffffffffu, e0.y, 1), k1 = e1.x + __shfl_xor_sync(0xffffffffu, e1.y, 1);
                    const bool second = m.q & 2;
                    out[t / 2] = (second ? k1 : k0) + __shfl_xor_sync(0xffffffffu, second ? k0 : k1, 2);
                }
            }
            if (!LOCAL)
#pragma unroll
                for (int t = 0; t < kTile; t += 2) sm.y[k][warp / CW][t + (m.q >> 1)][wc * kWarpChannels + m.lo] = out[t / 2];
            __syncthreads();
        }
        if (LOCAL) store_end(p, seg, b, mine, h, A2, sum);
        else if (p.hT && t1 == d.T) store_state(p, m, p.hT, b, g, ch, n0, h);
        return;
    }
    // ---- prepare tiles, write y ------------------------------------------------------------------------------------------------
    const int tid = threadIdx.x - 32 * kWalkers;
    const int it = tid / (CC / 8), ic = tid % (CC / 8) * 8;                // a token of the tile, eight channels of the CTA's
    const int left = it < kTile ? d.K - ct * CC - ic : 0;                  // with NB > 1 some threads have none
    const size_t col = (size_t)g * d.K + ct * CC + ic;
    if (tid < CC) {                                        // read by this half of the CTA only
        const bool in = ct * CC + tid < d.K;
        sm.bias[tid] = p.dt_bias && in ? p.dt_bias[(size_t)g * d.K + ct * CC + tid] : 0.f;
        sm.skip[tid] = p.D && in ? p.D[(size_t)g * d.K + ct * CC + tid] : 0.f;
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads / 2) : "memory");
    struct Raw { Pack<IO, 8> u, dt, z; Pack<IO, 4> bc[NB]; } next;
    struct Held { Pack<IO, 8> u, z; } held[2];                             // of the tiles i, i - 1
    next.u = next.dt = next.z = zero_pack<IO, 8>();
    auto fetch = [&](int tt) {
        const int t = tt + it;
        if (left > 0 && t < t1) {
            const size_t at = ((size_t)b * d.T + t) * d.D + col;
            next.u = load_pack<IO, 8>(static_cast<const IO*>(p.u) + at, left, p.vec);
            next.dt = load_pack<IO, 8>(static_cast<const IO*>(p.dt) + at, left, p.vec);
            if (!LOCAL && p.z) next.z = load_pack<IO, 8>(static_cast<const IO*>(p.z) + at, left, p.vec);
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {                                     // four states of B or C of a token
            const int x = tid + i * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
            next.bc[i] = zero_pack<IO, 4>();
            if (tt + bt < t1 && s < d.N && !(LOCAL && r >= NS / 4))
                next.bc[i] = load_pack<IO, 4>(static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm) + (((size_t)b * d.T + tt + bt) * d.G + g) * d.N + s,
                                              d.N - s, p.vecn);
        }
    };
    auto turn = [&](int tt, int k) {
        if (it < kTile) {
            const bool live = tt + it < t1;
            float fd[8], fx[8];
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                const float2 e = *reinterpret_cast<const float2*>(&sm.bias[ic + i]);
                float2 v = make_float2(pick(next.dt, i) + e.x, pick(next.dt, i + 1) + e.y);
                if (p.softplus) v = softplus(v.x, v.y);
                fd[i] = live && i < left ? v.x : 0.f;
                fd[i + 1] = live && i + 1 < left ? v.y : 0.f;
                fx[i] = live && i < left ? v.x * pick(next.u, i) : 0.f;
                fx[i + 1] = live && i + 1 < left ? v.y * pick(next.u, i + 1) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                store_pairs(&sm.dt[k][it][(ic + i) / 2], fd[i], fd[i + 1], fd[i + 2], fd[i + 3]);
                store_pairs(&sm.x[k][it][(ic + i) / 2], fx[i], fx[i + 1], fx[i + 2], fx[i + 3]);
            }
        }
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int x = tid + i * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
            f2x2* to = r < NS / 4 ? &sm.B[k][bt][s / 2] : &sm.C[k][bt][s / 2];
            to[0] = {both(pick(next.bc[i], 0)), both(pick(next.bc[i], 1))};
            to[1] = {both(pick(next.bc[i], 2)), both(pick(next.bc[i], 3))};
        }
    };
    auto finish = [&](int tt, int k) {
        if (!p.y || left <= 0 || tt + it >= t1) return;
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float s = sm.y[k][0][it][ic + i];
#pragma unroll
            for (int w = 1; w < NB; ++w) s += sm.y[k][w][it][ic + i];
            if (p.D) s = fmaf(sm.skip[ic + i], pick(held[1].u, i), s);
            const float zz = pick(held[1].z, i);
            o[i] = p.z ? s * (zz * gate_sigmoid(zz)) : s;
        }
        store_pack(static_cast<IO*>(p.y) + ((size_t)b * d.T + tt + it) * d.D + col, narrow<IO, 8>(o), left, p.vec);
    };
    fetch(t0);
    turn(t0, 0);
    held[0] = {next.u, next.z};
    if (n > 1) fetch(t0 + kTile);
    __syncthreads();
    for (int i = 0; i < n; ++i) {
        const int tt = t0 + i * kTile;
        if (!LOCAL && i > 0) finish(tt - kTile, (i - 1) & 1);
        held[1] = held[0];
        if (i + 1 < n) {
            turn(tt + kTile, (i + 1) & 1);
            held[0] = {next.u, next.z};
            if (i + 2 < n) fetch(tt + 2 * kTile);
        }
        __syncthreads();
    }
    if (!LOCAL) finish(t0 + (n - 1) * kTile, (n - 1) & 1);
}

}  // namespace

namespace scan {
namespace {
__global__ void __launch_bounds__(256) k_join(float* ends, const float* decays, int n, int from, int step, size_t count) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    float h = ends[(size_t)from * count + i];
#pragma unroll 4
    for (int k = 1; k < n; ++k) {
        const size_t at = (size_t)(from + k * step) * count + i;
        h = fmaf(decays[at], h, ends[at]);
        ends[at] = h;
    }
}
}  // namespace

// The segments are from, from + step, ..
cudaError_t join(float* ends, const float* decays, int n, int from, int step, size_t count, cudaStream_t stream) {
    return launch_overlapped(k_join, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, stream, ends, decays, n, from, step, count);
}

// As many segments as fill the GPU twice over, none where that would be fewer than three (walking all but the last twice costs what two
// gain), each of four tiles at least.
Cut cut(const Dims& d) {
    const long long units = (long long)d.B * d.G * d.ctas;
    long long n = 2 * kSMs / units;
    if (n < 3) n = 1;
    const long long most = d.T / (2 * kTile);
    if (n > most) n = most;
    if (n < 1) n = 1;
    const long long per = (d.T + n - 1) / n;
    Cut c;
    c.len = (int)((per + kTile - 1) / kTile * kTile);
    c.segs = (int)(((long long)d.T + c.len - 1) / c.len);
    return c;
}
}  // namespace scan

namespace {
struct FwdPlan { Dims d; Cut c; size_t saved, ends, bytes; };
FwdPlan fwd_plan(const qd_scan_shape& s, bool save) {
    FwdPlan q{};
    q.d = dims(s);
    q.c = cut(q.d);
    q.saved = save ? (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float) : 0;
    q.ends = (size_t)(q.c.segs - 1) * s.B * q.d.states * sizeof(float);
    q.bytes = q.saved + 2 * q.ends;
    return q;
}

template <typename IO, int NB>
cudaError_t launch(P p, cudaStream_t stream) {
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    constexpr size_t smem = sizeof(FwdSmem<NB>);
    cudaError_t e;
    if (p.segs > 1) {
        e = set_max_smem_once((const void*)k_scan_fwd<IO, NB, true>, smem);
        if (e == cudaSuccess)
            e = launch_overlapped(k_scan_fwd<IO, NB, true>, dim3((unsigned)(per * (p.segs - 1))), dim3(kThreads), smem, stream, p);
        if (e == cudaSuccess && p.joined) e = join(p.ends, p.decays, p.segs - 1, 0, 1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    e = set_max_smem_once((const void*)k_scan_fwd<IO, NB, false>, smem);
    if (e != cudaSuccess) return e;
    return launch_overlapped(k_scan_fwd<IO, NB, false>, dim3((unsigned)(per * p.segs)), dim3(kThreads), smem, stream, p);
}
template <typename IO>
cudaError_t launch(const P& p, cudaStream_t stream) {
    return p.d.nb == 1 ? launch<IO, 1>(p, stream) : p.d.nb == 2 ? launch<IO, 2>(p, stream) : launch<IO, 4>(p, stream);
}
}  // namespace

size_t scan_fwd_workspace(const qd_scan_shape& s, bool save) { return fwd_plan(s, save).bytes; }

cudaError_t scan_fwd(const ScanArgs& a) {
    const FwdPlan q = fwd_plan(a.s, a.save);
    P p{};
    p.d = q.d; p.segs = q.c.segs; p.seglen = q.c.len;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.D = a.D; p.dt_bias = a.dt_bias; p.h0 = a.h0;
    p.y = a.y; p.hT = a.hT;
    p.saved = a.save ? reinterpret_cast<float*>(a.ws) : nullptr;
    p.ends = reinterpret_cast<float*>(a.ws + q.saved);
    p.decays = reinterpret_cast<float*>(a.ws + q.saved + q.ends);
    p.softplus = a.softplus; p.vec = q.d.K % 8 == 0; p.vecn = a.s.N % 4 == 0;
    p.joined = p.segs - 1 > kMostJoined;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.stream) : launch<float>(p, a.stream);
}

}  // namespace qd

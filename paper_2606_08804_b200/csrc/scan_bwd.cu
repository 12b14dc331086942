// Backward of the selective scan (scan.cuh).  With g_t = dL/dh_t = dy_t C_t + a_{t+1} g_{t+1} (dy after the factor of z) and p_t = a_t h_{t-1}:
//   dC_t = sum_channels dy_t h_t        dB_t = sum_channels dt_t u_t g_t        du = dt <g, B> + D dy
//   ddt = u <g, B> + <g p, A>           dA = sum_t dt g p                       dh0 = a_1 g_1,   dz = dy y_raw SiLU'(z).
// The forward saved the state before every kSave-th token; from the last such tile to the first the states of its tokens are walked anew,
// a_t and p_t of all of them kept in registers (p, not h - dt u B, so that a small p keeps its precision), and then g is walked back.
// Per token, channel and state one exponential and 13 operations of the fp32 pipe: bound by that pipe and by what is issued beside it.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

constexpr unsigned kAll = 0xffffffffu;
constexpr int kWalkRegs = 184, kPrepareRegs = 72;          // of 2 x 128: what the launch gives a pair of threads, one of each role

template <int NB> struct BwdSmem {
    static constexpr int CC = kWalkers / NB * kWarpChannels, NS = NB * kWarpStates;
    float4 dt[2][kSave][CC / 2], x[2][kSave][CC / 2], dy[2][kSave][CC / 2];      // every pair of channels in both orders
    f2x2 B[2][kSave][NS / 2], C[2][kSave][NS / 2];         // each state's value twice
    float gB[2][NB][kSave][CC], gpA[2][NB][kSave][CC], y[2][NB][kSave][CC];
    float bc[2][kWalkers][kSave][32];                      // dB, dC summed over a warp's channels
    float bias[CC], skip[CC];
};

template <typename IO, int NB, bool LOCAL>
__global__ void __launch_bounds__(kThreads, 2) k_scan_bwd(const P p) {
    using S = BwdSmem<NB>;
    constexpr int CW = kWalkers / NB, CC = S::CC, NS = S::NS, K = kSave;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    S& sm = *reinterpret_cast<S*>(raw_smem);
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int warp = sm100::warp_index(), lane = threadIdx.x & 31;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int walked = LOCAL ? p.segs - 1 : p.segs;        // LOCAL: the first segment is not launched
    const int seg = idx % walked + (LOCAL ? 1 : 0), b = idx / walked;
    const int t0 = seg * p.seglen, t1 = min(d.T, t0 + p.seglen), n = (t1 - t0 + K - 1) / K;
    const size_t part = (size_t)seg * d.B + b;

    if (warp < kWalkers) {
        // ---- walk ----------------------------------------------------------------------------------------------------------
        if constexpr (!LOCAL) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWalkRegs));
        const Map m(lane);
        const int wc = warp % CW, wb = warp / CW, n0 = wb * kWarpStates, ch = ct * CC + wc * kWarpChannels;
        const size_t mine = (((size_t)g * d.ctas + ct) * kWalkers + warp) * kWarpTile + lane * 8;
        f2 A2[4], ga[4] = {0, 0, 0, 0}, dA[4] = {0, 0, 0, 0}, sum = 0;     // ga = a_{t+1} g_{t+1}
        load_decay(p, m, g, ch, n0, A2);
        if (seg == p.segs - 1) {
            if (p.dhT) load_state(p, m, p.dhT, b, g, ch, n0, ga);
        } else if (!LOCAL) load_end(p, p.segs - 2, -1, p.segs - 1 - seg, b, mine, ga);
        const float* saved = LOCAL ? nullptr : p.saved + ((size_t)b * ((d.T + K - 1) / K) + t0 / K) * d.states + mine;
        f2 h[4];
        if (!LOCAL) load_tile(saved + (size_t)(n - 1) * d.states, h);
        __syncthreads();
        for (int i = n - 1; i >= 0; --i) {
            const int k = i & 1;
            const f2 *dt = reinterpret_cast<const f2*>(sm.dt[k]) + wc * kWarpChannels + m.at, *x = reinterpret_cast<const f2*>(sm.x[k]) + wc * kWarpChannels + m.at;
            const f2* dy = reinterpret_cast<const f2*>(sm.dy[k]) + wc * kWarpChannels + m.at;
            const f2x2 *B = &sm.B[k][0][n0 / 2], *C = &sm.C[k][0][n0 / 2];
            if constexpr (LOCAL) {
#pragma unroll
                for (int t = K - 1; t >= 0; --t) {
                    const f2 vd = dt[t * CC], vy = dy[t * CC];
                    const f2x2 c0 = C[t * (NS / 2) + m.pair[0]], c1 = C[t * (NS / 2) + m.pair[1]];
                    const f2 vc[4] = {c0.a, c0.b, c1.a, c1.b};
#pragma unroll
                    for (int j = 0; j < 4; ++j) ga[j] = mul2(exp2_pair(mul2(vd, A2[j])), fma2(vy, vc[j], ga[j]));
                    sum = add2(sum, vd);
                }
            } else {
                f2 a[K][4], pr[K][4], tA[4];
#pragma unroll
                for (int t = 0; t < K; ++t) {
                    const f2 vd = dt[t * CC], vx = x[t * CC];
                    const f2x2 b0 = B[t * (NS / 2) + m.pair[0]], b1 = B[t * (NS / 2) + m.pair[1]];
                    const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b};
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        a[t][j] = exp2_pair(mul2(vd, A2[j]));
                        pr[t][j] = mul2(a[t][j], h[j]);
                        h[j] = fma2(vx, vb[j], pr[t][j]);
                    }
                }
                // stored when the tile is done: nothing stands in the way of the loads till then
                float held = 0.f, out_bc[K], out_g[K], out_y[K / 2];
                const bool odd = lane & 4, up = lane & 16, second = m.q & 2;
#pragma unroll
                for (int t = K - 1; t >= 0; --t) {
                    const f2 vd = dt[t * CC], vx = x[t * CC], vy = dy[t * CC];
                    const f2x2 b0 = B[t * (NS / 2) + m.pair[0]], b1 = B[t * (NS / 2) + m.pair[1]];
                    const f2x2 c0 = C[t * (NS / 2) + m.pair[0]], c1 = C[t * (NS / 2) + m.pair[1]];
                    const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b}, vc[4] = {c0.a, c0.b, c1.a, c1.b};
                    const float2 xs = unpack2(vx), ys = unpack2(vy);
                    f2 r1 = 0, r2 = 0, r3 = 0;
                    float vB[4], vC[4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f2 ht = fma2(vx, vb[j], pr[t][j]), gt = fma2(vy, vc[j], ga[j]), gp = mul2(gt, pr[t][j]);
                        const float2 hs = unpack2(ht), gs = unpack2(gt);
                        vB[j] = fmaf(gs.y, xs.y, gs.x * xs.x);
                        vC[j] = fmaf(hs.y, ys.y, hs.x * ys.x);
                        r1 = j ? fma2(gt, vb[j], r1) : mul2(gt, vb[j]);
                        r2 = j ? fma2(gp, A2[j], r2) : mul2(gp, A2[j]);
                        r3 = j ? fma2(ht, vc[j], r3) : mul2(ht, vc[j]);
                        tA[j] = t == K - 1 ? mul2(gp, vd) : fma2(gp, vd, tA[j]);
                        ga[j] = mul2(gt, a[t][j]);
                    }
                    // dB, dC over the eight lanes of equal q: a lane keeps its first pair of states, of that the state c & 1, of dB and dC
                    // that of c / 4
                    float w0 = vB[0] + __shfl_xor_sync(kAll, vB[2], 8), w1 = vB[1] + __shfl_xor_sync(kAll, vB[3], 8);
                    const float kB = (odd ? w1 : w0) + __shfl_xor_sync(kAll, odd ? w0 : w1, 4);
                    w0 = vC[0] + __shfl_xor_sync(kAll, vC[2], 8);
                    w1 = vC[1] + __shfl_xor_sync(kAll, vC[3], 8);
                    const float kC = (odd ? w1 : w0) + __shfl_xor_sync(kAll, odd ? w0 : w1, 4);
                    out_bc[t] = (up ? kC : kB) + __shfl_xor_sync(kAll, up ? kB : kC, 16);
                    // <g, B>, <g p, A>, <C, h> over the four lanes of equal c: a lane keeps its first channel, of the first two that of q / 2;
                    // of the third it keeps one of two tokens
                    const float2 e1 = unpack2(r1), e2 = unpack2(r2), e3 = unpack2(r3);
                    const float k1 = e1.x + __shfl_xor_sync(kAll, e1.y, 1), k2 = e2.x + __shfl_xor_sync(kAll, e2.y, 1);
                    const float k3 = e3.x + __shfl_xor_sync(kAll, e3.y, 1);
                    out_g[t] = (second ? k2 : k1) + __shfl_xor_sync(kAll, second ? k1 : k2, 2);
                    if (t & 1) held = k3;
                    else out_y[t / 2] = (second ? held : k3) + __shfl_xor_sync(kAll, second ? k3 : held, 2);
                    // the tile before: its state, in the registers of tokens that are done
                    if (t == K / 2 && i > 0) load_tile(saved + (size_t)(i - 1) * d.states, h);
                }
                float* g_to = &(second ? sm.gpA : sm.gB)[k][wb][0][wc * kWarpChannels + m.lo];
                float* bc_to = &sm.bc[k][warp][0][(up ? 16 : 0) + 2 * m.pair[0] + (odd ? 1 : 0)];
#pragma unroll
                for (int t = 0; t < K; ++t) {
                    bc_to[t * 32] = out_bc[t];
                    g_to[t * CC] = out_g[t];
                    if (!(t & 1)) sm.y[k][wb][t + (m.q >> 1)][wc * kWarpChannels + m.lo] = out_y[t / 2];
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) dA[j] = add2(dA[j], tA[j]);    // a tile's sum first: 2000 tokens one by one lose two digits
            }
            __syncthreads();
        }
        if (LOCAL) store_end(p, seg - 1, b, mine, ga, A2, sum);
        else {
            // [part][D][N]: the state of sequence `part`
            store_state(p, m, p.pA + (part - b) * d.D * d.N, b, g, ch, n0, dA);
            if (seg == 0 && p.dh0) store_state(p, m, p.dh0, b, g, ch, n0, ga);
        }
        if (!LOCAL) {
            __syncthreads();
            __syncthreads();
        }
        return;
    }
    // ---- prepare tiles, write gradients ---------------------------------------------------------------------------------------
    if constexpr (!LOCAL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPrepareRegs));
    constexpr int BCT = (NB + 1) / 2;                                      // groups of four states of B and C that a thread stages
    const int tid = threadIdx.x - 32 * kWalkers;
    const int it = tid / (CC / 4), ic = tid % (CC / 4) * 4;                // a token of the tile, four channels of the CTA's
    const int left = it < K ? d.K - ct * CC - ic : 0;
    const size_t col = (size_t)g * d.K + ct * CC + ic;
    if (tid < CC) {                                        // read by this half of the CTA only
        const bool in = ct * CC + tid < d.K;
        sm.bias[tid] = p.dt_bias && in ? p.dt_bias[(size_t)g * d.K + ct * CC + tid] : 0.f;
        sm.skip[tid] = p.D && in ? p.D[(size_t)g * d.K + ct * CC + tid] : 0.f;
    }
    asm volatile("bar.sync 1, %0;" ::"n"(kThreads / 2) : "memory");
    struct Raw { Pack<IO, 4> u, dt, z, y; } next, held[2];                 // held: of the tiles i, i + 1
    Pack<IO, 4> bc[BCT];
    float sumD[4] = {0.f, 0.f, 0.f, 0.f}, sumb[4] = {0.f, 0.f, 0.f, 0.f};
    next.u = next.dt = next.z = next.y = zero_pack<IO, 4>();
    auto fetch = [&](int tt) {
        const int t = tt + it;
        if (left > 0 && t < t1) {
            const size_t at = ((size_t)b * d.T + t) * d.D + col;
            if (!LOCAL) next.u = load_pack<IO, 4>(static_cast<const IO*>(p.u) + at, left, p.vec);
            next.dt = load_pack<IO, 4>(static_cast<const IO*>(p.dt) + at, left, p.vec);
            next.y = load_pack<IO, 4>(static_cast<const IO*>(p.dy) + at, left, p.vec);
            if (p.z) next.z = load_pack<IO, 4>(static_cast<const IO*>(p.z) + at, left, p.vec);
        }
#pragma unroll
        for (int i = 0; i < BCT; ++i) {
            const int x = tid + i * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
            bc[i] = zero_pack<IO, 4>();
            if (bt < K && tt + bt < t1 && s < d.N && !(LOCAL && r < NS / 4))
                bc[i] = load_pack<IO, 4>(static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm) + (((size_t)b * d.T + tt + bt) * d.G + g) * d.N + s,
                                         d.N - s, p.vecn);
        }
    };
    auto turn = [&](int tt, int k) {
        if (it < K) {
            const bool live = tt + it < t1;
            float fd[4], fx[4], fy[4];
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const float2 bi = *reinterpret_cast<const float2*>(&sm.bias[ic + i]);
                float2 v = make_float2(pick(next.dt, i) + bi.x, pick(next.dt, i + 1) + bi.y);
                if (p.softplus) v = softplus(v.x, v.y);
                const float e[2] = {v.x, v.y};
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const bool on = live && i + o < left;
                    const float z = pick(next.z, i + o), y = pick(next.y, i + o);
                    fd[i + o] = on ? e[o] : 0.f;
                    fx[i + o] = on && !LOCAL ? e[o] * pick(next.u, i + o) : 0.f;
                    fy[i + o] = on ? (p.z ? y * (z * gate_sigmoid(z)) : y) : 0.f;
                }
            }
            store_pairs(&sm.dt[k][it][ic / 2], fd[0], fd[1], fd[2], fd[3]);
            if (!LOCAL) store_pairs(&sm.x[k][it][ic / 2], fx[0], fx[1], fx[2], fx[3]);
            store_pairs(&sm.dy[k][it][ic / 2], fy[0], fy[1], fy[2], fy[3]);
        }
#pragma unroll
        for (int i = 0; i < BCT; ++i) {
            const int x = tid + i * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
            if (bt >= K) continue;
            f2x2* to = r < NS / 4 ? &sm.B[k][bt][s / 2] : &sm.C[k][bt][s / 2];
            to[0] = {both(pick(bc[i], 0)), both(pick(bc[i], 1))};
            to[1] = {both(pick(bc[i], 2)), both(pick(bc[i], 3))};
        }
    };
    // of a tile that has been walked; it is prepared over only afterwards, and a thread reads what it wrote there itself
    auto finish = [&](int tt, int k) {
        if (left > 0 && tt + it < t1) {
            const Raw& r = held[1];
            const float4 d0 = sm.dt[k][it][ic / 2], d1 = sm.dt[k][it][ic / 2 + 1], y0 = sm.dy[k][it][ic / 2], y1 = sm.dy[k][it][ic / 2 + 1];
            const float vdt[4] = {d0.x, d0.y, d1.x, d1.y}, vdy[4] = {y0.x, y0.y, y1.x, y1.y};
            float odu[4], odt[4], odz[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float e1 = 0.f, e2 = 0.f, ey = 0.f;
#pragma unroll
                for (int w = 0; w < NB; ++w) { e1 += sm.gB[k][w][it][ic + i]; e2 += sm.gpA[k][w][it][ic + i]; ey += sm.y[k][w][it][ic + i]; }
                const float uu = pick(r.u, i), sk = sm.skip[ic + i];
                odu[i] = fmaf(e1, vdt[i], sk * vdy[i]);
                odt[i] = fmaf(e1, uu, e2 * kLn2);
                if (p.softplus) odt[i] *= gate_sigmoid(pick(r.dt, i) + sm.bias[ic + i]);
                sumD[i] = fmaf(vdy[i], uu, sumD[i]);
                sumb[i] += odt[i];
                const float zz = pick(r.z, i), sg = gate_sigmoid(zz);
                odz[i] = pick(r.y, i) * fmaf(sk, uu, ey) * (sg * fmaf(zz, 1.f - sg, 1.f));
            }
            const size_t at = ((size_t)b * d.T + tt + it) * d.D + col;
            store_pack(static_cast<IO*>(p.du) + at, narrow<IO, 4>(odu), left, p.vec);
            store_pack(static_cast<IO*>(p.ddt) + at, narrow<IO, 4>(odt), left, p.vec);
            if (p.z) store_pack(static_cast<IO*>(p.dz) + at, narrow<IO, 4>(odz), left, p.vec);
        }
        const size_t rows = (size_t)d.B * d.T * d.G * d.N;
#pragma unroll
        for (int x = tid; x < K * 2 * NS; x += 128) {
            const int t = x / (2 * NS), which = x / NS % 2, s = x % NS;
            if (tt + t >= t1 || s >= d.N) continue;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < CW; ++w) v += sm.bc[k][s / kWarpStates * CW + w][t][which * 16 + s % kWarpStates];
            p.pBC[((size_t)ct * 2 + which) * rows + (((size_t)b * d.T + tt + t) * d.G + g) * d.N + s] = v;
        }
    };
    fetch(t0 + (n - 1) * K);
    turn(t0 + (n - 1) * K, (n - 1) & 1);
    held[0] = next;
    if (n > 1) fetch(t0 + (n - 2) * K);
    __syncthreads();
    for (int i = n - 1; i >= 0; --i) {
        const int tt = t0 + i * K;
        if (!LOCAL && i < n - 1) finish(tt + K, (i + 1) & 1);
        held[1] = held[0];
        if (i > 0) {
            turn(tt - K, (i - 1) & 1);
            held[0] = next;
            if (i > 1) fetch(tt - 2 * K);
        }
        __syncthreads();
    }
    if (LOCAL) return;
    finish(t0, 0);
    // sums over the tokens of a channel: the rows of a tile in order (the walkers are at the same barriers)
    float* cols = reinterpret_cast<float*>(sm.x);
    __syncthreads();
    if (it < K)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cols[it * CC + ic + i] = sumD[i];
            cols[(K + it) * CC + ic + i] = sumb[i];
        }
    __syncthreads();
    for (int x = tid; x < 2 * CC; x += 128) {
        const int which = x / CC, c = x % CC;
        if (ct * CC + c >= d.K) continue;
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < K; ++r) v += cols[(which * K + r) * CC + c];
        p.pD[(part * 2 + which) * d.D + (size_t)g * d.K + ct * CC + c] = v;
    }
}

// dB and dC from the CTAs' partials, in their order.
template <typename IO>
__global__ void __launch_bounds__(256) k_sum_bc(const float* part, int parts, size_t rows, IO* dB, IO* dC) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= 2 * rows) return;
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += part[(size_t)k * 2 * rows + i];
    st(i < rows ? dB : dC, i < rows ? i : i - rows, v);
}

struct BwdPlan { Dims d; Cut c; size_t saved, ends, pA, pD, pBC, bytes; };
BwdPlan bwd_plan(const qd_scan_shape& s) {
    BwdPlan q{};
    q.d = dims(s);
    q.c = cut(q.d);
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    q.saved = (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float);
    q.ends = (size_t)(q.c.segs - 1) * s.B * q.d.states * sizeof(float);
    q.pA = up((size_t)q.c.segs * s.B * s.D * s.N * sizeof(float));
    q.pD = up((size_t)q.c.segs * s.B * 2 * s.D * sizeof(float));
    q.pBC = up((size_t)q.d.ctas * 2 * s.B * s.T * s.G * s.N * sizeof(float));
    q.bytes = q.saved + 2 * q.ends + q.pA + q.pD + q.pBC;                  // more than a saving forward's
    return q;
}

template <typename IO, int NB>
cudaError_t launch(const P& p, cudaStream_t stream) {
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    constexpr size_t smem = sizeof(BwdSmem<NB>);
    cudaError_t e;
    if (p.segs > 1) {
        e = set_max_smem_once((const void*)k_scan_bwd<IO, NB, true>, smem);
        if (e == cudaSuccess)
            e = launch_overlapped(k_scan_bwd<IO, NB, true>, dim3((unsigned)(per * (p.segs - 1))), dim3(kThreads), smem, stream, p);
        if (e == cudaSuccess && p.joined) e = join(p.ends, p.decays, p.segs - 1, p.segs - 2, -1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    e = set_max_smem_once((const void*)k_scan_bwd<IO, NB, false>, smem);
    if (e != cudaSuccess) return e;
    return launch_overlapped(k_scan_bwd<IO, NB, false>, dim3((unsigned)(per * p.segs)), dim3(kThreads), smem, stream, p);
}
template <typename IO>
cudaError_t launch(const P& p, const ScanArgs& a) {
    cudaError_t e = p.d.nb == 1 ? launch<IO, 1>(p, a.stream) : p.d.nb == 2 ? launch<IO, 2>(p, a.stream) : launch<IO, 4>(p, a.stream);
    if (e != cudaSuccess) return e;
    const size_t rows = (size_t)p.d.B * p.d.T * p.d.G * p.d.N;
    return launch_overlapped(k_sum_bc<IO>, dim3((unsigned)((2 * rows + 255) / 256)), dim3(256), 0, a.stream, p.pBC, p.d.ctas, rows,
                             static_cast<IO*>(a.dBm), static_cast<IO*>(a.dCm));
}
}  // namespace

size_t scan_bwd_workspace(const qd_scan_shape& s) { return bwd_plan(s).bytes; }

cudaError_t scan_bwd(const ScanArgs& a) {
    const BwdPlan q = bwd_plan(a.s);
    P p{};
    p.d = q.d; p.segs = q.c.segs; p.seglen = q.c.len;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.D = a.D; p.dt_bias = a.dt_bias;
    p.dy = a.dy; p.dhT = a.dhT; p.du = a.du; p.ddt = a.ddt; p.dz = a.dz; p.dh0 = a.dh0;
    char* w = a.ws;
    p.saved = reinterpret_cast<float*>(w); w += q.saved;
    p.ends = reinterpret_cast<float*>(w); w += q.ends;
    p.decays = reinterpret_cast<float*>(w); w += q.ends;
    p.pA = reinterpret_cast<float*>(w); w += q.pA;
    p.pD = reinterpret_cast<float*>(w); w += q.pD;
    p.pBC = reinterpret_cast<float*>(w);
    p.softplus = a.softplus; p.vec = q.d.K % 4 == 0; p.vecn = a.s.N % 4 == 0;
    p.joined = p.segs - 1 > kMostJoined;
    cudaError_t e = a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a) : launch<float>(p, a);
    if (e != cudaSuccess) return e;
    const long long D = a.s.D, DN = D * a.s.N;
    const int parts = q.c.segs * a.s.B;
    e = sum_parts(p.pA, parts, DN, DN, DN, 1, a.dA, nullptr, a.stream);
    if (e != cudaSuccess || (!a.dD && !a.ddt_bias)) return e;
    return sum_parts(p.pD, parts, 2 * D, D, D, 1, a.dD, a.ddt_bias, a.stream);
}

}  // namespace qd

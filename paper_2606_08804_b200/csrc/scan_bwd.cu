// Backward of the selective scan (scan.cuh).  With g_t = dL/dh_t = dy_t C_t + a_{t+1} g_{t+1} (dy after the factor of z) and p_t = a_t h_{t-1}:
//   dC_t = sum_channels dy_t h_t        dB_t = sum_channels dt_t u_t g_t        du = dt <g, B> + D dy
//   ddt = u <g, B> + <g p, A>           dA = sum_t dt g p                       dh0 = a_1 g_1,   dz = dy y_raw SiLU'(z).
// The forward saved the state before every kSave-th token; from the last such chunk to the first the states of its tokens are walked anew,
// a_t and p_t of all of them kept in registers (p, not h - dt u B, so that a small p keeps its precision), and then g is walked back.
// Per token, channel and state one exponential and 13 operations of the fp32 pipe: bound by that pipe and by what is issued beside it.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

// v[0 .. 7] over the eight lanes of equal q: lane c ends with the sum of v[c].
__device__ __forceinline__ float spread8(const float (&v)[8], int lane) {
    float w[4], x[2];
    const bool b2 = lane & 16, b1 = lane & 8, b0 = lane & 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (b2 ? v[4 + i] : v[i]) + __shfl_xor_sync(0xffffffffu, b2 ? v[i] : v[4 + i], 16);
#pragma unroll
    for (int i = 0; i < 2; ++i) x[i] = (b1 ? w[2 + i] : w[i]) + __shfl_xor_sync(0xffffffffu, b1 ? w[i] : w[2 + i], 8);
    return (b0 ? x[1] : x[0]) + __shfl_xor_sync(0xffffffffu, b0 ? x[0] : x[1], 4);
}
// v[0 .. 3] over the four lanes of equal c: lane q ends with the sum of v[q].
__device__ __forceinline__ float spread4(const float (&v)[4], int lane) {
    float w[2];
    const bool b1 = lane & 2, b0 = lane & 1;
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = (b1 ? v[2 + i] : v[i]) + __shfl_xor_sync(0xffffffffu, b1 ? v[i] : v[2 + i], 2);
    return (b0 ? w[1] : w[0]) + __shfl_xor_sync(0xffffffffu, b0 ? w[0] : w[1], 1);
}

template <typename IO, int NB, bool LOCAL>
__global__ void __launch_bounds__(NB == 1 ? 128 : 64 * NB) k_scan_bwd(const P p) {
    constexpr int CW = NB == 1 ? 4 : 2, NT = 32 * CW * NB, CC = CW * kWarpChannels, NS = NB * kWarpStates, K = kSave;
    constexpr int ITEMS = K * CC / 4;                      // groups of four channels of a chunk
    constexpr int BCI = K * 2 * (NS / 4), BCT = (BCI + NT - 1) / NT;
    static_assert(ITEMS <= NT, "a thread has one group of channels");
    __shared__ __align__(16) float sdt[K][CC], sx[K][CC], sdy[K][CC];
    __shared__ __align__(16) f2 sB[K][NS], sC[K][NS];
    __shared__ float s1[NB][K][CC], s2[NB][K][CC], sy[NB][K][CC];
    __shared__ float red[CW * NB][K][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, c = lane >> 2;
    const int wc = warp % CW, wb = warp / CW;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int walked = LOCAL ? p.segs - 1 : p.segs;        // LOCAL: the first segment is not launched
    const int seg = idx % walked + (LOCAL ? 1 : 0), b = idx / walked;
    const int t0 = seg * p.seglen, t1 = min(d.T, t0 + p.seglen);
    const int ch = ct * CC + wc * kWarpChannels + 2 * c;
    const int n0 = wb * kWarpStates + 4 * q;
    const size_t tile = (((size_t)g * d.ctas + ct) * CW + wc) * NB + wb;
    const size_t row = (size_t)g * d.K + ch;
    const bool in0 = ch < d.K, in1 = ch + 1 < d.K;

    f2 A2[4], ga[4], dA[4];                                // ga = a_{t+1} g_{t+1}
    float2 sum = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        const bool in = n0 + n < d.N;
        A2[n] = pack2(in && in0 ? p.A[row * d.N + n0 + n] * kLog2e : 0.f, in && in1 ? p.A[(row + 1) * d.N + n0 + n] * kLog2e : 0.f);
        dA[n] = 0;
        ga[n] = 0;
        if (seg == p.segs - 1) {
            if (p.dhT) {
                const float* s = p.dhT + ((size_t)b * d.D + row) * d.N + n0 + n;
                ga[n] = pack2(in && in0 ? s[0] : 0.f, in && in1 ? s[d.N] : 0.f);
            }
        } else if (!LOCAL) {
            const float* s = p.ends + ((size_t)seg * d.B + b) * d.states + tile * kWarpTile + lane * 8;
            ga[n] = pack2(s[2 * n], s[2 * n + 1]);
        }
    }
    const int it = tid / (CC / 4), ic = tid % (CC / 4) * 4;
    const int left = tid < ITEMS ? d.K - ct * CC - ic : 0;
    const size_t col = (size_t)g * d.K + ct * CC + ic;
    Pack<IO, 4> ru = zero_pack<IO, 4>(), rdt = ru, rz = ru, ry = ru;
    Pack<IO, 4> rbc[BCT];
    f2x2 rh[2] = {{0, 0}, {0, 0}};
    float bias[4], skip[4], sumD[4], sumb[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bias[i] = p.dt_bias && i < left ? p.dt_bias[col + i] : 0.f;
        skip[i] = !LOCAL && p.D && i < left ? p.D[col + i] : 0.f;
        sumD[i] = 0.f;
        sumb[i] = 0.f;
    }
    auto fetch = [&](int tt) {
        const int t = tt + it;
        if (left > 0 && t < t1) {
            const size_t at = ((size_t)b * d.T + t) * d.D + col;
            if (!LOCAL) ru = load_pack<IO, 4>(static_cast<const IO*>(p.u) + at, left, p.vec);
            rdt = load_pack<IO, 4>(static_cast<const IO*>(p.dt) + at, left, p.vec);
            ry = load_pack<IO, 4>(static_cast<const IO*>(p.dy) + at, left, p.vec);
            if (p.z) rz = load_pack<IO, 4>(static_cast<const IO*>(p.z) + at, left, p.vec);
        }
#pragma unroll
        for (int i = 0; i < BCT; ++i) {
            const int x = tid + i * NT, bt = x / (NS / 2), r = x % (NS / 2), n = r % (NS / 4) * 4;
            const IO* src = static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm);
            rbc[i] = zero_pack<IO, 4>();
            if (x < BCI && tt + bt < t1 && n < d.N && !(LOCAL && r < NS / 4))
                rbc[i] = load_pack<IO, 4>(src + (((size_t)b * d.T + tt + bt) * d.G + g) * d.N + n, d.N - n, p.vecn);
        }
        if (!LOCAL) {
            const f2x2* from = reinterpret_cast<const f2x2*>(p.saved + ((size_t)b * ((d.T + K - 1) / K) + tt / K) * d.states + tile * kWarpTile + lane * 8);
            rh[0] = from[0];
            rh[1] = from[1];
        }
    };
    const int last = t0 + (t1 - t0 - 1) / K * K;
    fetch(last);
    for (int tt = last; tt >= t0; tt -= K) {
        const Pack<IO, 4> u = ru, z = rz, y = ry, raw = rdt;
        f2 h[4] = {rh[0].a, rh[0].b, rh[1].a, rh[1].b};
        const bool live = left > 0 && tt + it < t1;
        float vdt[4], vdy[4];
        if (tid < ITEMS) {
            float fx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool on = live && i < left;
                const float r = pick(raw, i) + bias[i], zz = pick(z, i);
                vdt[i] = on ? (p.softplus ? softplus(r) : r) : 0.f;
                vdy[i] = on ? (p.z ? pick(y, i) * (zz * sigmoid(zz)) : pick(y, i)) : 0.f;
                fx[i] = on ? vdt[i] * pick(u, i) : 0.f;
            }
            *reinterpret_cast<float4*>(&sdt[it][ic]) = make_float4(vdt[0], vdt[1], vdt[2], vdt[3]);
            *reinterpret_cast<float4*>(&sx[it][ic]) = make_float4(fx[0], fx[1], fx[2], fx[3]);
            *reinterpret_cast<float4*>(&sdy[it][ic]) = make_float4(vdy[0], vdy[1], vdy[2], vdy[3]);
        }
#pragma unroll
        for (int i = 0; i < BCT; ++i) {
            const int x = tid + i * NT, bt = x / (NS / 2), r = x % (NS / 2), n = r % (NS / 4) * 4;
            if (x < BCI) {
                f2* to = r < NS / 4 ? &sB[bt][n] : &sC[bt][n];
#pragma unroll
                for (int j = 0; j < 4; ++j) to[j] = pack2(pick(rbc[i], j), pick(rbc[i], j));
            }
        }
        if (tt - K >= t0) fetch(tt - K);
        __syncthreads();
        const int w = wc * kWarpChannels + 2 * c;
        if constexpr (LOCAL) {
#pragma unroll
            for (int t = K - 1; t >= 0; --t) {
                const f2 vd = *reinterpret_cast<const f2*>(&sdt[t][w]), vy = *reinterpret_cast<const f2*>(&sdy[t][w]);
                const f2x2 c0 = *reinterpret_cast<const f2x2*>(&sC[t][n0]), c1 = *reinterpret_cast<const f2x2*>(&sC[t][n0 + 2]);
                const f2 vc[4] = {c0.a, c0.b, c1.a, c1.b};
#pragma unroll
                for (int n = 0; n < 4; ++n) ga[n] = mul2(exp2_pair(mul2(vd, A2[n])), fma2(vy, vc[n], ga[n]));
                const float2 v = unpack2(vd);
                sum.x += v.x;
                sum.y += v.y;
            }
        } else {
            f2 a[K][4], pr[K][4];
#pragma unroll
            for (int t = 0; t < K; ++t) {
                const f2 vd = *reinterpret_cast<const f2*>(&sdt[t][w]), vx = *reinterpret_cast<const f2*>(&sx[t][w]);
                const f2x2 b0 = *reinterpret_cast<const f2x2*>(&sB[t][n0]), b1 = *reinterpret_cast<const f2x2*>(&sB[t][n0 + 2]);
                const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b};
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    a[t][n] = exp2_pair(mul2(vd, A2[n]));
                    pr[t][n] = mul2(a[t][n], h[n]);
                    h[n] = fma2(vx, vb[n], pr[t][n]);
                }
            }
            float yy[4];
#pragma unroll
            for (int t = K - 1; t >= 0; --t) {
                const f2 vd = *reinterpret_cast<const f2*>(&sdt[t][w]), vx = *reinterpret_cast<const f2*>(&sx[t][w]);
                const f2 vy = *reinterpret_cast<const f2*>(&sdy[t][w]);
                const f2x2 b0 = *reinterpret_cast<const f2x2*>(&sB[t][n0]), b1 = *reinterpret_cast<const f2x2*>(&sB[t][n0 + 2]);
                const f2x2 c0 = *reinterpret_cast<const f2x2*>(&sC[t][n0]), c1 = *reinterpret_cast<const f2x2*>(&sC[t][n0 + 2]);
                const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b}, vc[4] = {c0.a, c0.b, c1.a, c1.b};
                const float2 x = unpack2(vx), dy = unpack2(vy);
                f2 r1 = 0, r2 = 0, ry2 = 0;
                float v[8];
#pragma unroll
                for (int n = 0; n < 4; ++n) {
                    const f2 ht = fma2(vx, vb[n], pr[t][n]), gt = fma2(vy, vc[n], ga[n]), gp = mul2(gt, pr[t][n]);
                    const float2 hs = unpack2(ht), gs = unpack2(gt);
                    v[n] = fmaf(gs.y, x.y, gs.x * x.x);
                    v[4 + n] = fmaf(hs.y, dy.y, hs.x * dy.x);
                    r1 = n ? fma2(gt, vb[n], r1) : mul2(gt, vb[n]);
                    r2 = n ? fma2(gp, A2[n], r2) : mul2(gp, A2[n]);
                    ry2 = n ? fma2(ht, vc[n], ry2) : mul2(ht, vc[n]);
                    dA[n] = fma2(gp, vd, dA[n]);
                    ga[n] = mul2(gt, a[t][n]);
                }
                red[warp][t][(lane >> 4) * 16 + 4 * q + (lane >> 2 & 3)] = spread8(v, lane);
                const float2 e1 = unpack2(r1), e2 = unpack2(r2), ey = unpack2(ry2);
                const float r[4] = {e1.x, e1.y, e2.x, e2.y};
                const float got = spread4(r, lane);
                (q & 2 ? s2 : s1)[wb][t][w + (q & 1)] = got;
                yy[(t & 1) * 2] = ey.x;
                yy[(t & 1) * 2 + 1] = ey.y;
                if (!(t & 1)) sy[wb][t + (q >> 1)][w + (q & 1)] = spread4(yy, lane);
            }
        }
        __syncthreads();
        if (!LOCAL) {
            if (live) {
                float odu[4], odt[4], odz[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float e1 = 0.f, e2 = 0.f, ey = 0.f;
#pragma unroll
                    for (int k = 0; k < NB; ++k) { e1 += s1[k][it][ic + i]; e2 += s2[k][it][ic + i]; ey += sy[k][it][ic + i]; }
                    const float uu = pick(u, i);
                    odu[i] = fmaf(e1, vdt[i], skip[i] * vdy[i]);
                    odt[i] = fmaf(e1, uu, e2 * kLn2);
                    if (p.softplus) odt[i] *= sigmoid(pick(raw, i) + bias[i]);
                    sumD[i] = fmaf(vdy[i], uu, sumD[i]);
                    sumb[i] += odt[i];
                    const float zz = pick(z, i), sg = sigmoid(zz);
                    odz[i] = pick(y, i) * fmaf(skip[i], uu, ey) * (sg * fmaf(zz, 1.f - sg, 1.f));
                }
                const size_t at = ((size_t)b * d.T + tt + it) * d.D + col;
                store_pack(static_cast<IO*>(p.du) + at, narrow<IO, 4>(odu), left, p.vec);
                store_pack(static_cast<IO*>(p.ddt) + at, narrow<IO, 4>(odt), left, p.vec);
                if (p.z) store_pack(static_cast<IO*>(p.dz) + at, narrow<IO, 4>(odz), left, p.vec);
            }
            const size_t rows = (size_t)d.B * d.T * d.G * d.N;
            for (int x = tid; x < K * 2 * NS; x += NT) {
                const int t = x / (2 * NS), which = x / NS % 2, n = x % NS;
                if (tt + t >= t1 || n >= d.N) continue;
                float v = 0.f;
#pragma unroll
                for (int k = 0; k < CW; ++k) v += red[n / kWarpStates * CW + k][t][which * 16 + n % kWarpStates];
                p.pBC[((size_t)ct * 2 + which) * rows + (((size_t)b * d.T + tt + t) * d.G + g) * d.N + n] = v;
            }
        }
    }
    if (LOCAL) {
        const size_t at = ((size_t)(seg - 1) * d.B + b) * d.states + tile * kWarpTile + lane * 8;
        f2x2 *e = reinterpret_cast<f2x2*>(p.ends + at), *a = reinterpret_cast<f2x2*>(p.decays + at);
        const f2 v = pack2(sum.x, sum.y);
        e[0] = {ga[0], ga[1]};
        e[1] = {ga[2], ga[3]};
        a[0] = {exp2_pair(mul2(v, A2[0])), exp2_pair(mul2(v, A2[1]))};
        a[1] = {exp2_pair(mul2(v, A2[2])), exp2_pair(mul2(v, A2[3]))};
        return;
    }
    const size_t part = (size_t)seg * d.B + b;
#pragma unroll
    for (int n = 0; n < 4; ++n) {
        if (n0 + n >= d.N) break;
        const float2 v = unpack2(dA[n]), e = unpack2(ga[n]);
        float* to = p.pA + (part * d.D + row) * d.N + n0 + n;
        if (in0) to[0] = v.x;
        if (in1) to[d.N] = v.y;
        if (seg == 0 && p.dh0) {
            float* h = p.dh0 + ((size_t)b * d.D + row) * d.N + n0 + n;
            if (in0) h[0] = e.x;
            if (in1) h[d.N] = e.y;
        }
    }
    // sums over the tokens of a channel: the rows of a chunk in order
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        __syncthreads();
        if (tid < ITEMS)
#pragma unroll
            for (int i = 0; i < 4; ++i) sdt[it][ic + i] = which ? sumb[i] : sumD[i];
        __syncthreads();
        for (int x = tid; x < CC; x += NT) {
            if (ct * CC + x >= d.K) continue;
            float v = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) v += sdt[k][x];
            p.pD[(part * 2 + which) * d.D + (size_t)g * d.K + ct * CC + x] = v;
        }
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
#pragma unroll 4
    for (int k = 0; k < parts; ++k) v += part[(size_t)k * 2 * rows + i];
    st(i < rows ? dB : dC, i < rows ? i : i - rows, v);
}

struct BwdPlan { Dims d; int segs, seglen; size_t saved, ends, pA, pD, pBC, bytes; };
BwdPlan bwd_plan(const qd_scan_shape& s) {
    BwdPlan q{};
    q.d = dims(s);
    q.segs = segments(q.d, kSMs * 2, 4 * kTile);
    q.seglen = segment_tokens(s.T, q.segs);
    q.segs = (int)(((long long)s.T + q.seglen - 1) / q.seglen);
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    q.saved = (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float);
    q.ends = (size_t)(q.segs - 1) * s.B * q.d.states * sizeof(float);
    q.pA = up((size_t)q.segs * s.B * s.D * s.N * sizeof(float));
    q.pD = up((size_t)q.segs * s.B * 2 * s.D * sizeof(float));
    q.pBC = up((size_t)q.d.ctas * 2 * s.B * s.T * s.G * s.N * sizeof(float));
    const size_t fwd = scan_fwd_workspace(s, true);
    q.bytes = q.saved + 2 * q.ends + q.pA + q.pD + q.pBC;
    if (q.bytes < fwd) q.bytes = fwd;
    return q;
}

template <typename IO, int NB>
cudaError_t launch(const P& p, cudaStream_t stream) {
    constexpr int NT = NB == 1 ? 128 : 64 * NB;
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    if (p.segs > 1) {
        cudaError_t e = launch_overlapped(k_scan_bwd<IO, NB, true>, dim3((unsigned)(per * (p.segs - 1))), dim3(NT), 0, stream, p);
        if (e != cudaSuccess) return e;
        e = join(p.ends, p.decays, p.segs - 1, p.segs - 2, -1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(k_scan_bwd<IO, NB, false>, dim3((unsigned)(per * p.segs)), dim3(NT), 0, stream, p);
}
template <typename IO>
cudaError_t launch(const P& p, const ScanArgs& a) {
    cudaError_t e = p.d.nb == 1   ? launch<IO, 1>(p, a.stream)
                    : p.d.nb == 2 ? launch<IO, 2>(p, a.stream)
                    : p.d.nb == 3 ? launch<IO, 3>(p, a.stream)
                                  : launch<IO, 4>(p, a.stream);
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
    p.d = q.d; p.segs = q.segs; p.seglen = q.seglen;
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
    cudaError_t e = a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a) : launch<float>(p, a);
    if (e != cudaSuccess) return e;
    const long long D = a.s.D, DN = D * a.s.N;
    const int parts = q.segs * a.s.B;
    e = sum_parts(p.pA, parts, DN, DN, DN, 1, a.dA, nullptr, a.stream);
    if (e != cudaSuccess || (!a.dD && !a.ddt_bias)) return e;
    return sum_parts(p.pD, parts, 2 * D, D, D, 1, a.dD, a.ddt_bias, a.stream);
}

}  // namespace qd

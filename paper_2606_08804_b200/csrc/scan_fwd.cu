// Forward of the selective scan (scan.cuh).  Per token, channel and state: one exponential and the products dt A, dt u B, a h + ., <C, h>.
// The special function unit gives 4 exponentials per clock and sub-partition, so a warp's 16 x 16 states need 64 clocks of it and 32 of the
// fp32 pipe: bound by the exponentials, not by HBM, when there are warps enough.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

template <typename IO, int NB, bool LOCAL>
__global__ void __launch_bounds__(NB == 1 ? 128 : 64 * NB) k_scan_fwd(const P p) {
    constexpr int CW = NB == 1 ? 4 : 2, NT = 32 * CW * NB, CC = CW * kWarpChannels, NS = NB * kWarpStates;
    constexpr int ITEMS = kTile * CC / 8;                  // groups of eight channels of a tile: a thread has one or none
    constexpr int BCI = kTile * 2 * (NS / 4), BCT = (BCI + NT - 1) / NT;      // groups of four states of B and C
    static_assert(ITEMS <= NT, "a thread has one group of channels");
    __shared__ __align__(16) float sdt[kTile][CC], sx[kTile][CC];          // dt, dt u
    __shared__ __align__(16) f2 sB[kTile][NS], sC[kTile][NS];              // each twice, for both channels of a pair
    __shared__ float sy[NB][kTile][CC];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, c = lane >> 2;
    const int wc = warp % CW, wb = warp / CW;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int seg = idx % p.segs, b = idx / p.segs;        // LOCAL: the last segment is not launched
    const int t0 = seg * p.seglen, t1 = min(d.T, t0 + p.seglen);
    const int ch = ct * CC + wc * kWarpChannels + 2 * c;   // in the group
    const int n0 = wb * kWarpStates + 4 * q;
    const size_t tile = (((size_t)g * d.ctas + ct) * CW + wc) * NB + wb;   // in warp order

    f2 A2[4], h[4];
    float2 sum = {0.f, 0.f};                               // of dt
    {
        const size_t row = (size_t)g * d.K + ch;
        const bool in0 = ch < d.K, in1 = ch + 1 < d.K;
        const float* prev = !LOCAL && seg ? p.ends + ((size_t)(seg - 1) * d.B + b) * d.states + tile * kWarpTile + lane * 8 : nullptr;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            const bool in = n0 + n < d.N;
            A2[n] = pack2(in && in0 ? p.A[row * d.N + n0 + n] * kLog2e : 0.f, in && in1 ? p.A[(row + 1) * d.N + n0 + n] * kLog2e : 0.f);
            if (prev) h[n] = pack2(prev[2 * n], prev[2 * n + 1]);
            else if (seg == 0 && p.h0) {
                const float* s = p.h0 + ((size_t)b * d.D + row) * d.N + n0 + n;
                h[n] = pack2(in && in0 ? s[0] : 0.f, in && in1 ? s[d.N] : 0.f);
            } else h[n] = 0;
        }
    }
    // this thread's group of eight channels of a tile's tokens
    const int it = tid / (CC / 8), ic = tid % (CC / 8) * 8;
    const int left = tid < ITEMS ? d.K - ct * CC - ic : 0;
    const size_t col = (size_t)g * d.K + ct * CC + ic;
    Pack<IO, 8> ru = zero_pack<IO, 8>(), rdt = ru, rz = ru;
    Pack<IO, 4> rbc[BCT];
    float bias[8], skip[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        bias[i] = p.dt_bias && i < left ? p.dt_bias[col + i] : 0.f;
        skip[i] = !LOCAL && p.D && i < left ? p.D[col + i] : 0.f;
    }
    auto fetch = [&](int tt) {
        const int t = tt + it;
        if (left > 0 && t < t1) {
            const size_t at = ((size_t)b * d.T + t) * d.D + col;
            ru = load_pack<IO, 8>(static_cast<const IO*>(p.u) + at, left, p.vec);
            rdt = load_pack<IO, 8>(static_cast<const IO*>(p.dt) + at, left, p.vec);
            if (!LOCAL && p.z) rz = load_pack<IO, 8>(static_cast<const IO*>(p.z) + at, left, p.vec);
        }
#pragma unroll
        for (int i = 0; i < BCT; ++i) {
            const int x = tid + i * NT, bt = x / (NS / 2), r = x % (NS / 2), n = r % (NS / 4) * 4;
            const IO* src = static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm);
            rbc[i] = zero_pack<IO, 4>();
            if (x < BCI && tt + bt < t1 && n < d.N && !(LOCAL && r >= NS / 4))
                rbc[i] = load_pack<IO, 4>(src + (((size_t)b * d.T + tt + bt) * d.G + g) * d.N + n, d.N - n, p.vecn);
        }
    };
    fetch(t0);
    for (int tt = t0; tt < t1; tt += kTile) {
        const Pack<IO, 8> u = ru, z = rz;
        if (tid < ITEMS) {
            const bool live = tt + it < t1;
            float fd[8], fx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float raw = pick(rdt, i) + bias[i];
                fd[i] = live && i < left ? (p.softplus ? softplus(raw) : raw) : 0.f;
                fx[i] = live && i < left ? fd[i] * pick(u, i) : 0.f;
            }
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<float4*>(&sdt[it][ic + i]) = make_float4(fd[i], fd[i + 1], fd[i + 2], fd[i + 3]);
                *reinterpret_cast<float4*>(&sx[it][ic + i]) = make_float4(fx[i], fx[i + 1], fx[i + 2], fx[i + 3]);
            }
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
        if (tt + kTile < t1) fetch(tt + kTile);
        __syncthreads();
#pragma unroll 2
        for (int t = 0; t < kTile; t += 2) {
            if (!LOCAL && p.saved && t % kSave == 0 && tt + t < t1) {
                f2x2* to = reinterpret_cast<f2x2*>(p.saved + ((size_t)b * ((d.T + kSave - 1) / kSave) + (tt + t) / kSave) * d.states + tile * kWarpTile + lane * 8);
                to[0] = {h[0], h[1]};
                to[1] = {h[2], h[3]};
            }
            f2 y[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int w = wc * kWarpChannels + 2 * c;
                const f2 vd = *reinterpret_cast<const f2*>(&sdt[t + s][w]), vx = *reinterpret_cast<const f2*>(&sx[t + s][w]);
                const f2x2 b0 = *reinterpret_cast<const f2x2*>(&sB[t + s][n0]), b1 = *reinterpret_cast<const f2x2*>(&sB[t + s][n0 + 2]);
                const f2 vb[4] = {b0.a, b0.b, b1.a, b1.b};
#pragma unroll
                for (int n = 0; n < 4; ++n) h[n] = fma2(exp2_pair(mul2(vd, A2[n])), h[n], mul2(vx, vb[n]));
                if (LOCAL) {
                    const float2 v = unpack2(vd);
                    sum.x += v.x;
                    sum.y += v.y;
                } else {
                    const f2x2 c0 = *reinterpret_cast<const f2x2*>(&sC[t + s][n0]), c1 = *reinterpret_cast<const f2x2*>(&sC[t + s][n0 + 2]);
                    y[s] = fma2(h[3], c1.b, fma2(h[2], c1.a, fma2(h[1], c0.b, mul2(h[0], c0.a))));
                }
            }
            if (!LOCAL) {
                // two tokens of two channels over four lanes: lane q ends with token q / 2, channel q % 2
                const float2 y0 = unpack2(y[0]), y1 = unpack2(y[1]);
                const bool hi = q & 2, odd = q & 1;
                float k0 = hi ? y1.x : y0.x, k1 = hi ? y1.y : y0.y;
                k0 += __shfl_xor_sync(0xffffffffu, hi ? y0.x : y1.x, 2);
                k1 += __shfl_xor_sync(0xffffffffu, hi ? y0.y : y1.y, 2);
                const float k = (odd ? k1 : k0) + __shfl_xor_sync(0xffffffffu, odd ? k0 : k1, 1);
                sy[wb][t + (q >> 1)][wc * kWarpChannels + 2 * c + (q & 1)] = k;
            }
        }
        __syncthreads();
        if (!LOCAL && p.y && left > 0 && tt + it < t1) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float s = sy[0][it][ic + i];
#pragma unroll
                for (int k = 1; k < NB; ++k) s += sy[k][it][ic + i];
                s = fmaf(skip[i], pick(u, i), s);
                const float zz = pick(z, i);
                o[i] = p.z ? s * (zz * sigmoid(zz)) : s;
            }
            store_pack(static_cast<IO*>(p.y) + ((size_t)b * d.T + tt + it) * d.D + col, narrow<IO, 8>(o), left, p.vec);
        }
    }
    if (LOCAL) {
        const size_t at = ((size_t)seg * d.B + b) * d.states + tile * kWarpTile + lane * 8;
        f2x2 *e = reinterpret_cast<f2x2*>(p.ends + at), *a = reinterpret_cast<f2x2*>(p.decays + at);
        const f2 v = pack2(sum.x, sum.y);
        e[0] = {h[0], h[1]};
        e[1] = {h[2], h[3]};
        a[0] = {exp2_pair(mul2(v, A2[0])), exp2_pair(mul2(v, A2[1]))};
        a[1] = {exp2_pair(mul2(v, A2[2])), exp2_pair(mul2(v, A2[3]))};
    } else if (p.hT && t1 == d.T) {
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            if (n0 + n >= d.N) break;
            const float2 v = unpack2(h[n]);
            float* to = p.hT + ((size_t)b * d.D + (size_t)g * d.K + ch) * d.N + n0 + n;
            if (ch < d.K) to[0] = v.x;
            if (ch + 1 < d.K) to[d.N] = v.y;
        }
    }
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
    for (int k = 1; k < n; ++k) {
        const size_t at = (size_t)(from + k * step) * count + i;
        h = fmaf(decays[at], h, ends[at]);
        ends[at] = h;
    }
}
}  // namespace

// True states at the ends of `n` segments from those of each walked alone, which they overwrite; the segments are from, from + step, ..
cudaError_t join(float* ends, const float* decays, int n, int from, int step, size_t count, cudaStream_t stream) {
    if (n <= 1) return cudaSuccess;
    return launch_overlapped(k_join, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, stream, ends, decays, n, from, step, count);
}

// Segments of a sequence: as many as fill the GPU's `slots` CTAs, none where the channels do, each of `shortest` tokens at least.
int segments(const Dims& d, int slots, int shortest) {
    const long long units = (long long)d.B * d.G * d.ctas;
    if (units * 2 > slots) return 1;
    long long n = slots / units;
    const long long most = d.T / shortest;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}
int segment_tokens(int T, int segs) {
    const long long per = ((long long)T + segs - 1) / segs;
    return (int)((per + kTile - 1) / kTile * kTile);
}
}  // namespace scan

namespace {
struct FwdPlan { Dims d; int segs, seglen; size_t saved, ends, bytes; };
FwdPlan fwd_plan(const qd_scan_shape& s, bool save) {
    FwdPlan q{};
    q.d = dims(s);
    q.segs = segments(q.d, kSMs * 4 / q.d.nb, 4 * kTile);
    q.seglen = segment_tokens(s.T, q.segs);
    q.segs = (int)(((long long)s.T + q.seglen - 1) / q.seglen);
    q.saved = save ? (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float) : 0;
    q.ends = (size_t)(q.segs - 1) * s.B * q.d.states * sizeof(float);
    q.bytes = q.saved + 2 * q.ends;
    return q;
}

template <typename IO, int NB>
cudaError_t launch(P p, cudaStream_t stream) {
    constexpr int NT = NB == 1 ? 128 : 64 * NB;
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    if (p.segs > 1) {
        P l = p;
        l.segs = p.segs - 1;
        cudaError_t e = launch_overlapped(k_scan_fwd<IO, NB, true>, dim3((unsigned)(per * l.segs)), dim3(NT), 0, stream, l);
        if (e != cudaSuccess) return e;
        e = join(p.ends, p.decays, l.segs, 0, 1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(k_scan_fwd<IO, NB, false>, dim3((unsigned)(per * p.segs)), dim3(NT), 0, stream, p);
}
template <typename IO>
cudaError_t launch(const P& p, cudaStream_t stream) {
    switch (p.d.nb) {
        case 1: return launch<IO, 1>(p, stream);
        case 2: return launch<IO, 2>(p, stream);
        case 3: return launch<IO, 3>(p, stream);
        default: return launch<IO, 4>(p, stream);
    }
}
}  // namespace

size_t scan_fwd_workspace(const qd_scan_shape& s, bool save) { return fwd_plan(s, save).bytes; }

cudaError_t scan_fwd(const ScanArgs& a) {
    const FwdPlan q = fwd_plan(a.s, a.save);
    P p{};
    p.d = q.d; p.segs = q.segs; p.seglen = q.seglen;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.D = a.D; p.dt_bias = a.dt_bias; p.h0 = a.h0;
    p.y = a.y; p.hT = a.hT;
    p.saved = a.save ? reinterpret_cast<float*>(a.ws) : nullptr;
    p.ends = reinterpret_cast<float*>(a.ws + q.saved);
    p.decays = reinterpret_cast<float*>(a.ws + q.saved + q.ends);
    p.softplus = a.softplus; p.vec = q.d.K % 8 == 0; p.vecn = a.s.N % 4 == 0;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.stream) : launch<float>(p, a.stream);
}

}  // namespace qd

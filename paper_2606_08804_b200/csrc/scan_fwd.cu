// Forward of the selective scan (scan.cuh).  Per token, channel and state: one exponential and the products dt A, dt u B, a h + ., <C, h>.
// The special function unit gives 4 exponentials per clock and sub-partition, so a warp's 16 x 16 states need 64 clocks of it and 32 of the
// fp32 pipe, softplus and gate another 16.  8 x 2048 tokens of 2048 bf16 channels, 16 states: 256 us when it saves for a backward (237
// without) against 144 of that unit and 40 of HBM; fp32 275 (258).  With two walking and two preparing warps a sub-partition nothing is full:
// on the SMs that have two CTAs the special function unit 65 %, shared memory and shuffles 74 %, issue slots 49 %.  Not faster, measured when
// these took 257 (the walk alone then took 189, preparing alone 170): eight preparing warps, copies further ahead, part of the exponentials
// as polynomials on the fp32 pipe (271).
#include "scan.cuh"

#include <algorithm>

namespace qd {
namespace {
using namespace scan;

template <typename IO, int NB> struct FwdSmem {
    static constexpr int CC = kWalkers / NB * kWarpChannels, NS = NB * kWarpStates;
    static constexpr int PAIRS = CC / 2, ROWS = 128 / PAIRS, PASSES = kTile / ROWS;      // of a thread that prepares: a pair of channels, PASSES tokens
    static constexpr int RING = sizeof(IO) == 2 ? 5 : 4;   // tiles of what is copied: i - 1 (for y), i, i + 1 (prepared now), i + 2 (has come), fp32 no more
    float4 step[2][kTile][2][PAIRS];                       // dt, dt, dt u, dt u of a pair of channels, in both orders
    float4 B[2][kTile][NS / 4], C[2][kTile][NS / 4];       // four states
    alignas(16) float y[2][NB][kTile][CC];
    // rings, each behind the one before (TileRun)
    alignas(16) IO u[RING][kTile * CC], dt[RING][kTile * CC], z[RING][kTile * CC];
    Pack<IO, 4> bc[RING][NB][128];
};

// SAVE: for a backward.
template <typename IO, int NB, bool LOCAL, bool SAVE>
__global__ void __launch_bounds__(kThreads, 2) k_scan_fwd(const P p) {
    using S = FwdSmem<IO, NB>;
    constexpr int CW = kWalkers / NB, CC = S::CC, NS = S::NS;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    S& sm = *reinterpret_cast<S*>(raw_smem);
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int warp = sm100::warp_index(), lane = threadIdx.x & 31;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int b = idx % d.B, seg = (LOCAL ? p.segs - 2 : p.segs - 1) - idx / d.B;       // LOCAL: without the last; the first, which may be short, last
    const int t0 = seg ? p.first + (seg - 1) * p.seglen : 0, t1 = min(d.T, p.first + seg * p.seglen), n = (t1 - t0 + kTile - 1) / kTile;

    if (warp < kWalkers) {
        // ---- walk ----------------------------------------------------------------------------------------------------------
        const Map m(lane, false);
        const int wc = warp % CW, wb = warp / CW, n0 = wb * kWarpStates, ch = ct * CC + wc * kWarpChannels;
        const size_t mine = (((size_t)g * d.ctas + ct) * kWalkers + warp) * kWarpTile + lane * 8, state = (size_t)b * d.D * d.N;
        f2 A2[4], h[4] = {0, 0, 0, 0};
        float sum[2] = {0.f, 0.f};
        load_A(p, m, g, ch, n0, A2);
        if (seg == 0) {
            if (p.h0) load_state(p, m, p.h0 + state, g, ch, n0, 1.f, h);
        } else if (!LOCAL) load_end(p, 0, 1, seg, b, mine, h);
        float* saved = SAVE ? p.saved + ((size_t)b * ((d.T + kSave - 1) / kSave) + t0 / kSave) * d.states + mine : nullptr;
        const int pair = wc * (kWarpChannels / 2) + (lane >> 2), quad = n0 / 4 + m.q;
        __syncthreads();
        for (int i = 0; i < n; ++i) {
            const int k = i & 1;
            const float4 *step = &sm.step[k][0][m.order][pair], *B = &sm.B[k][0][quad], *C = &sm.C[k][0][quad];
            float out[kTile / 2], held[2];                 // stored when the tile is done: nothing stands in the way of the loads till then
#pragma unroll
            for (int t = 0; t < kTile; ++t) {
                if (SAVE && !LOCAL && t % kSave == 0 && t0 + i * kTile + t < t1) {
                    store_tile(saved, h);
                    saved += d.states;
                }
                const float4 v = step[t * 2 * S::PAIRS], vb = B[t * (NS / 4)];
                const f2 dt[2] = {both(v.x), both(v.y)}, x[2] = {both(v.z), both(v.w)}, bp[2] = {pack2(vb.x, vb.y), pack2(vb.z, vb.w)};
#pragma unroll
                for (int j = 0; j < 4; ++j) h[j] = fma2(decay(dt[j >> 1], A2[j]), h[j], mul2(x[j >> 1], bp[j & 1]));
                if (LOCAL) {
                    sum[0] += v.x;
                    sum[1] += v.y;
                } else {
                    const float4 vc = C[t * (NS / 4)];
                    const f2 cp[2] = {pack2(vc.x, vc.y), pack2(vc.z, vc.w)};
                    const float y0 = sum_pair(fma2(h[1], cp[1], mul2(h[0], cp[0]))), y1 = sum_pair(fma2(h[3], cp[1], mul2(h[2], cp[0])));
                    // over the four lanes: a lane keeps its first channel, then of two tokens that of its q / 2
                    held[t & 1] = y0 + __shfl_xor_sync(0xffffffffu, y1, 1);
                    if (t & 1) {
                        const bool second = m.q & 2;
                        out[t / 2] = (second ? held[1] : held[0]) + __shfl_xor_sync(0xffffffffu, second ? held[0] : held[1], 2);
                    }
                }
            }
            if (!LOCAL)
#pragma unroll
                for (int t = 0; t < kTile; t += 2) sm.y[k][wb][t + (m.q >> 1)][wc * kWarpChannels + m.ch[0]] = out[t / 2];
            __syncthreads();
        }
        if (LOCAL) store_end(p, seg, b, mine, h, A2, sum);
        else if (p.hT && t1 == d.T) store_state(p, m, p.hT + state, g, ch, n0, h);
        return;
    }
    // ---- prepare tiles, write y ------------------------------------------------------------------------------------------------
    const int tid = threadIdx.x - 32 * kWalkers;
    const size_t rows = (size_t)b * d.T, col = (size_t)g * d.K + ct * CC;
    const int left = d.K - ct * CC;
    // a tile is prepared by pairs of channels and written out by groups of eight (where NB > 1 some threads have none)
    const int pr = tid % S::PAIRS, first = tid / S::PAIRS, it = tid / (CC / 8), ic = tid % (CC / 8) * 8;
    float bias[2], skip[8];
#pragma unroll
    for (int e = 0; e < 2; ++e) bias[e] = p.dt_bias && 2 * pr + e < left ? p.dt_bias[col + 2 * pr + e] : 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) skip[e] = !LOCAL && p.D && ic + e < left ? p.D[col + ic + e] : 0.f;
    TileRun<kTile, CC, S::RING, IO, 3> run(&sm.u[0][0], {p.u, p.dt, LOCAL ? nullptr : p.z}, rows + t0, d.D, col, left, kTile, tid);
    StateRun<NS, IO> states(p, rows + t0, g, true, !LOCAL, kTile, tid);
    auto fetch = [&](int i) {
        if (i < n) {
            const int tt = t0 + i * kTile, slot = i % S::RING;
            const bool whole = tt + kTile <= t1;
            if (whole && p.rows == kWhole) run.copy(slot, d.D);
            else copy_tiles<kTile, CC, IO, 3>({sm.u[slot], sm.dt[slot], sm.z[slot]}, {p.u, p.dt, LOCAL ? nullptr : p.z}, rows, d.D, tt, t1, col, left, p.rows, tid);
            if (whole && p.bc == kWhole) states.template copy<kTile>(sm.bc[slot], tid);
            else
#pragma unroll
            for (int j = 0; j < NB; ++j) {                                 // four states of B or C of a token, which this thread prepares too
                const int x = tid + j * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
                const int have = tt + bt < t1 && !(LOCAL && r >= NS / 4) ? d.N - s : 0;
                copy_group<4>(reinterpret_cast<IO*>(&sm.bc[slot][j][tid]),
                              static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm) + (have > 0 ? ((rows + tt + bt) * d.G + g) * d.N + s : 0), have, p.bc);
            }
        }
        run.move();
        states.move();
        copy_commit();
    };
    // Channels past the last have u = 0 and any step; tokens past the last a step of 0.
    auto turn = [&](int i) {
        const int k = i & 1, slot = i % S::RING;
#pragma unroll
        for (int r = 0; r < S::PASSES; ++r) {
            const int row = first + r * S::ROWS;
            const Pack<IO, 2> dt = load_pack<IO, 2>(&sm.dt[slot][row * CC + 2 * pr], 2, true), u = load_pack<IO, 2>(&sm.u[slot][row * CC + 2 * pr], 2, true);
            float2 v = make_float2(pick(dt, 0) + bias[0], pick(dt, 1) + bias[1]);
            if (p.softplus) v = softplus(v.x, v.y);
            if (t0 + i * kTile + row >= t1) v.x = v.y = 0.f;
            const float x0 = v.x * pick(u, 0), x1 = v.y * pick(u, 1);
            sm.step[k][row][0][pr] = make_float4(v.x, v.y, x0, x1);
            sm.step[k][row][1][pr] = make_float4(v.y, v.x, x1, x0);
        }
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int x = tid + j * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4);
            const Pack<IO, 4> v = sm.bc[slot][j][tid];
            (r < NS / 4 ? sm.B[k][bt] : sm.C[k][bt])[s] = make_float4(pick(v, 0), pick(v, 1), pick(v, 2), pick(v, 3));
        }
    };
    auto finish = [&](int i) {
        const int t = t0 + i * kTile + it, k = i & 1, slot = i % S::RING;
        if (!p.y || it >= kTile || ic >= left || t >= t1) return;
        const Pack<IO, 8> u = load_pack<IO, 8>(&sm.u[slot][it * CC + ic], 8, true), z = load_pack<IO, 8>(&sm.z[slot][it * CC + ic], 8, true);
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NB; ++w)
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float4 v = *reinterpret_cast<const float4*>(&sm.y[k][w][it][ic + e]);
                o[e] += v.x; o[e + 1] += v.y; o[e + 2] += v.z; o[e + 3] += v.w;
            }
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            f2 v = pack2(o[e], o[e + 1]);
            if (p.D) v = fma2(pack2(skip[e], skip[e + 1]), pack2(pick(u, e), pick(u, e + 1)), v);
            if (p.z) {
                const f2 zz = pack2(pick(z, e), pick(z, e + 1));
                const float2 den = unpack2(add2(exp2_pair(mul2(zz, both(-kLog2e))), both(1.f)));
                v = mul2(v, mul2(zz, pack2(reciprocal(den.x), reciprocal(den.y))));
            }
            const float2 r = unpack2(v);
            o[e] = r.x;
            o[e + 1] = r.y;
        }
        store_pack(static_cast<IO*>(p.y) + (rows + t) * d.D + col + ic, narrow<IO, 8>(o), left - ic, p.rows == kWhole && left - ic >= 8 && (d.K * sizeof(IO)) % 16 == 0);
    };
#pragma unroll
    for (int i = 0; i < S::RING - 2; ++i) fetch(i);
    copy_wait<S::RING - 4>();                                              // tiles 0 and 1
    prepare_barrier();
    turn(0);
    __syncthreads();
    for (int i = 0; i < n; ++i) {
        if (!LOCAL && i > 0) finish(i - 1);
        fetch(i + S::RING - 2);                                            // where a tile stood that was finished before the last barrier
        if (i + 1 < n) turn(i + 1);
        copy_wait<S::RING - 4>();                                          // tile i + 2, for all after the barrier
        __syncthreads();
    }
    if (!LOCAL) finish(n - 1);
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
        h = joined(decays[at], h, ends[at]);
        ends[at] = h;
    }
}
}  // namespace

// The segments are from, from + step, ..
cudaError_t join(float* ends, const float* decays, int n, int from, int step, size_t count, cudaStream_t stream) {
    return launch_overlapped(k_join, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, stream, ends, decays, n, from, step, count);
}

// What a walk of a token costs, in ns: without outputs and with them, by a CTA that has an SM for itself and by one of two (4096 x 16
// channels of 16 states and of twice as many).
struct Cost { int end_alone, end_paired, alone, paired; };
constexpr Cost kForward{54, 85, 78, 128}, kBackward{88, 118, 228, 358};

Cut cut(const Dims& d, bool backward) {
    const Cost& w = backward ? kBackward : kForward;
    const long long units = (long long)d.B * d.G * d.ctas;
    auto waves = [](long long ctas, int alone, int paired) {
        const long long rest = ctas % (2 * kSMs);
        return ctas / (2 * kSMs) * paired + (rest == 0 ? 0 : rest <= kSMs ? alone : paired);
    };
    auto tiles = [](long long tokens) { return (int)((tokens + kTile - 1) / kTile * kTile); };
    Cut c{1, tiles(d.T), tiles(d.T)};
    long long least = waves(units, w.alone, w.paired) * (d.T + kBegin);
    for (int k = 1; k <= 2 * kMostWaves; ++k) {            // of those that need as many waves of CTAs the largest number is the best
        const long long n = std::min<long long>(k * kSMs / units, d.T / (2 * kTile));
        if (n < 2) continue;
        Cut x{0, 0, tiles((d.T + n - 1) / n)};
        x.first = x.len;
        x.segs = (d.T + x.len - 1) / x.len;
        const long long time = (waves(units * (x.segs - 1), w.end_alone, w.end_paired) + waves(units * x.segs, w.alone, w.paired)) * (x.len + kBegin) + kLaunch;
        if (time < least) {
            least = time;
            c = x;
        }
    }
    if (units > kSMs && units < 2 * kSMs) {                // turns: short segments that a place left over takes; many of them even out
        const long long places = 2 * kSMs, free = places - units, turns = (units + free - 1) / free;
        const int shorter = (int)(turns > 3 ? d.T * free / places : d.T / (turns + 1)) / kTile * kTile, longer = tiles(d.T - shorter);
        const long long time = w.end_paired * (shorter + kBegin) + w.paired * (longer + kBegin) + kLaunch;
        if (shorter >= 2 * kTile && time * 13 < least * 12) c = backward ? Cut{2, longer, longer} : Cut{2, shorter, longer};
    }
    return c;
}
}  // namespace scan

namespace {
struct FwdPlan { Dims d; Cut c; size_t saved, ends, bytes; };
FwdPlan fwd_plan(const qd_scan_shape& s, bool save) {
    FwdPlan q{};
    q.d = dims(s);
    q.c = cut(q.d, false);
    q.saved = save ? (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float) : 0;
    q.ends = (size_t)(q.c.segs - 1) * s.B * q.d.states * sizeof(float);
    q.bytes = q.saved + 2 * q.ends;
    return q;
}

template <typename IO, int NB, bool SAVE>
cudaError_t launch(const P& p, cudaStream_t stream) {
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    constexpr size_t smem = sizeof(FwdSmem<IO, NB>);
    constexpr size_t most = smem > kAloneSmem ? smem : kAloneSmem;
    const auto local = k_scan_fwd<IO, NB, true, SAVE>, all = k_scan_fwd<IO, NB, false, SAVE>;
    cudaError_t e;
    if (p.segs > 1) {
        e = set_max_smem_once((const void*)local, most);
        if (e == cudaSuccess) e = launch_overlapped(local, dim3((unsigned)(per * (p.segs - 1))), dim3(kThreads), per * (p.segs - 1) > kSMs ? smem : most, stream, p);
        if (e == cudaSuccess && p.joined) e = join(p.ends, p.decays, p.segs - 1, 0, 1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    e = set_max_smem_once((const void*)all, most);
    return e != cudaSuccess ? e : launch_overlapped(all, dim3((unsigned)(per * p.segs)), dim3(kThreads), per * p.segs > kSMs ? smem : most, stream, p);
}
template <typename IO, int NB>
cudaError_t launch(const P& p, cudaStream_t stream) {
    return p.saved ? launch<IO, NB, true>(p, stream) : launch<IO, NB, false>(p, stream);
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
    p.d = q.d; p.segs = q.c.segs; p.first = q.c.first; p.seglen = q.c.len;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.D = a.D; p.dt_bias = a.dt_bias; p.h0 = a.h0;
    p.y = a.y; p.hT = a.hT;
    p.saved = a.save ? reinterpret_cast<float*>(a.ws) : nullptr;
    p.ends = reinterpret_cast<float*>(a.ws + q.saved);
    p.decays = reinterpret_cast<float*>(a.ws + q.saved + q.ends);
    p.softplus = a.softplus; p.rows = copy_of(q.d.K, a.s.dtype == QD_BF16 ? 8 : 4, a.s.dtype); p.bc = copy_of(a.s.N, 4, a.s.dtype);
    p.joined = p.segs - 1 > kMostJoined;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.stream) : launch<float>(p, a.stream);
}

}  // namespace qd

// Backward of the selective scan (scan.cuh).  With g_t = dL/dh_t = dy_t C_t + a_{t+1} g_{t+1} (dy after the factor of z) and p_t = a_t h_{t-1}:
//   dC_t = sum_channels dy_t h_t        dB_t = sum_channels dt_t u_t g_t        du = dt <g, B> + D dy
//   ddt = u <g, B> + <g p, A>           dA = sum_t dt g p                       dh0 = a_1 g_1,   dz = dy y_raw SiLU'(z).
// The forward saved the state before every kSave-th token; from the last such tile to the first the states of its tokens are walked anew,
// a_t and h_{t-1} kept in registers, and then g is walked back, (a g) h_{t-1} being g p.  The registers hold half a tile; the first half is
// walked once more ahead, to the state in the middle (a state saved every fourth token would be 134 MB more for each 8192 x 2048 x 16).
// Per token, channel and state 1.5 exponentials and 13 operations of the fp32 pipe, 190 instructions a token and warp, a third of them
// preparing: 8 x 2048 tokens of 2048 bf16 channels, 16 states, take 646 us with the sums (fp32 800), where two CTAs to an SM issue in 64 % of
// the clocks, the special function unit is busy in 39 % and shared memory in 62; what is left are the latencies of a chain of shuffles and
// products, and registers leave no room for a third.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

constexpr unsigned kAll = 0xffffffffu;
constexpr int kWalkRegs = 152, kPrepareRegs = 104;         // of 2 x 128: what the launch gives a pair of threads, one of each half of the CTA
constexpr int kHalf = kSave / 2;             // tokens whose a_t, h_{t-1} are in registers at a time

template <typename IO, int NB> struct BwdSmem {
    static constexpr int CC = kWalkers / NB * kWarpChannels, NS = NB * kWarpStates;
    static constexpr int PAIRS = CC / 2, ROWS = 128 / PAIRS, PASSES = ROWS < kSave ? kSave / ROWS : 1;     // who prepares: a pair of channels, PASSES tokens
    static constexpr int RING = sizeof(IO) == 2 ? 5 : 4;   // tiles of what is copied: the one walked before, this, the next two, bf16 one more
    static constexpr int SAVED = 4;
    static constexpr int BC = kSave * 2 * NS / 4, BCT = (BC + 127) / 128;         // groups of four states of B and C of a tile; of a thread
    float4 step[2][kSave][2][PAIRS];                       // dt, dt, dt u, dt u of a pair of channels, in both orders
    float4 dy[2][kSave][PAIRS];                            // dy of a pair of channels in both orders
    float4 B[2][kSave][2][NS / 4], C[2][kSave][2][NS / 4]; // four states, the pairs in both orders
    alignas(16) float gB[2][NB][kSave][CC], gpA[2][NB][kSave][CC], y[2][NB][kSave][CC];
    alignas(16) float bc[2][kWalkers][kSave][32];          // dB, dC summed over a warp's channels
    f2x2 saved[SAVED][2][128];                             // of a thread that walks
    // rings, each behind the one before (TileRun)
    alignas(16) IO u[RING][kSave * CC], dt[RING][kSave * CC], z[RING][kSave * CC], gy[RING][kSave * CC];
    Pack<IO, 4> rbc[RING][BCT][128];
};

template <typename IO, int NB, bool LOCAL>
__global__ void __launch_bounds__(kThreads, 2) k_scan_bwd(const P p) {
    using S = BwdSmem<IO, NB>;
    constexpr int CW = kWalkers / NB, CC = S::CC, NS = S::NS, K = kSave, H = kHalf;
    extern __shared__ __align__(16) unsigned char raw_smem[];
    S& sm = *reinterpret_cast<S*>(raw_smem);
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const Dims& d = p.d;
    const int warp = sm100::warp_index(), lane = threadIdx.x & 31;
    int idx = blockIdx.x;
    const int ct = idx % d.ctas; idx /= d.ctas;
    const int g = idx % d.G; idx /= d.G;
    const int b = idx % d.B, seg = idx / d.B + (LOCAL ? 1 : 0);            // LOCAL: without the first; the last may be short
    const int t0 = seg ? p.first + (seg - 1) * p.seglen : 0, t1 = min(d.T, p.first + seg * p.seglen), n = (t1 - t0 + K - 1) / K;
    const size_t part = (size_t)seg * d.B + b;

    if (warp < kWalkers) {
        // ---- walk, from the last tile to the first ----------------------------------------------------------------------------
        if constexpr (!LOCAL) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kWalkRegs));
        const Map m(lane, true);
        const int wc = warp % CW, wb = warp / CW, n0 = wb * kWarpStates, ch = ct * CC + wc * kWarpChannels;
        const size_t mine = (((size_t)g * d.ctas + ct) * kWalkers + warp) * kWarpTile + lane * 8, state = (size_t)b * d.D * d.N;
        f2 A2[4], ga[4] = {0, 0, 0, 0}, dA[4] = {0, 0, 0, 0};              // ga = a_{t+1} g_{t+1}
        float sum[2] = {0.f, 0.f};
        load_A(p, m, g, ch, n0, A2);
        if (seg == p.segs - 1) {
            if (p.dhT) load_state(p, m, p.dhT + state, g, ch, n0, 1.f, ga);
        } else if (!LOCAL) load_end(p, p.segs - 2, -1, p.segs - 1 - seg, b, mine, ga);
        const float* saved = LOCAL ? nullptr : p.saved + ((size_t)b * ((d.T + K - 1) / K) + t0 / K) * d.states + mine;
        auto fetch = [&](int i) {                          // the state before tile i, three tiles ahead
            if (i >= 0)
#pragma unroll
                for (int e = 0; e < 2; ++e) copy_bytes<16>(&sm.saved[i % S::SAVED][e][threadIdx.x], saved + (size_t)i * d.states + 4 * e, 16);
            copy_commit();
        };
        if (!LOCAL)
#pragma unroll
            for (int e = 1; e < S::SAVED; ++e) fetch(n - e);
        const int pair = wc * (kWarpChannels / 2) + (lane >> 2), quad = n0 / 4 + m.q;
        const bool odd = lane & 4, up = lane & 16, second = m.q & 2;
        __syncthreads();
        for (int i = n - 1; i >= 0; --i) {
            const int k = i & 1;
            const float4 *step = &sm.step[k][0][m.order][pair], *B = &sm.B[k][0][m.swap][quad], *C = &sm.C[k][0][m.swap][quad];
            const float2* dy = reinterpret_cast<const float2*>(&sm.dy[k][0][pair]) + m.order;
            if constexpr (LOCAL) {
#pragma unroll
                for (int t = K - 1; t >= 0; --t) {
                    const float4 v = step[t * 2 * S::PAIRS], c4 = C[t * 2 * (NS / 4)];
                    const float2 vy = dy[t * 2 * S::PAIRS];
                    const f2 dt[2] = {both(v.x), both(v.y)}, gy[2] = {both(vy.x), both(vy.y)}, vc[2] = {pack2(c4.x, c4.y), pack2(c4.z, c4.w)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) ga[j] = mul2(decay(dt[j >> 1], A2[j]), fma2(gy[j >> 1], vc[j & 1], ga[j]));
                    sum[0] += v.x;
                    sum[1] += v.y;
                }
            } else {
                copy_wait<S::SAVED - 2>();
                f2 hs[4], hm[4], tA[4] = {0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 4; ++j)                // the forward has the pairs of states in their order
                    hs[j] = hm[j] = reinterpret_cast<const f2*>(&sm.saved[i % S::SAVED][j >> 1][threadIdx.x])[(j & 1) ^ m.swap];
                fetch(i - (S::SAVED - 1));
#pragma unroll
                for (int t = 0; t < H; ++t) {              // the state in the middle of the tile
                    const float4 v = step[t * 2 * S::PAIRS], b4 = B[t * 2 * (NS / 4)];
                    const f2 dt[2] = {both(v.x), both(v.y)}, x[2] = {both(v.z), both(v.w)}, vb[2] = {pack2(b4.x, b4.y), pack2(b4.z, b4.w)};
#pragma unroll
                    for (int j = 0; j < 4; ++j) hm[j] = fma2(decay(dt[j >> 1], A2[j]), hm[j], mul2(x[j >> 1], vb[j & 1]));
                }
                auto half = [&](int base, f2(&h)[4]) {
                    f2 a[H][4], hp[H][4];
#pragma unroll
                    for (int t = 0; t < H; ++t) {
                        const float4 v = step[(base + t) * 2 * S::PAIRS], b4 = B[(base + t) * 2 * (NS / 4)];
                        const f2 dt[2] = {both(v.x), both(v.y)}, x[2] = {both(v.z), both(v.w)}, vb[2] = {pack2(b4.x, b4.y), pack2(b4.z, b4.w)};
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            a[t][j] = decay(dt[j >> 1], A2[j]);
                            hp[t][j] = h[j];
                            h[j] = fma2(a[t][j], h[j], mul2(x[j >> 1], vb[j & 1]));
                        }
                    }
                    // stored when the half is done: nothing stands in the way of the loads till then
                    float held = 0.f, out_bc[H], out_g[H], out_y[H / 2];
#pragma unroll
                    for (int t = H - 1; t >= 0; --t) {
                        const int tt = base + t;
                        const float4 v = step[tt * 2 * S::PAIRS], b4 = B[tt * 2 * (NS / 4)], c4 = C[tt * 2 * (NS / 4)];
                        const float2 vy = dy[tt * 2 * S::PAIRS];
                        const f2 dt[2] = {both(v.x), both(v.y)}, x[2] = {both(v.z), both(v.w)}, gy[2] = {both(vy.x), both(vy.y)};
                        const f2 vb[2] = {pack2(b4.x, b4.y), pack2(b4.z, b4.w)}, vc[2] = {pack2(c4.x, c4.y), pack2(c4.z, c4.w)};
                        f2 gB[2], gC[2], r1[2], r2[2], r3[2];
#pragma unroll
                        for (int c = 0; c < 2; ++c)
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                const int j = 2 * c + e;
                                const f2 ht = t == H - 1 ? h[j] : hp[t + 1 < H ? t + 1 : 0][j], gt = fma2(gy[c], vc[e], ga[j]);
                                ga[j] = mul2(gt, a[t][j]);
                                const f2 gp = mul2(ga[j], hp[t][j]);
                                gB[e] = c ? fma2(gt, x[c], gB[e]) : mul2(gt, x[c]);
                                gC[e] = c ? fma2(ht, gy[c], gC[e]) : mul2(ht, gy[c]);
                                r1[c] = e ? fma2(gt, vb[e], r1[c]) : mul2(gt, vb[e]);
                                r2[c] = e ? fma2(gp, A2[j], r2[c]) : mul2(gp, A2[j]);
                                r3[c] = e ? fma2(ht, vc[e], r3[c]) : mul2(ht, vc[e]);
                                tA[j] = fma2(gp, dt[c], tA[j]);
                            }
                        // dB, dC over the eight lanes of equal q: a lane keeps its first pair of states, of that the state c & 1, of dB and
                        // dC that of c / 4
                        const float2 B0 = unpack2(gB[0]), B1 = unpack2(gB[1]), C0 = unpack2(gC[0]), C1 = unpack2(gC[1]);
                        float w0 = B0.x + __shfl_xor_sync(kAll, B1.x, 8), w1 = B0.y + __shfl_xor_sync(kAll, B1.y, 8);
                        const float kB = (odd ? w1 : w0) + __shfl_xor_sync(kAll, odd ? w0 : w1, 4);
                        w0 = C0.x + __shfl_xor_sync(kAll, C1.x, 8);
                        w1 = C0.y + __shfl_xor_sync(kAll, C1.y, 8);
                        const float kC = (odd ? w1 : w0) + __shfl_xor_sync(kAll, odd ? w0 : w1, 4);
                        out_bc[t] = (up ? kC : kB) + __shfl_xor_sync(kAll, up ? kB : kC, 16);
                        // <g, B>, <g p, A>, <C, h> over the four lanes of equal c: a lane keeps its first channel, of the first two that of
                        // q / 2; of the third it keeps one of two tokens
                        const float k1 = sum_pair(r1[0]) + __shfl_xor_sync(kAll, sum_pair(r1[1]), 1);
                        const float k2 = sum_pair(r2[0]) + __shfl_xor_sync(kAll, sum_pair(r2[1]), 1);
                        const float k3 = sum_pair(r3[0]) + __shfl_xor_sync(kAll, sum_pair(r3[1]), 1);
                        out_g[t] = (second ? k2 : k1) + __shfl_xor_sync(kAll, second ? k1 : k2, 2);
                        if (t & 1) held = k3;
                        else out_y[t / 2] = (second ? held : k3) + __shfl_xor_sync(kAll, second ? k3 : held, 2);
                    }
                    float* g_to = &(second ? sm.gpA : sm.gB)[k][wb][base][wc * kWarpChannels + m.ch[0]];
                    float* bc_to = &sm.bc[k][warp][base][(up ? 16 : 0) + m.state(0, odd ? 1 : 0)];
#pragma unroll
                    for (int t = 0; t < H; ++t) {
                        bc_to[t * 32] = out_bc[t];
                        g_to[t * CC] = out_g[t];
                        if (!(t & 1)) sm.y[k][wb][base + t + (m.q >> 1)][wc * kWarpChannels + m.ch[0]] = out_y[t / 2];
                    }
                };
                half(H, hm);
                half(0, hs);
#pragma unroll
                for (int j = 0; j < 4; ++j) dA[j] = add2(dA[j], tA[j]);    // a tile's sum first: 2000 tokens one by one lose two digits
            }
            __syncthreads();
        }
        if (LOCAL) {
            store_end(p, seg - 1, b, mine, ga, A2, sum);
            return;
        }
        store_state(p, m, p.pA + part * d.D * d.N, g, ch, n0, dA);
        if (seg == 0 && p.dh0) store_state(p, m, p.dh0 + state, g, ch, n0, ga);
        return;
    }
    // ---- prepare tiles, write gradients ---------------------------------------------------------------------------------------
    if constexpr (!LOCAL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kPrepareRegs));
    const int tid = threadIdx.x - 32 * kWalkers;
    const size_t rows = (size_t)b * d.T, col = (size_t)g * d.K + ct * CC;
    const int left = d.K - ct * CC;
    // a thread prepares pairs of channels of PASSES tokens (where NB > 1 some threads none), keeps what it needs of them until the walk has
    // been there two tiles later, and writes out their gradients
    const int pr = tid % S::PAIRS, first = tid / S::PAIRS;
    float bias[2], skips[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        bias[e] = p.dt_bias && 2 * pr + e < left ? p.dt_bias[col + 2 * pr + e] : 0.f;
        skips[e] = !LOCAL && p.D && 2 * pr + e < left ? p.D[col + 2 * pr + e] : 0.f;
    }
    const f2 skip = pack2(skips[0], skips[1]);
    f2 sumD = 0, sumb = 0;
    struct Kept { f2 u, dt, dy, slope, gate; };             // slope: of the softplus; gate: dy SiLU'(z), with dy as it came in
    const size_t begin = rows + t0 + (n - 1) * K;          // of the last tile
    TileRun<K, CC, S::RING, IO, 4> run(&sm.u[0][0], {LOCAL ? nullptr : p.u, p.dt, p.z, p.dy}, begin, d.D, col, left, -K, tid);
    StateRun<NS, IO> states(p, begin, g, !LOCAL, true, -K, tid);
    auto fetch = [&](int i) {
        if (i >= 0) {
            const int tt = t0 + i * K, slot = i % S::RING;
            const bool whole = tt + K <= t1;
            if (whole && p.rows == kWhole) run.copy(slot, d.D);
            else copy_tiles<K, CC, IO, 4>({sm.u[slot], sm.dt[slot], sm.z[slot], sm.gy[slot]}, {LOCAL ? nullptr : p.u, p.dt, p.z, p.dy}, rows, d.D, tt, t1, col, left,
                                     p.rows, tid);
            if (whole && p.bc == kWhole) states.template copy<K>(sm.rbc[slot], tid);
            else
#pragma unroll
            for (int j = 0; j < S::BCT; ++j) {                             // four states of B or C of a token, which this thread prepares too
                const int x = tid + j * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4) * 4;
                if (bt >= K) break;
                const int have = tt + bt < t1 && !(LOCAL && r < NS / 4) ? d.N - s : 0;
                copy_group<4>(reinterpret_cast<IO*>(&sm.rbc[slot][j][tid]),
                              static_cast<const IO*>(r < NS / 4 ? p.Bm : p.Cm) + (have > 0 ? ((rows + tt + bt) * d.G + g) * d.N + s : 0), have, p.bc);
            }
        }
        run.move();
        states.move();
        copy_commit();
    };
    // Channels past the last have u = dy = 0 and any step; tokens past the last a step of 0.
    auto turn = [&](int i, Kept(&kept)[S::PASSES]) {
        const int k = i & 1, slot = i % S::RING;
#pragma unroll
        for (int r = 0; r < S::PASSES; ++r) {
            const int row = first + r * S::ROWS, at = row * CC + 2 * pr;
            if (S::ROWS > K && row >= K) break;
            const Pack<IO, 2> dt = load_pack<IO, 2>(&sm.dt[slot][at], 2, true), gy = load_pack<IO, 2>(&sm.gy[slot][at], 2, true);
            const Pack<IO, 2> u = LOCAL ? dt : load_pack<IO, 2>(&sm.u[slot][at], 2, true);
            float2 v = make_float2(pick(dt, 0) + bias[0], pick(dt, 1) + bias[1]), y = make_float2(pick(gy, 0), pick(gy, 1));
            if (p.softplus) {
                if (!LOCAL) kept[r].slope = pack2(gate_sigmoid(v.x), gate_sigmoid(v.y));
                v = softplus(v.x, v.y);
            }
            if (t0 + i * K + row >= t1) v.x = v.y = 0.f;
            if (p.z) {
                const Pack<IO, 2> z = load_pack<IO, 2>(&sm.z[slot][at], 2, true);
                const float z0 = pick(z, 0), z1 = pick(z, 1), s0 = gate_sigmoid(z0), s1 = gate_sigmoid(z1);
                if (!LOCAL) kept[r].gate = pack2(y.x * (s0 * fmaf(z0, 1.f - s0, 1.f)), y.y * (s1 * fmaf(z1, 1.f - s1, 1.f)));
                y.x *= z0 * s0;
                y.y *= z1 * s1;
            }
            const float u0 = pick(u, 0), u1 = pick(u, 1), x0 = v.x * u0, x1 = v.y * u1;
            if (!LOCAL) {
                kept[r].u = pack2(u0, u1);
                kept[r].dt = pack2(v.x, v.y);
                kept[r].dy = pack2(y.x, y.y);
            }
            sm.step[k][row][0][pr] = make_float4(v.x, v.y, x0, x1);
            sm.step[k][row][1][pr] = make_float4(v.y, v.x, x1, x0);
            sm.dy[k][row][pr] = make_float4(y.x, y.y, y.y, y.x);
        }
#pragma unroll
        for (int j = 0; j < S::BCT; ++j) {
            const int x = tid + j * 128, bt = x / (NS / 2), r = x % (NS / 2), s = r % (NS / 4);
            if (bt >= K) break;
            const Pack<IO, 4> v = sm.rbc[slot][j][tid];
            float4(&to)[2][NS / 4] = r < NS / 4 ? sm.B[k][bt] : sm.C[k][bt];
            to[0][s] = make_float4(pick(v, 0), pick(v, 1), pick(v, 2), pick(v, 3));
            to[1][s] = make_float4(pick(v, 2), pick(v, 3), pick(v, 0), pick(v, 1));
        }
    };
    const bool pairs = sizeof(IO) == 2 ? p.rows != kSingle : p.rows == kWhole;             // of the gradients, aligned
    auto finish = [&](int i, const Kept(&kept)[S::PASSES]) {                               // of a tile that has been walked
        const int k = i & 1;
#pragma unroll
        for (int r = 0; r < S::PASSES; ++r) {
            const int row = first + r * S::ROWS, t = t0 + i * K + row;
            if (row >= K || 2 * pr >= left || t >= t1) break;
            f2 gB = 0, gpA = 0, y = 0;
#pragma unroll
            for (int w = 0; w < NB; ++w) {
                const f2 a = *reinterpret_cast<const f2*>(&sm.gB[k][w][row][2 * pr]), c = *reinterpret_cast<const f2*>(&sm.gpA[k][w][row][2 * pr]);
                const f2 f = *reinterpret_cast<const f2*>(&sm.y[k][w][row][2 * pr]);
                gB = w ? add2(gB, a) : a;
                gpA = w ? add2(gpA, c) : c;
                y = w ? add2(y, f) : f;
            }
            const Kept& x = kept[r];
            f2 ddt = fma2(gB, x.u, mul2(gpA, both(kLn2)));
            if (p.softplus) ddt = mul2(ddt, x.slope);
            sumD = fma2(x.dy, x.u, sumD);
            sumb = add2(sumb, ddt);
            const size_t to = (rows + t) * d.D + col + 2 * pr;
            auto put = [&](void* out, f2 v) {
                const float2 o = unpack2(v);
                const float w[2] = {o.x, o.y};
                store_pack(static_cast<IO*>(out) + to, narrow<IO, 2>(w), left - 2 * pr, pairs);
            };
            put(p.du, fma2(gB, x.dt, mul2(skip, x.dy)));
            put(p.ddt, ddt);
            if (p.z) put(p.dz, mul2(x.gate, fma2(skip, x.u, y)));
        }
        // dB, dC of the CTA's channels: four states of a token
#pragma unroll
        for (int j = 0; j < S::BCT; ++j) {
            const int x = tid + j * 128, tk = x / (NS / 2), which = x / (NS / 4) % 2, s = x % (NS / 4) * 4, tt = t0 + i * K + tk;
            if (tk >= K || tt >= t1 || s >= d.N) continue;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < CW; ++w) {
                const float4 a = *reinterpret_cast<const float4*>(&sm.bc[k][s / kWarpStates * CW + w][tk][which * 16 + s % kWarpStates]);
                v[0] += a.x; v[1] += a.y; v[2] += a.z; v[3] += a.w;
            }
            Pack<float, 4> o;
#pragma unroll
            for (int e = 0; e < 4; ++e) o.w[e] = __float_as_uint(v[e]);
            store_pack(p.pBC + ((size_t)ct * 2 + which) * p.bcs + ((rows + tt) * d.G + g) * d.N + s, o, d.N - s, p.bc == kWhole);
        }
    };
#pragma unroll
    for (int e = 1; e <= S::RING - 2; ++e) fetch(n - e);
    copy_wait<S::RING - 4>();                                              // the first two tiles
    prepare_barrier();
    Kept kept[2][S::PASSES];                                               // of the next tile to be finished, of the one after it
    turn(n - 1, kept[1]);
    __syncthreads();
    for (int i = n - 1; i >= 0; --i) {
        if (!LOCAL) {
            if (i < n - 1) finish(i + 1, kept[0]);
#pragma unroll
            for (int r = 0; r < S::PASSES; ++r) kept[0][r] = kept[1][r];
        }
        fetch(i - (S::RING - 2));                                          // where a tile stood that was finished before the last barrier
        // (the next tile's steps, dy, B and C take the place of those of the tile before, which the walk read before the last barrier; what is
        // finished here lies elsewhere)
        if (i > 0) turn(i - 1, kept[1]);
        copy_wait<S::RING - 4>();                                          // tile i - 2, for all after the barrier
        __syncthreads();
    }
    if (LOCAL) return;
    finish(0, kept[0]);
    // sums over the tokens of a channel: the threads that share it in order
    constexpr int R = S::ROWS < K ? S::ROWS : K;
    float* cols = reinterpret_cast<float*>(sm.step);
    prepare_barrier();
    if (first < K) {
        *reinterpret_cast<f2*>(&cols[first * CC + 2 * pr]) = sumD;
        *reinterpret_cast<f2*>(&cols[(R + first) * CC + 2 * pr]) = sumb;
    }
    prepare_barrier();
    for (int x = tid; x < 2 * CC; x += 128) {
        const int which = x / CC, c = x % CC;
        if (c >= left) continue;
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) v += cols[(which * R + r) * CC + c];
        p.pD[(part * 2 + which) * d.D + col + c] = v;
    }
}

// Partials added in their order: dB and dC from the CTAs', and where there are few, dA, dD and that of dt_bias from the sequences' and
// segments' (one launch instead of three: 24 us instead of 27 for the backward of 100 tokens of 512 channels; with 64 parts 153 and 151).
constexpr int kFewParts = 32;
struct Sums {
    const float *bc, *A, *D;
    size_t rows, DN, D2;                     // values of dB; of dA and of dD and ddt_bias, 0 if they are not for this kernel
    int bc_parts, parts;
    void *dB, *dC;
    float *dA, *dD, *dbias;
};
__device__ __forceinline__ float sum_column(const float* part, int parts, size_t stride) {
    float v = 0.f;
#pragma unroll 8
    for (int k = 0; k < parts; ++k) v += part[k * stride];
    return v;
}
template <typename IO>
__global__ void __launch_bounds__(256) k_scan_sums(const Sums s) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (i < 2 * s.rows) {
        st(static_cast<IO*>(i < s.rows ? s.dB : s.dC), i < s.rows ? i : i - s.rows, sum_column(s.bc + i, s.bc_parts, 2 * s.rows));
        return;
    }
    i -= 2 * s.rows;
    if (i < s.DN) {
        s.dA[i] = sum_column(s.A + i, s.parts, s.DN);
        return;
    }
    i -= s.DN;
    if (i >= s.D2) return;
    float* out = i < s.D2 / 2 ? s.dD : s.dbias;
    if (out) out[i < s.D2 / 2 ? i : i - s.D2 / 2] = sum_column(s.D + i, s.parts, s.D2);
}

struct BwdPlan { Dims d; Cut c; size_t saved, ends, pA, pD, pBC, bytes; };
BwdPlan bwd_plan(const qd_scan_shape& s) {
    BwdPlan q{};
    q.d = dims(s);
    q.c = cut(q.d, true);
    const auto up = [](size_t n) { return (n + 255) / 256 * 256; };
    q.saved = (size_t)s.B * ((s.T + kSave - 1) / kSave) * q.d.states * sizeof(float);
    q.ends = (size_t)(q.c.segs - 1) * s.B * q.d.states * sizeof(float);
    q.pA = up((size_t)q.c.segs * s.B * s.D * s.N * sizeof(float));
    q.pD = up((size_t)q.c.segs * s.B * 2 * s.D * sizeof(float));
    q.pBC = up((size_t)q.d.ctas * 2 * s.B * s.T * s.G * s.N * sizeof(float));
    q.bytes = q.saved + 2 * q.ends + q.pA + q.pD + q.pBC;
    return q;
}

template <typename IO, int NB>
cudaError_t launch(const P& p, cudaStream_t stream) {
    const long long per = (long long)p.d.ctas * p.d.G * p.d.B;
    constexpr size_t smem = sizeof(BwdSmem<IO, NB>);
    constexpr size_t most = smem > kAloneSmem ? smem : kAloneSmem;
    cudaError_t e;
    if (p.segs > 1) {
        e = set_max_smem_once((const void*)k_scan_bwd<IO, NB, true>, most);
        if (e == cudaSuccess)
            e = launch_overlapped(k_scan_bwd<IO, NB, true>, dim3((unsigned)(per * (p.segs - 1))), dim3(kThreads), per * (p.segs - 1) > kSMs ? smem : most, stream, p);
        if (e == cudaSuccess && p.joined) e = join(p.ends, p.decays, p.segs - 1, p.segs - 2, -1, (size_t)p.d.B * p.d.states, stream);
        if (e != cudaSuccess) return e;
    }
    e = set_max_smem_once((const void*)k_scan_bwd<IO, NB, false>, most);
    if (e != cudaSuccess) return e;
    return launch_overlapped(k_scan_bwd<IO, NB, false>, dim3((unsigned)(per * p.segs)), dim3(kThreads), per * p.segs > kSMs ? smem : most, stream, p);
}
template <typename IO>
cudaError_t launch(const P& p, const ScanArgs& a) {
    cudaError_t e = p.d.nb == 1 ? launch<IO, 1>(p, a.stream) : p.d.nb == 2 ? launch<IO, 2>(p, a.stream) : launch<IO, 4>(p, a.stream);
    if (e != cudaSuccess) return e;
    Sums s{};
    s.bc = p.pBC; s.A = p.pA; s.D = p.pD;
    s.rows = (size_t)p.d.B * p.d.T * p.d.G * p.d.N;
    s.bc_parts = p.d.ctas; s.parts = p.segs * p.d.B;
    s.dB = a.dBm; s.dC = a.dCm; s.dA = a.dA; s.dD = a.dD; s.dbias = a.ddt_bias;
    const bool few = s.parts <= kFewParts, columns = a.dD || a.ddt_bias;
    if (few) {
        s.DN = (size_t)p.d.D * p.d.N;
        s.D2 = columns ? 2 * (size_t)p.d.D : 0;
    }
    const size_t n = 2 * s.rows + s.DN + s.D2;
    e = launch_overlapped(k_scan_sums<IO>, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, a.stream, s);
    if (e != cudaSuccess || few) return e;
    const long long D = p.d.D, DN = D * p.d.N;
    e = sum_parts(p.pA, s.parts, DN, DN, DN, 1, a.dA, nullptr, a.stream);
    return e != cudaSuccess || !columns ? e : sum_parts(p.pD, s.parts, 2 * D, D, D, 1, a.dD, a.ddt_bias, a.stream);
}
}  // namespace

// that of the forward that saves for it, too
size_t scan_bwd_workspace(const qd_scan_shape& s) {
    const size_t fwd = scan_fwd_workspace(s, true), bwd = bwd_plan(s).bytes;
    return fwd > bwd ? fwd : bwd;
}

cudaError_t scan_bwd(const ScanArgs& a) {
    const BwdPlan q = bwd_plan(a.s);
    P p{};
    p.d = q.d; p.segs = q.c.segs; p.first = q.c.first; p.seglen = q.c.len;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.D = a.D; p.dt_bias = a.dt_bias;
    p.dy = a.dy; p.dhT = a.dhT; p.du = a.du; p.ddt = a.ddt; p.dz = a.dz; p.dh0 = a.dh0;
    char* w = a.ws;
    p.saved = reinterpret_cast<float*>(w); w += q.saved;
    p.ends = reinterpret_cast<float*>(w); w += q.ends;
    p.decays = reinterpret_cast<float*>(w); w += q.ends;
    p.pA = reinterpret_cast<float*>(w); w += q.pA;
    p.pD = reinterpret_cast<float*>(w); w += q.pD;
    p.pBC = reinterpret_cast<float*>(w);
    p.bcs = (size_t)a.s.B * a.s.T * a.s.G * a.s.N;
    p.softplus = a.softplus; p.rows = copy_of(q.d.K, a.s.dtype == QD_BF16 ? 8 : 4, a.s.dtype); p.bc = copy_of(a.s.N, 4, a.s.dtype);
    p.joined = p.segs - 1 > kMostJoined;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a) : launch<float>(p, a);
}

}  // namespace qd

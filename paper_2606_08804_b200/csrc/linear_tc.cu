// Linear attention in bf16 on the tensor cores: a walk (linear.cuh) over chunks of 128 tokens to a CTA, every product a tcgen05.mma:
//     P = (a b^T) o D  (rounded to bf16 as the next operand)      out = P c + rho (a S)      S <- e^{g n} S + (kappa b)^T c
// Row r of out has the factor e^{g (r - 63)} (backward e^{g (64 - r)}) in all its terms, which is multiplied in last: what is left of D and rho
// depends on the column alone, and is at most e^{64 |g|} either way.  That much of fp32's range is lost at both ends, for weights, states and
// outputs, so heads with |g| > kSlight, 2^16, form D as it stands and multiply a S by rho between the two products: 8 x 2048 x 16 forward
// 65 us for 64, without the state 67 for 59, backward 170 for 163 where four heads do (66, 66 and 186 where all do).
// The state stays in fp32 registers; each chunk's sum comes from tensor memory and is added there (the tensor cores cut as they accumulate).
// For a S it goes to shared memory in bf16.  In S the factor kappa stands with c, as bf16 planes cut from kappa c: three, which hold all of its
// 24 bits, where the state is returned (with two, even rounded ones, it is 2.4e-6 of its length off, more than a whole fp32 sum over a sequence
// is); two, 2^-15 apart, where it serves bf16 outputs alone (with one, dq and dk are off by 1.53 times what their own rounding costs, with two
// by 1.35).
//
// 8 x 2048 tokens, 16 heads of 128 x 128, 128 CTAs: 59 us, 5300 cycles a chunk, 4.5 TB/s of the 6.46 that a copy has (its bytes alone 41.5); 64 us with
// three planes.  No unit is full (tensor pipe 43 %, issue slots 47 %): it is a chunk's chain, scores to weights to out, and sum to state to a S,
// with one CTA to an SM and 20 SMs without any.  The products of a chunk are 2560 cycles, 512 more with three planes.  Next to that it is
// shared memory, 128 bytes a cycle, which a product of 128 x 128 with both operands there takes all of; so P and the planes are operands in
// tensor memory (c read transposed from its tile), and the parts of out, a S and P c, share one accumulator, scaled in between: 78 us with the
// planes in shared memory and two accumulators.  Six tile buffers, two chunks deep: b, c, a of each; out leaves through a's.  All sixteen warps make planes, a quarter each; with the state's left out of it 61 us, 48 for 44 at
// 64 x 64, backward 173 for 160 then.  Launched again and again it runs into the GPU's power limit (forward and backward 235 us in short loops, 271
// in long ones).
// The sums of segments alone (ENDS), 32768 tokens of 16 heads: 60 us, of bytes 41.5.
//   warps 0-7    two warpgroups: planes of the first two parts; P, half of the columns, from tensor memory and back to it; out, half of the
//                columns, staged in a's tile, stored by TMA
//   warps 8-15   planes of the other two parts; state, transposed: a column of S to a lane, half of the rows to a warpgroup; a S times rho, if
//                |g| > kSlight
//   warp 16      issues the products;  warp 17  loads
// Out's rows before a token take nothing of it, also where it is infinite or NaN: the planes' warps, which read all of c, put a 0 in such an
// element's place for P c and note its column and place; from there on the column of out is NaN (as the state is for later chunks).
// All waits are bounded; on expiry the status word says so, everybody leaves, what is in flight is waited for, and what the CTA was to write
// becomes NaN: calls whose workspace nobody sees, those through autograd, do not go on with half a result.
#include "linear.cuh"
#include "rows.cuh"

namespace qd {
namespace {
using namespace sm100;

constexpr int kTokens = 128, kPart = 32, kParts = kTokens / kPart, kTcThreads = 18 * 32;
// Registers: 18 warps are launched with 96 a thread (five to one of the SM's quarters), too few for the state's and a part of planes.
constexpr int kLaunchRegs = 96, kGroupRegs = 80, kStateRegs = 112;
static_assert(kGroupRegs + kStateRegs <= 2 * kLaunchRegs, "what one takes another has given");
constexpr float kSlight = 0.173f;            // e^{64 kSlight} < 2^16

// The upper halves of a pair of fp32 values as packed bf16; what they leave stays behind, exactly.
__device__ __forceinline__ uint32_t cut(f2& x) {
    const float2 v = unpack2(x);
    const uint32_t lo = __float_as_uint(v.x), hi = __float_as_uint(v.y);
    x = add2(x, pack2(-__uint_as_float(lo & 0xffff0000u), -__uint_as_float(hi & 0xffff0000u)));
    return __byte_perm(lo, hi, 0x7632);
}

struct LinearMaps { CUtensorMap a[kLinearWalks], b[kLinearWalks], c[kLinearWalks], out[kLinearWalks]; };

template <int DB, int DC, bool ENDS>
struct TcLinear {
    static constexpr int kSlot = kTokens * (DB > DC ? DB : DC) * 2;
    static constexpr int kPer = ENDS ? 2 : 3;                         // tiles of a chunk: b, c, a
    static constexpr int kRing = 2 * kPer;                            // two chunks: barriers of chunks n and n + 2 are the same
    static constexpr int kState = ENDS ? 0 : DB * DC * 2;
    static constexpr int kSmem = kState + kRing * kSlot + 1024;
    static constexpr int kPlane = kPart / 2;                          // columns of tensor memory: scores, out, sum, planes
    static constexpr int kOut = ENDS ? 0 : kTokens, kSum = ENDS ? 0 : kOut + DC;
    static constexpr int kSums = ENDS ? 2 : 1, kPlanes = kSum + kSums * DB;   // of a chunk's sum: one is read while the next is made, where there is room
    static constexpr int kUsed = kPlanes + kParts * (ENDS ? 3 : 2) * kPlane;      // all of a chunk's parts; three planes through two places
    static constexpr int kColumns = kUsed > 256 ? 512 : kUsed > 128 ? 256 : 128;
    static_assert(kSmem <= 232448 - 2048, "the tables and barriers below need the rest");
};

template <int DB, int DC, bool ENDS>
__global__ void __launch_bounds__(kTcThreads, 1) k_linear_tc(const __grid_constant__ LinearMaps maps, const LinearP p) {
    typedef TcLinear<DB, DC, ENDS> L;
    constexpr int kRing = L::kRing, kPer = L::kPer, kA = 2, kC = 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char *sState = smem, *sRing = smem + L::kState;
    // bar_s, bar_o2, bar_o, bar_kq, bar_kv: products complete (scores, a S, out twice, a part's and all of a chunk's sum); bar_p, bar_os, bar_k,
    // bar_h: operands in place; bar_of, bar_kr: out's and the sum's accumulator have been read; bar_af: a's tile is free.  Where one side
    // runs up to two phases ahead there is one for even and one for odd phases.
    __shared__ uint64_t bar_full[kRing], bar_s, bar_o2, bar_o, bar_c[2], bar_kv[2], bar_kq[kParts], bar_p, bar_os, bar_k[kParts], bar_h, bar_of, bar_kr[L::kSums], bar_af[2], bar_end;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int s_abort, s_unfit;                  // s_unfit: c has had an element that is infinite or NaN
    // What is left of D for a column; or, |g| > kSlight, D(|m|), m from -128, of which one half counts.  In the other, for every column of c: the
    // first element that is infinite or NaN, counted in the order of the walk.
    __shared__ __align__(16) float s_d[2 * kTokens + 1];
    __shared__ Keep s_keep[2];                                 // over a whole chunk, over the sequence's last
    __shared__ float s_k[kTokens + 1];                                             // kappa of a whole chunk; 0 behind it

    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, wq = warp & 3;
    const int walk = blockIdx.x % p.walks, cta = blockIdx.x / p.walks, segment = cta % p.segments, bh = cta / p.segments;
    const int b = bh / p.H, hh = bh % p.H;
    const LinearWalk& w = p.w[walk];
    const int first = segment * p.length, end = min(p.T, first + p.length), chunks = (end - first + kTokens - 1) / kTokens;
    // the state that is returned is that of the last segment, and what the others' sums make of it before
    const bool reverse = w.reverse, last_one = segment == (reverse ? 0 : p.segments - 1), exact = w.exact && (ENDS || last_one);
    auto token0 = [&](int n) { return first + (reverse ? chunks - 1 - n : n) * kTokens; };

    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(&bar_full[i], 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&bar_c[i], 1); mbar_init(&bar_af[i], DC == 128 ? 8 : 4); }
        for (int i = 0; i < kParts; ++i) { mbar_init(&bar_kq[i], 1); mbar_init(&bar_k[i], 4); }
        mbar_init(&bar_s, 1); mbar_init(&bar_o2, 1); mbar_init(&bar_o, 1); mbar_init(&bar_p, 8); mbar_init(&bar_os, 8); mbar_init(&bar_of, DC == 128 ? 8 : 4);
        mbar_init(&bar_h, 8);
        for (int i = 0; i < L::kSums; ++i) mbar_init(&bar_kr[i], 8);
        mbar_init(&bar_end, 1);
        mbar_init_fence();
        s_abort = s_unfit = 0;
    }
    if (warp == 0) { tmem_alloc(&tmem_slot, L::kColumns); tmem_relinquish(); }
    grid_dep_wait();
    grid_dep_launch();
    const float g = p.g[hh], g2 = g * 1.4426950408889634f;
    const bool steep = !(fabsf(g) <= kSlight);
    const int other = !steep ? kTokens : reverse ? kTokens + 1 : 0;
    volatile int* const s_first = reinterpret_cast<volatile int*>(s_d) + other;
    if (tid <= 2 * kTokens)
        s_d[tid] = tid >= other && tid < other + kTokens ? __int_as_float(0x7fffffff)
                                                         : p.scale * decay_power(g2, steep ? abs(tid - kTokens) : reverse ? tid - 64 : 63 - tid);
    if (tid <= kTokens) s_k[tid] = tid == kTokens ? 0.f : reverse ? p.scale * decay_power(g2, tid + 1) : decay_power(g2, kTokens - 1 - tid);
    if (tid < 2) s_keep[tid] = keep_power(g, tid ? end - first - (chunks - 1) * kTokens : kTokens);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = uniform(tmem_slot);
    const uint32_t tS = tb, tO = tb + L::kOut, tKV = tb + L::kSum, tPlanes = tb + L::kPlanes;
    const uint32_t lanes = (uint32_t)wq * 32;

    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_try_wait(bar, parity) || wait_on(bar, parity, s_abort, p.status); };
    auto all = [&](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };
    auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
    auto slot = [&](int m) { return sRing + m % kRing * L::kSlot; };
    auto full = [&](int m) { return wait(&bar_full[m % kRing], (m / kRing) & 1); };

    // kappa c of part q, 32 tokens, transposed: a column of c to a lane of tensor memory, in three planes or in two.
    const int count = exact ? 3 : 2;
    const bool shared = !ENDS && exact;                            // two places for four parts
    auto place_of = [&](int q) { return shared ? (q & 1) * 3 * L::kPlane : q * (ENDS ? 3 : 2) * L::kPlane; };
    auto planes = [&](int n, int q) {
        const int live = min(kTokens, end - token0(n)), late = reverse ? 0 : kTokens - live;
        // what was in this place before: this part of the chunk before, or, three planes through two places, two parts before
        const bool same = shared && q >= 2;
        if ((n > 0 || same) && !all(wait(&bar_kq[shared ? q ^ 2 : q], (same ? n : n - 1) & 1))) return false;
        const unsigned char* tile = slot(n * kPer + kC);
        const uint32_t to = tmem_addr(tPlanes, lanes, place_of(q));
        constexpr int kHalves = DC == 128 ? 2 : 1;                                    // 64 rows: 16 to each of a warpgroup's four warps
        uint32_t seen = 0;
#pragma unroll 1
        for (int k = 0; k < 2; ++k) {                                                 // 16 tokens
            float kappa[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int t = q * kPart + 16 * k + 8 * (e >> 1) + 2 * (lane & 3) + (e & 1);
                kappa[e] = s_k[t >= live ? kTokens : t + late];
            }
#pragma unroll
            for (int half = 0; half < kHalves; ++half) {
                uint32_t raw[4], r[4];
                const int col = (DC == 128 ? 32 * wq + 16 * half : 16 * wq) + ((lane >> 3) & 1) * 8;
                ldsm4<true>(tile + (col >> 6) * kTokens * 128 + sw128_chunk(q * kPart + 16 * k + (lane >> 4) * 8 + (lane & 7), (col >> 3) & 7), raw);
                if (!ENDS) { see_unfit(seen, raw[0], raw[1]); see_unfit(seen, raw[2], raw[3]); }
                f2 x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[e] = mul2(pack2(kappa[e & ~1], kappa[e | 1]), pack2(__uint_as_float(raw[e] << 16), __uint_as_float(raw[e] & 0xffff0000u)));
                const uint32_t at = tmem_addr(to, 16 * half, 8 * k);
#pragma unroll
                for (int m = 0; m < 3; ++m) {                                         // cut to 8 bits, three times: nothing is left of 24
                    if (m == 2 && !exact) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) r[e] = cut(x[e]);
                    tmem_st_frag2(at + m * L::kPlane, r);
                }
            }
        }
        if (!ENDS && __any_sync(0xffffffffu, seen_unfit(seen))) {                            // what this warp has read, element by element
            constexpr int wide = DC / 4;
            unsigned char* const mine = slot(n * kPer + kC);
#pragma unroll 1
            for (int i = lane; i < kPart * wide; i += 32) {
                const int t = q * kPart + i / wide, col = wq * wide + i % wide;
                volatile unsigned short* const x =
                    reinterpret_cast<volatile unsigned short*>(mine + (col >> 6) * kTokens * 128 + sw128_chunk(t, (col >> 3) & 7)) + (col & 7);
                if ((*x & 0x7f80) != 0x7f80) continue;
                *x = 0;
                atomicMin(const_cast<int*>(s_first) + col, n * kTokens + (reverse ? kTokens - 1 - t : t));
                s_unfit = 1;
            }
            fence_proxy_async();
        }
        tmem_st_wait();
        tc_fence_before();
        arrive(&bar_k[q]);
        return true;
    };
    int loads = 0;                                                        // issued by this thread
    if (p.clear && blockIdx.x == 0 && tid == 0) *p.status = 0;
    if (ENDS && last_one) {
        // nobody begins with the sums of this one
    } else if (warp < 8) {
        // ---------------------------------- planes, weights and output ----------------------------------
        // Two warpgroups, alike: of the weights' columns and of out's each takes half.
        // One copy of every piece of code, and loops as loops: what all warps go through in a chunk has to fit the instruction cache
        // (planes and weights written out: 12000 cycles a chunk).
        give_registers<kGroupRegs>();
        const int r = (int)lanes + lane, group = warp >> 2;
        const float* far = s_d + kTokens + r;
        const float last = steep ? 1.f : decay_power(g2, reverse ? 64 - r : r - 63);
        constexpr bool kSplit = DC == 128;                         // else the second group has all of out: 64 columns are one box
        int stored = -1;                                           // chunk whose output this thread has stored and not seen read
        auto output = [&](int n) {
            if (!kSplit && group == 0) return true;
            if (!all(wait(&bar_o, n & 1))) return false;
            tc_fence_after();
            unsigned char* stage = slot(n * kPer + kA) + (kSplit ? group * kTokens * 128 : 0);
            const uint32_t from = tmem_addr(tO, lanes, kSplit ? 64 * group : 0);
            float x[2][16];                                        // the next columns come while these are written
            tmem_ld16(from, x[0]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                tmem_ld_wait();
                if (j < 3) tmem_ld16(from + 16 * j + 16, x[(j + 1) & 1]);
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float2 y = unpack2(mul2(pack2(x[j & 1][e], x[j & 1][e + 1]), both(last)));
                    x[j & 1][e] = y.x; x[j & 1][e + 1] = y.y;
                }
#pragma unroll
                for (int ch = 0; ch < 2; ++ch) sts128(stage + sw128_chunk(r, 2 * j + ch), pack8(x[j & 1] + 8 * ch));
            }
            if (s_unfit) {
                const int at = n * kTokens + (reverse ? kTokens - 1 - r : r);
#pragma unroll 1
                for (int col = 0; col < 64; ++col)
                    if (at >= s_first[(kSplit ? 64 * group : 0) + col])
                        reinterpret_cast<volatile unsigned short*>(stage + sw128_chunk(r, col >> 3))[col & 7] = 0x7fff;
            }
            tc_fence_before();
            arrive(&bar_of);
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                const int t0 = token0(n) + (int)lanes;
                if (t0 < p.T) {                                    // rows past the end of the sequence are skipped
                    tma_store_3d(&maps.out[walk], stage + lanes * 128, hh * DC + (kSplit ? 64 * group : 0), t0, b);
                    tma_store_commit();
                }
                stored = n;
            }
            __syncwarp();
            return true;
        };
        auto weights = [&](int n) {
            if (!all(wait(&bar_s, n & 1))) return false;
            tc_fence_after();
#pragma unroll 1
            for (int j = 2 * group; j < 2 * group + 2; ++j) {      // 32 columns i, which become 16 packed ones in the place of what has been read
                uint32_t o[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0;
                if (reverse ? j >= wq : j <= wq) {
                    float v[32];
                    tmem_ld32(tmem_addr(tS, lanes, 32 * j), v);
                    tmem_ld_wait();
                    if (steep) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] *= far[-32 * j - e];
                        const int live = min(kTokens, end - token0(n)) - 32 * j;
                        if (reverse && live < 32)                  // tokens past the end, whose D may be infinite
#pragma unroll
                            for (int e = 0; e < 32; ++e) v[e] = e < live ? v[e] : 0.f;
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            const float4 t = *reinterpret_cast<const float4*>(s_d + 32 * j + e);
                            const float2 x = unpack2(mul2(pack2(v[e], v[e + 1]), pack2(t.x, t.y))), y = unpack2(mul2(pack2(v[e + 2], v[e + 3]), pack2(t.z, t.w)));
                            v[e] = x.x; v[e + 1] = x.y; v[e + 2] = y.x; v[e + 3] = y.y;
                        }
                    }
                    if (j == wq)                                   // an infinite product past the diagonal leaves nothing either
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = (reverse ? e >= lane : e <= lane) ? v[e] : 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                }
                tmem_st8(tmem_addr(tS, lanes, 32 * group + 16 * j), o);
                tmem_st8(tmem_addr(tS, lanes, 32 * group + 16 * j + 8), o + 8);
            }
            tmem_st_wait();
            tc_fence_before();
            arrive(&bar_p);
            if (stored >= 0) {                                     // the output of the chunk before has been read by now: its tile is free
                tma_store_wait_read();
                mbar_arrive(&bar_af[stored & 1]);
                stored = -1;
            }
            __syncwarp();
            return true;
        };
        bool ok = true;
#pragma unroll 1
        for (int n = 0; n <= chunks && ok; ++n) {
            if (n < chunks) ok = all(full(n * kPer + kC)) && planes(n, group);
            if (ENDS || !ok) continue;
            if (n > 0) ok = output(n - 1);
            if (n < chunks) ok = ok && weights(n);
        }
        if (lane == 0) tma_store_wait_all();
    } else if (warp < 16) {
        // ---------------------------------- state ----------------------------------
        take_registers<kStateRegs>();
        constexpr int HC = DB / 2, size = DB * DC;
        const int r = DC == 128 ? (int)lanes + lane : 16 * wq + (lane & 15), c0 = (warp - 8) / 4 * HC;
        const bool live_row = DC == 128 || lane < 16;
        float h[HC];
        auto place = [&](int i) { return w.flip ? r * DB + c0 + i : (c0 + i) * DC + r; };
        const float* entry = !ENDS && w.s0 && live_row ? w.s0 + ((size_t)bh * p.segments + segment) * size : nullptr;
        if (entry && w.flip) {
#pragma unroll
            for (int i = 0; i < HC; i += 4) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(entry + place(i)));
                h[i] = t.x; h[i + 1] = t.y; h[i + 2] = t.z; h[i + 3] = t.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < HC; ++i) h[i] = entry ? __ldcg(entry + place(i)) : 0.f;
        }
        auto put = [&](int n) {                                    // as chunk n's operand
            if (ENDS) return;
            const float f = steep ? 1.f : reverse ? decay_power(g2, min(kTokens, end - token0(n)) - 65) : p.scale * decay_power(g2, 64);
            if (live_row)
#pragma unroll
                for (int ch = 0; ch < HC / 8; ++ch) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float2 y = unpack2(mul2(pack2(h[8 * ch + e], h[8 * ch + e + 1]), both(f)));
                        x[e] = y.x; x[e + 1] = y.y;
                    }
                    sts128(sState + (c0 + 8 * ch) / 64 * (DC * 128) + sw128_chunk(r, ((c0 >> 3) + ch) & 7), pack8(x));
                }
            fence_proxy_async();
            arrive(&bar_h);
        };
        put(0);
        // planes a chunk ahead of the state, where their place does not wait for a sum that waits for the state
        for (int n = shared ? 0 : -1; n < chunks; ++n) {
            const int live = min(kTokens, end - token0(n)), row = (int)lanes + lane, ahead = shared ? n : n + 1;
            if (ahead < chunks && (!all(full(ahead * kPer + kC)) || !planes(ahead, warp >> 2))) break;
            if (n < 0) continue;
            if (!ENDS && steep) {                                  // a S times rho, half of the columns to a warpgroup
                const float rho = row >= live ? 0.f : reverse ? decay_power(g2, live - 1 - row) : p.scale * decay_power(g2, row + 1);
                if (!all(wait(&bar_o2, n & 1))) break;
                tc_fence_after();
#pragma unroll 1
                for (int j = 0; j < DC / 32; ++j) {
                    const uint32_t at = tmem_addr(tO, lanes, (warp - 8) / 4 * (DC / 2) + 16 * j);
                    float v[16];
                    tmem_ld16(at, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] *= rho;
                    tmem_st8(at, reinterpret_cast<const uint32_t*>(v));
                    tmem_st8(at + 8, reinterpret_cast<const uint32_t*>(v + 8));
                }
                tmem_st_wait();
                tc_fence_before();
                arrive(&bar_os);
            }
            if (!all(wait(&bar_kv[n & 1], (n >> 1) & 1))) break;
            tc_fence_after();
            const Keep keep = s_keep[live < kTokens];
            const f2 base = both(keep.base), more = both(keep.more);
#pragma unroll
            for (int j = 0; j < HC / 16; ++j) {
                float v[16];
                tmem_ld16(tmem_addr(tKV, lanes, n % L::kSums * DB + c0 + 16 * j), v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const f2 x = pack2(h[16 * j + e], h[16 * j + e + 1]);
                    const float2 y = unpack2(fma2(more, x, fma2(base, x, pack2(v[e], v[e + 1]))));
                    h[16 * j + e] = y.x; h[16 * j + e + 1] = y.y;
                }
            }
            tc_fence_before();
            arrive(&bar_kr[n % L::kSums]);
            if (n + 1 < chunks) put(n + 1);
        }
        float* left = ENDS ? w.ends + ((size_t)bh * p.segments + segment) * size
                           : last_one && w.sT ? w.sT + (size_t)bh * size : nullptr;
        if (left && live_row && !s_abort) {
            if (w.flip) {
#pragma unroll
                for (int i = 0; i < HC; i += 4) *reinterpret_cast<float4*>(left + place(i)) = make_float4(h[i], h[i + 1], h[i + 2], h[i + 3]);
            } else {
#pragma unroll
                for (int i = 0; i < HC; ++i) left[place(i)] = h[i];
            }
        }
    } else if (warp == 16) {
        // ---------------------------------- products, by the converged warp ----------------------------------
        const uint32_t issue = elect_lane();
        const uint32_t aState = smem_u32(sState), aRing = smem_u32(sRing);
        auto tile = [&](int m) { return aRing + (uint32_t)(m % kRing) * L::kSlot; };
        constexpr uint32_t blk = kTokens * 128;
        auto scores = [&](int n) {
            if (!all(full(n * kPer))) return false;
            if (ENDS) return true;
            if (!all(full(n * kPer + kA))) return false;
            umma_product_w<false, false>(tS, tile(n * kPer + kA), blk, tile(n * kPer), blk, kTokens, DB, false, issue);
            umma_commit_w(&bar_s, issue);
            return true;
        };
        auto part = [&](int n, int q) {
            if (!all(wait(&bar_k[q], n & 1))) return false;
            tc_fence_after();
#pragma unroll 1
            for (int m = 0; m < count; ++m)
                umma_product_ts_w<true, DC>(tKV + n % L::kSums * DB, tPlanes + place_of(q) + m * L::kPlane, tile(n * kPer) + q * kPart * 128, blk, DB, kPart, q + m > 0, issue);
            umma_commit_w(&bar_kq[q], issue);
            return true;
        };
        // The state that a chunk begins with is made under the two products that do not need it, the weights under those of the sum.
        if (scores(0))
            for (int n = 0; n < chunks; ++n) {
                if (n >= L::kSums && !all(wait(&bar_kr[n % L::kSums], (n / L::kSums - 1) & 1))) break;      // what was in this sum's place
                tc_fence_after();
                bool ok = true;
#pragma unroll 1
                for (int q = 0; q < kParts && ok; ++q) {
                    ok = part(n, q);
                    if (ENDS || q != kParts / 2 - 1 || !ok) continue;
                    ok = all(wait(&bar_h, n & 1)) && (n == 0 || all(wait(&bar_of, (n - 1) & 1)));
                    if (!ok) break;
                    tc_fence_after();
                    umma_product_w<false, false>(tO, tile(n * kPer + kA), blk, aState, DC * 128, DC, DB, false, issue);
                    umma_commit_w(&bar_o2, issue);
                }
                if (!ok) break;
                umma_commit_w(&bar_kv[n & 1], issue);
                if (!ENDS) {
                    if (!all(wait(&bar_p, n & 1)) || (steep && !all(wait(&bar_os, n & 1)))) break;
                    tc_fence_after();
#pragma unroll
                    for (int g = 0; g < 2; ++g)                    // of either warpgroup
                        umma_product_ts_w<true>(tO, tS + 64 * g, tile(n * kPer + kC) + g * kTokens * 64, blk, DC, kTokens / 2, true, issue);
                    umma_commit_w(&bar_o, issue);
                    umma_commit_w(&bar_c[n & 1], issue);
                }
                if (n + 1 < chunks && !scores(n + 1)) break;
            }
        umma_commit_w(&bar_end, issue);                           // leaves when its products have come to their end, whatever has expired
        mbar_drain(&bar_end, 0);
    } else if (lane == 0) {
        // ---------------------------------- loads ----------------------------------
        const int tiles = chunks * kPer;
        auto each_box = [&](int m, auto f) {
            const int j = m % kPer, width = j == kC ? DC : DB;
            const CUtensorMap* map = j == 0 ? &maps.b[walk] : j == kC ? &maps.c[walk] : &maps.a[walk];
            for (int blk = 0; blk < width / 64; ++blk) f(map, blk, hh * width + blk * 64, token0(m / kPer));
        };
        for (int m = 0; m < tiles; ++m, ++loads) {
            if (m >= kRing) {
                const int on = m / kPer - 2, j = m % kPer;
                if (!wait(ENDS || j == 0 ? &bar_kv[on & 1] : j == kC ? &bar_c[on & 1] : &bar_af[on & 1], (on >> 1) & 1)) break;
            }
            uint64_t* bar = &bar_full[m % kRing];
            mbar_expect_tx(bar, kTokens * (m % kPer == kC ? DC : DB) * 2);
            each_box(m, [&](const CUtensorMap* map, int blk, int x, int t0) { tma_load_3d(slot(m) + blk * kTokens * 128, map, x, t0, b, bar); });
            // what no buffer is free for yet comes to L2, once the first chunks are on their way (all of them at once: 6 us to the first product)
            if (m >= kPer && m + kRing < tiles)
                each_box(m + kRing, [&](const CUtensorMap* map, int, int x, int t0) { tma_prefetch_3d(map, x, t0, b); });
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (s_abort && loads) mbar_drain_ring(bar_full, kRing, loads);       // unless a wait has expired somebody has waited for every one
    if (s_abort) {                                             // nobody takes half a result for one: NaN, in either type
        auto spoil = [&](void* at, size_t words) {
#pragma unroll 1
            for (size_t i = tid; i < words; i += kTcThreads) static_cast<uint32_t*>(at)[i] = 0x7fff7fffu;
        };
        const size_t state = (size_t)DB * DC;
        if (ENDS) spoil(w.ends + ((size_t)bh * p.segments + segment) * state, state);
        else
#pragma unroll 1
            for (int t = first; t < end; ++t) spoil(static_cast<unsigned short*>(w.out) + (((size_t)b * p.T + t) * p.H + hh) * DC, DC / 2);
        if (!ENDS && last_one && w.sT) spoil(w.sT + (size_t)bh * state, state);
    }
    if (warp == 0) tmem_dealloc(tb, L::kColumns);
}

template <int DB, int DC, bool ENDS>
cudaError_t launch(LinearP p, int B, cudaStream_t stream) {
    LinearMaps m;
    for (int i = 0; i < p.walks; ++i) {
        const LinearWalk& w = p.w[i];
        if (!make_tmap_tokens(&m.b[i], w.b, B, p.T, p.H, DB, kTokens) || !make_tmap_tokens(&m.c[i], w.c, B, p.T, p.H, DC, kTokens)) return cudaErrorUnknown;
        if (!ENDS && (!make_tmap_tokens(&m.a[i], w.a, B, p.T, p.H, DB, kTokens) || !make_tmap_tokens(&m.out[i], w.out, B, p.T, p.H, DC, 32)))
            return cudaErrorUnknown;
    }
    const auto kern = k_linear_tc<DB, DC, ENDS>;
    const cudaError_t e = set_max_smem_once((const void*)kern, TcLinear<DB, DC, ENDS>::kSmem);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kern, dim3((unsigned)(p.BH * p.segments * p.walks)), dim3(kTcThreads), TcLinear<DB, DC, ENDS>::kSmem, stream, m, p);
}
template <bool ENDS>
cudaError_t launch(const LinearP& p, int db, int dc, int B, cudaStream_t stream) {
    if (db == 128) return dc == 128 ? launch<128, 128, ENDS>(p, B, stream) : launch<128, 64, ENDS>(p, B, stream);
    return dc == 128 ? launch<64, 128, ENDS>(p, B, stream) : launch<64, 64, ENDS>(p, B, stream);
}

}  // namespace

cudaError_t linear_tc(const LinearP& p, int db, int dc, cudaStream_t stream) {
    return p.w[0].out ? launch<false>(p, db, dc, p.BH / p.H, stream) : launch<true>(p, db, dc, p.BH / p.H, stream);
}

}  // namespace qd

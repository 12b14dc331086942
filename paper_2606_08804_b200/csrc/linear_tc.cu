// Linear attention in bf16 on the tensor cores: a walk (linear.cuh) over chunks of 128 tokens to a CTA, every product a tcgen05.mma:
//     P = (a b^T) o D  (rounded to bf16 as the next operand)      out = P c + rho (a S)      S <- e^{g n} S + (kappa b)^T c
// The state stays in fp32 registers; each chunk's sum comes from tensor memory and is added there (the tensor cores cut as they accumulate).
// For a S it goes to shared memory in bf16.  kappa b is three bf16 planes, which hold all of its 24 bits: with two the state is 2.4e-6 of its
// length off, which is half of what a whole fp32 sum over a sequence is allowed to be.
//
// Bound by HBM: per token and head two tensors of its width in and one out besides c, 2.5 us a chunk of 128 x 128 with 128 CTAs; the products of
// a chunk are 3072 cycles.  So a chunk's steps need not overlap perfectly, only loads must never stop: five (six) tile buffers, in each of
// which b, a and c of the chunks follow one another, and out leaves through a's.  The first plane takes b's place, the others of 32 tokens at a
// time go through two buffers.
//   warps 0-3    P: row r = lane, from tensor memory and back to it as an operand
//   warps 4-7    the planes of kappa b, then out: 32 rows each, staged in a's tile, stored by TMA
//   warps 8-15   state: a row to a lane, half of the columns to a warpgroup
//   warp 16      issues the products;  warp 17  loads
// All waits are bounded; on expiry the status word says so, everybody leaves, what is in flight is waited for.
#include "linear.cuh"

namespace qd {
namespace {
using namespace sm100;

constexpr int kTokens = 128, kPart = 32, kParts = kTokens / kPart, kTcThreads = 18 * 32;

// The upper halves of eight fp32 values as packed bf16; what they leave stays behind, exactly.
__device__ __forceinline__ uint4 upper8(float (&x)[8]) {
    uint32_t r[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t lo = __float_as_uint(x[2 * e]), hi = __float_as_uint(x[2 * e + 1]) & 0xffff0000u;
        r[e] = lo >> 16 | hi;
        x[2 * e] -= __uint_as_float(lo & 0xffff0000u);
        x[2 * e + 1] -= __uint_as_float(hi);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

struct LinearMaps { CUtensorMap a[kLinearWalks], b[kLinearWalks], c[kLinearWalks], out[kLinearWalks]; };

template <int DB, int DC, bool ENDS>
struct TcLinear {
    static constexpr int kSlot = kTokens * (DB > DC ? DB : DC) * 2;
    static constexpr int kRing = ENDS ? 4 : DB == 128 ? 5 : 6;        // at most two chunks ahead: barriers of chunks n and n + 2 are the same
    static constexpr int kPer = ENDS ? 2 : 3;                         // tiles of a chunk: b, a, c
    static constexpr int kState = ENDS ? 0 : DB * DC * 2, kPlane = kPart * DB * 2, kRest = 4 * kPlane;
    static constexpr int kOffRest = kState, kOffRing = kOffRest + kRest, kSmem = kOffRing + kRing * kSlot + 1024;
    static constexpr int kColumns = ENDS ? DC : 512;
    static_assert(kSmem <= 232448 - 1024, "shared memory");
};

template <int DB, int DC, bool ENDS>
__global__ void __launch_bounds__(kTcThreads, 1) k_linear_tc(const __grid_constant__ LinearMaps maps, const LinearP p) {
    typedef TcLinear<DB, DC, ENDS> L;
    constexpr int kRing = L::kRing, kPer = L::kPer, kA = 1, kC = kPer - 1;
    extern __shared__ unsigned char smem_raw[];
    unsigned char* smem = (unsigned char*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    unsigned char *sState = smem, *sRest = smem + L::kOffRest, *sRing = smem + L::kOffRing;
    // bar_s, bar_o, bar_kv, bar_kq: products complete; bar_p, bar_k, bar_h: operands in place; bar_of: out's accumulators have been
    // read; bar_af: a's tile is free.  Where one side runs up to two phases ahead there is one for even and one for odd phases.
    __shared__ uint64_t bar_full[kRing], bar_s, bar_o, bar_kv[2], bar_kq[2], bar_p, bar_k[2], bar_h, bar_of, bar_af[2], bar_end;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int s_abort;
    __shared__ float s_d[2 * kTokens];                                    // D(|m|), m from -128

    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, wq = warp & 3;
    const int walk = blockIdx.x % p.walks, cta = blockIdx.x / p.walks, segment = cta % p.segments, bh = cta / p.segments;
    const int b = bh / p.H, hh = bh % p.H;
    const LinearWalk& w = p.w[walk];
    const bool reverse = w.reverse;
    const int first = segment * p.length, end = min(p.T, first + p.length), chunks = (end - first + kTokens - 1) / kTokens;
    auto token0 = [&](int n) { return first + (reverse ? chunks - 1 - n : n) * kTokens; };

    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(&bar_full[i], 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&bar_kq[i], 1); mbar_init(&bar_k[i], 4); mbar_init(&bar_af[i], 4); }
        mbar_init(&bar_s, 1); mbar_init(&bar_o, 1); mbar_init(&bar_p, 4); mbar_init(&bar_h, 8); mbar_init(&bar_of, 4);
        mbar_init(&bar_end, 1);
        mbar_init_fence();
        s_abort = 0;
    }
    if (warp == 0) { tmem_alloc(&tmem_slot, L::kColumns); tmem_relinquish(); }
    grid_dep_wait();
    grid_dep_launch();
    const float g2 = p.g[hh] * 1.4426950408889634f;
    if (tid < 2 * kTokens) s_d[tid] = p.scale * decay_power(g2, abs(tid - kTokens));
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tb = uniform(tmem_slot);
    const uint32_t tS = tb, tO1 = tb + 128, tO2 = tO1 + DC, tKV = ENDS ? tb : tO2 + DC;
    const uint32_t lanes = (uint32_t)wq * 32;

    auto wait = [&](uint64_t* bar, uint32_t parity) { return mbar_try_wait(bar, parity) || wait_on(bar, parity, s_abort, p.status); };
    auto all = [&](bool ok) { return __all_sync(0xffffffffu, ok) != 0; };
    auto arrive = [&](uint64_t* bar) { __syncwarp(); if (lane == 0) mbar_arrive(bar); };
    auto slot = [&](int m) { return sRing + m % kRing * L::kSlot; };
    auto full = [&](int m) { return wait(&bar_full[m % kRing], (m / kRing) & 1); };

    int loads = 0;                                                        // issued by this thread
    if (p.clear && blockIdx.x == 0 && tid == 0) *p.status = 0;
    if (ENDS && segment == (reverse ? 0 : p.segments - 1)) {
        // nobody begins with the sums of this one
    } else if (warp < 4) {
        // ---------------------------------- weights ----------------------------------
        const float* far = s_d + kTokens + lanes + lane;
        for (int n = 0; n < chunks && !ENDS; ++n) {
            if (!all(wait(&bar_s, n & 1))) break;
            tc_fence_after();
#pragma unroll
            for (int j = 0; j < 4; ++j) {                          // 32 columns i, which become 16 packed ones in the place of what has been read
                uint32_t o[16];
                if (reverse ? j >= wq : j <= wq) {
                    float v[32];
                    tmem_ld32(tmem_addr(tS, lanes, 32 * j), v);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] *= far[-32 * j - e];
                    if (j == wq)                                   // an infinite product past the diagonal leaves nothing either
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = (reverse ? e >= lane : e <= lane) ? v[e] : 0.f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = pack_bf16(v[2 * e], v[2 * e + 1]);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[e] = 0;
                }
                tmem_st8(tmem_addr(tS, lanes, 16 * j), o);
                tmem_st8(tmem_addr(tS, lanes, 16 * j + 8), o + 8);
            }
            tmem_st_wait();
            tc_fence_before();
            arrive(&bar_p);
        }
    } else if (warp < 8) {
        // ---------------------------------- planes and output ----------------------------------
        const int r = (int)lanes + lane;
        int stored = -1;                                           // chunk whose output this thread has stored and not seen read
        for (int n = 0; n < chunks; ++n) {
            const int t0 = token0(n), live = min(kTokens, end - t0);
            // b has been multiplied with a: its rows times kappa, a row to a lane, a quarter of the columns to a warp
            if (!ENDS && !all(wait(&bar_s, n & 1))) break;
            if (!all(full(n * kPer))) break;
            bool ok = true;
            for (int q = 0; q < kParts && ok; ++q) {
                const int i = n * kParts + q, row = q * kPart + lane;
                if (q == 1 && stored >= 0) {                       // the output of the chunk before has been read by now: its tile is free
                    tma_store_wait_read();
                    mbar_arrive(&bar_af[stored & 1]);
                    stored = -1;
                }
                if (i >= 2) ok = all(wait(&bar_kq[i & 1], ((i - 2) >> 1) & 1));
                const float kappa = row >= live ? 0.f : reverse ? p.scale * decay_power(g2, row + 1) : decay_power(g2, live - 1 - row);
                unsigned char *tile = slot(n * kPer), *rest = sRest + (i & 1) * 2 * L::kPlane;
#pragma unroll
                for (int k = 0; k < DB / 32; ++k) {
                    const int ch = wq * (DB / 32) + k, blk = ch >> 3;
                    const uint32_t off = sw128_chunk(row, ch & 7), part = sw128_chunk(lane, ch & 7) + blk * kPart * 128;
                    unsigned char* at = tile + blk * kTokens * 128 + off;
                    const uint4 raw = *reinterpret_cast<const uint4*>(at);
                    const uint32_t in[4] = {raw.x, raw.y, raw.z, raw.w};
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[2 * e] = kappa * __uint_as_float(in[e] << 16);
                        x[2 * e + 1] = kappa * __uint_as_float(in[e] & 0xffff0000u);
                    }
                    // cut to 8 bits, three times: nothing is left of 24
                    sts128(at, upper8(x));
                    sts128(rest + part, upper8(x));
                    sts128(rest + L::kPlane + part, upper8(x));
                }
                fence_proxy_async();
                arrive(&bar_k[i & 1]);
            }
            if (!ok) break;
            if (ENDS) continue;
            const float rho = r >= live ? 0.f : reverse ? decay_power(g2, live - 1 - r) : p.scale * decay_power(g2, r + 1);
            if (!all(wait(&bar_o, n & 1))) break;
            tc_fence_after();
            unsigned char* stage = slot(n * kPer + kA);
#pragma unroll
            for (int j = 0; j < DC / 16; ++j) {
                float x[16], y[16];
                tmem_ld16(tmem_addr(tO1, lanes, 16 * j), x);
                tmem_ld16(tmem_addr(tO2, lanes, 16 * j), y);
                tmem_ld_wait();
                if (j == DC / 16 - 1) { tc_fence_before(); arrive(&bar_of); }
#pragma unroll
                for (int e = 0; e < 16; ++e) x[e] = fmaf(rho, y[e], x[e]);
#pragma unroll
                for (int ch = 0; ch < 2; ++ch)
                    sts128(stage + (j >> 2) * kTokens * 128 + sw128_chunk(r, (j & 3) * 2 + ch), pack8(x + 8 * ch));
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (t0 + (int)lanes < p.T) {                       // rows past the end of the sequence are skipped
#pragma unroll
                    for (int blk = 0; blk < DC / 64; ++blk)
                        tma_store_3d(&maps.out[walk], stage + blk * kTokens * 128 + lanes * 128, hh * DC + blk * 64, t0 + (int)lanes, b);
                    tma_store_commit();
                }
                stored = n;
            }
            __syncwarp();
        }
        if (lane == 0) tma_store_wait_all();
    } else if (warp < 16) {
        // ---------------------------------- state ----------------------------------
        constexpr int HC = DC / 2, size = DB * DC;
        // 64-row products put 16 rows on each of a warpgroup's four warps
        const int r = DB == 128 ? (int)lanes + lane : 16 * wq + (lane & 15), c0 = (warp - 8) / 4 * HC;
        const bool live_row = DB == 128 || lane < 16;
        float h[HC];
        auto place = [&](int i) { return w.flip ? (c0 + i) * DB + r : r * DC + c0 + i; };
        const float* entry = !ENDS && w.s0 && live_row ? w.s0 + ((size_t)bh * p.segments + segment) * size : nullptr;
        if (entry && !w.flip) {
#pragma unroll
            for (int i = 0; i < HC; i += 4) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(entry + place(i)));
                h[i] = t.x; h[i + 1] = t.y; h[i + 2] = t.z; h[i + 3] = t.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < HC; ++i) h[i] = entry ? __ldcg(entry + place(i)) : 0.f;
        }
        auto put = [&]() {
            if (!ENDS && live_row)
#pragma unroll
                for (int ch = 0; ch < HC / 8; ++ch)
                    sts128(sState + (c0 + 8 * ch) / 64 * (DB * 128) + sw128_chunk(r, ((c0 >> 3) + ch) & 7), pack8(h + 8 * ch));
            fence_proxy_async();
            arrive(&bar_h);
        };
        put();
        for (int n = 0; n < chunks; ++n) {
            if (!all(wait(&bar_kv[n & 1], (n >> 1) & 1))) break;
            tc_fence_after();
            const float keep = decay_power(g2, min(kTokens, end - token0(n)));
#pragma unroll
            for (int j = 0; j < HC / 16; ++j) {
                float v[16];
                tmem_ld16(tmem_addr(tKV, lanes, c0 + 16 * j), v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) h[16 * j + e] = fmaf(keep, h[16 * j + e], v[e]);
            }
            tc_fence_before();
            if (n + 1 < chunks) put();
        }
        float* left = ENDS ? w.ends + ((size_t)bh * p.segments + segment) * size
                           : segment == (reverse ? 0 : p.segments - 1) && w.sT ? w.sT + (size_t)bh * size : nullptr;
        if (left && live_row && !s_abort) {
            if (!w.flip) {
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
        const uint32_t aState = smem_u32(sState), aRest = smem_u32(sRest), aRing = smem_u32(sRing);
        auto tile = [&](int m) { return aRing + (uint32_t)(m % kRing) * L::kSlot; };
        constexpr uint32_t blk = kTokens * 128;
        auto scores = [&](int n) {
            if (ENDS) return true;
            if (!all(full(n * kPer) && full(n * kPer + kA))) return false;
            umma_product_w<false, false>(tS, tile(n * kPer + kA), blk, tile(n * kPer), blk, kTokens, DB, false, issue);
            umma_commit_w(&bar_s, issue);
            return true;
        };
        for (int n = 0; n < chunks; ++n) {
            const uint32_t tB = tile(n * kPer), tA = tile(n * kPer + kA), tC = tile(n * kPer + kC);
            if (n == 0 && !scores(0)) break;
            if (!all(wait(&bar_h, n & 1))) break;
            tc_fence_after();
            if (!ENDS) {
                if (n > 0 && !all(wait(&bar_of, (n - 1) & 1))) break;
                tc_fence_after();
                umma_product_w<false, true>(tO2, tA, blk, aState, DB * 128, DC, DB, false, issue);
            }
            if (!all(full(n * kPer + kC))) break;
            bool ok = true;
#pragma unroll
            for (int q = 0; q < kParts; ++q) {
                if (!ENDS && q == kParts / 2) {                   // the weights have been made beside the first two parts
                    ok = ok && all(wait(&bar_p, n & 1));
                    if (!ok) break;
                    tc_fence_after();
                    umma_product_ts_w<true>(tO1, tS, tC, blk, DC, kTokens, false, issue);
                    umma_commit_w(&bar_o, issue);
                    ok = n + 1 == chunks || scores(n + 1);        // its weights are made beside the rest of this one
                }
                const int i = n * kParts + q;
                ok = ok && all(wait(&bar_k[i & 1], (i >> 1) & 1));
                if (!ok) break;
                tc_fence_after();
                const uint32_t rest = aRest + (uint32_t)(i & 1) * 2 * L::kPlane, line = q * kPart * 128;
                umma_product_w<true, true, DB>(tKV, tB + line, blk, tC + line, blk, DC, kPart, q > 0, issue);
                umma_product_w<true, true, DB>(tKV, rest, kPart * 128, tC + line, blk, DC, kPart, true, issue);
                umma_product_w<true, true, DB>(tKV, rest + L::kPlane, kPart * 128, tC + line, blk, DC, kPart, true, issue);
                umma_commit_w(&bar_kq[i & 1], issue);
            }
            if (!ok) break;
            umma_commit_w(&bar_kv[n & 1], issue);
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
        // what no buffer is free for yet comes to L2 two chunks ahead
        constexpr int kAhead = 2 * kPer;
        auto prefetch = [&](int m) { each_box(m, [&](const CUtensorMap* map, int, int x, int t0) { tma_prefetch_3d(map, x, t0, b); }); };
        for (int m = kRing; m < kAhead && m < tiles; ++m) prefetch(m);
        for (int m = 0; m < tiles; ++m, ++loads) {
            if (m + kAhead < tiles) prefetch(m + kAhead);
            if (m >= kRing) {
                const int old = m - kRing, on = old / kPer;
                uint64_t* bar = !ENDS && old % kPer == kA ? &bar_af[on & 1] : &bar_kv[on & 1];
                if (!wait(bar, (on >> 1) & 1)) break;
            }
            uint64_t* bar = &bar_full[m % kRing];
            mbar_expect_tx(bar, kTokens * (m % kPer == kC ? DC : DB) * 2);
            each_box(m, [&](const CUtensorMap* map, int blk, int x, int t0) { tma_load_3d(slot(m) + blk * kTokens * 128, map, x, t0, b, bar); });
        }
    }
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    if (s_abort && loads) mbar_drain_ring(bar_full, kRing, loads);       // unless a wait has expired somebody has waited for every one
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

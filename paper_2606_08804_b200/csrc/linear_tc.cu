// Linear attention in bf16 on the tensor cores: a walk (linear.cuh) over chunks of 128 tokens to a CTA, every product a tcgen05.mma:
//     P = (a b^T) o D  (rounded to bf16 as the next operand)      out = P c + rho (a S)      S <- e^{g n} S + (kappa b)^T c
// The state stays in fp32 registers; each chunk's sum comes from tensor memory and is added there (the tensor cores cut as they
// accumulate).  For a S it goes to shared memory in bf16; kappa b goes there in two bf16 planes, so that the state has 16 bits of every term.
//
// Bound by HBM: per token and head two tensors of its width in and one out besides c, 2.5 us a chunk of 128 x 128 with 128 CTAs; the five products of
// a chunk are 2560 cycles.  So a chunk's steps need not overlap perfectly, only loads must never stop: five (six) tile buffers, in each of
// which b, a and c of the chunks follow one another, and out leaves through a's.
//   warps 0-3    P: row r = lane, from tensor memory and back to it as an operand; then kappa b in place and its rest
//   warps 4-7    out: 32 rows each, staged in a's tile, stored by TMA
//   warps 8-15   state: a row to a lane, half of the columns to a warpgroup
//   warp 16      issues the products;  warp 17  loads
// All waits are bounded; on expiry the status word says so, everybody leaves, what is in flight is waited for.
#include "linear.cuh"

namespace qd {
namespace {
using namespace sm100;

constexpr int kTokens = 128, kTcThreads = 18 * 32;

struct LinearMaps { CUtensorMap a[kLinearWalks], b[kLinearWalks], c[kLinearWalks], out[kLinearWalks]; };

template <int DB, int DC, bool ENDS>
struct TcLinear {
    static constexpr int kSlot = kTokens * (DB > DC ? DB : DC) * 2;
    static constexpr int kRing = ENDS ? 4 : DB == 128 ? 5 : 6;        // at most two chunks ahead: barriers of chunks n and n + 2 are the same
    static constexpr int kPer = ENDS ? 2 : 3;                         // tiles of a chunk: b, a, c
    static constexpr int kState = ENDS ? 0 : DB * DC * 2, kRest = kTokens * DB * 2;
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
    // bar_s, bar_o, bar_kv: products complete; bar_p, bar_k, bar_h: operands in place; bar_of: out's accumulators have been read;
    // bar_af: a's tile is free.  bar_kv and bar_af have one for even and one for odd chunks, since the loads run up to two ahead.
    __shared__ uint64_t bar_full[kRing], bar_s, bar_o, bar_kv[2], bar_p, bar_k, bar_h, bar_of, bar_af[2], bar_end;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int s_abort;
    __shared__ float s_d[kTokens];

    const int tid = threadIdx.x, warp = warp_index(), lane = tid & 31, wq = warp & 3;
    const int walk = blockIdx.x % p.walks, cta = blockIdx.x / p.walks, segment = cta % p.segments, bh = cta / p.segments;
    const int b = bh / p.H, hh = bh % p.H;
    const LinearWalk& w = p.w[walk];
    const bool reverse = w.reverse;
    const int first = segment * p.length, end = min(p.T, first + p.length), chunks = (end - first + kTokens - 1) / kTokens;
    auto token0 = [&](int n) { return first + (reverse ? chunks - 1 - n : n) * kTokens; };

    if (tid == 0) {
        for (int i = 0; i < kRing; ++i) mbar_init(&bar_full[i], 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_kv[i], 1); mbar_init(&bar_af[i], 4); }
        mbar_init(&bar_s, 1); mbar_init(&bar_o, 1); mbar_init(&bar_p, 4); mbar_init(&bar_k, 4); mbar_init(&bar_h, 8); mbar_init(&bar_of, 4);
        mbar_init(&bar_end, 1);
        mbar_init_fence();
        s_abort = 0;
    }
    if (warp == 0) { tmem_alloc(&tmem_slot, L::kColumns); tmem_relinquish(); }
    grid_dep_wait();
    grid_dep_launch();
    const float g2 = p.g[hh] * 1.4426950408889634f;
    if (tid < kTokens) s_d[tid] = p.scale * decay_power(g2, tid);
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
        // ---------------------------------- weights and scaled rows ----------------------------------
        const int r = (int)lanes + lane;
        for (int n = 0; n < chunks; ++n) {
            const int live = min(kTokens, end - token0(n));
            if (!ENDS) {
                if (!all(wait(&bar_s, n & 1))) break;
                tc_fence_after();
#pragma unroll
                for (int j = 0; j < 4; ++j) {                      // 32 columns i, which become 16 packed ones in the place of what has been read
                    uint32_t o[16];
                    if (reverse ? j >= wq : j <= wq) {
                        float v[32];
                        tmem_ld32(tmem_addr(tS, lanes, 32 * j), v);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 32; ++e) {
                            const int u = reverse ? 32 * j + e - r : r - 32 * j - e;
                            v[e] = u >= 0 ? v[e] * s_d[u & (kTokens - 1)] : 0.f;
                        }
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
            } else if (n > 0 && !all(wait(&bar_kv[(n - 1) & 1], ((n - 1) >> 1) & 1))) {
                break;
            }
            // the product with b has been taken (there is none in ENDS): its rows times kappa, and what bf16 leaves of them
            if (!all(full(n * kPer))) break;
            const float kappa = r >= live ? 0.f : reverse ? p.scale * decay_power(g2, r + 1) : decay_power(g2, live - 1 - r);
            unsigned char *tile = slot(n * kPer), *rest = sRest;
#pragma unroll
            for (int blk = 0; blk < DB / 64; ++blk, tile += kTokens * 128, rest += kTokens * 128)
#pragma unroll 4
                for (int ch = 0; ch < 8; ++ch) {
                    const uint32_t off = sw128_chunk(r, ch);
                    float x[8], y[8];
                    load8(tile + off, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] *= kappa;
                    const uint4 hi = pack8(x);
                    const uint32_t h[4] = {hi.x, hi.y, hi.z, hi.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        y[2 * e] = x[2 * e] - __uint_as_float(h[e] << 16);
                        y[2 * e + 1] = x[2 * e + 1] - __uint_as_float(h[e] & 0xffff0000u);
                    }
                    sts128(tile + off, hi);
                    sts128(rest + off, pack8(y));
                }
            fence_proxy_async();
            arrive(&bar_k);
        }
    } else if (warp < 8) {
        // ---------------------------------- output ----------------------------------
        const int r = (int)lanes + lane;
        for (int n = 0; n < chunks && !ENDS; ++n) {
            const int t0 = token0(n), live = min(kTokens, end - t0);
            const float rho = r >= live ? 0.f : reverse ? decay_power(g2, live - 1 - r) : p.scale * decay_power(g2, r + 1);
            if (!all(wait(&bar_o, n & 1))) break;
            tc_fence_after();
            unsigned char* stage = slot(n * kPer + kA);
#pragma unroll
            for (int j = 0; j < DC / 32; ++j) {
                float x[32], y[32];
                tmem_ld32(tmem_addr(tO1, lanes, 32 * j), x);
                tmem_ld32(tmem_addr(tO2, lanes, 32 * j), y);
                tmem_ld_wait();
                if (j == DC / 32 - 1) { tc_fence_before(); arrive(&bar_of); }
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] = fmaf(rho, y[e], x[e]);
#pragma unroll
                for (int ch = 0; ch < 4; ++ch)
                    sts128(stage + (j >> 1) * kTokens * 128 + sw128_chunk(r, (j & 1) * 4 + ch), pack8(x + 8 * ch));
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                if (t0 + (int)lanes < p.T) {                       // rows past the end of the sequence are skipped
#pragma unroll
                    for (int blk = 0; blk < DC / 64; ++blk)
                        tma_store_3d(&maps.out[walk], stage + blk * kTokens * 128 + lanes * 128, hh * DC + blk * 64, t0 + (int)lanes, b);
                    tma_store_commit();
                    tma_store_wait_read();
                }
                mbar_arrive(&bar_af[n & 1]);
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
#pragma unroll
        for (int i = 0; i < HC; ++i) h[i] = !ENDS && live_row ? linear_entry(p, w, bh, segment, size, place(i), g2) : 0.f;
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
            for (int j = 0; j < HC / 32; ++j) {
                float v[32];
                tmem_ld32(tmem_addr(tKV, lanes, c0 + 32 * j), v);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) h[32 * j + e] = fmaf(keep, h[32 * j + e], v[e]);
            }
            tc_fence_before();
            if (n + 1 < chunks) put();
        }
        float* left = ENDS ? w.ends + ((size_t)bh * p.segments + segment) * size
                           : segment == (reverse ? 0 : p.segments - 1) && w.sT ? w.sT + (size_t)bh * size : nullptr;
        if (left && live_row && !s_abort)
#pragma unroll
            for (int i = 0; i < HC; ++i) left[place(i)] = h[i];
    } else if (warp == 16) {
        // ---------------------------------- products, by the converged warp ----------------------------------
        const uint32_t issue = elect_lane();
        const uint32_t aState = smem_u32(sState), aRest = smem_u32(sRest), aRing = smem_u32(sRing);
        auto tile = [&](int m) { return aRing + (uint32_t)(m % kRing) * L::kSlot; };
        for (int n = 0; n < chunks; ++n) {
            const uint32_t tB = tile(n * kPer), tA = tile(n * kPer + kA), tC = tile(n * kPer + kC);
            constexpr uint32_t blk = kTokens * 128;
            if (!ENDS) {
                if (!all(full(n * kPer) && full(n * kPer + kA))) break;
                umma_product_w<false, false>(tS, tA, blk, tB, blk, kTokens, DB, false, issue);
                umma_commit_w(&bar_s, issue);
            }
            if (!all(wait(&bar_h, n & 1))) break;
            tc_fence_after();
            if (!ENDS) {
                if (n > 0 && !all(wait(&bar_of, (n - 1) & 1))) break;
                tc_fence_after();
                umma_product_w<false, true>(tO2, tA, blk, aState, DB * 128, DC, DB, false, issue);
            }
            if (!all(full(n * kPer + kC))) break;
            if (!ENDS) {
                if (!all(wait(&bar_p, n & 1))) break;
                tc_fence_after();
                umma_product_ts_w<true>(tO1, tS, tC, blk, DC, kTokens, false, issue);
                umma_commit_w(&bar_o, issue);
            }
            if (!all(wait(&bar_k, n & 1))) break;
            tc_fence_after();
            umma_product_w<true, true, DB>(tKV, tB, blk, tC, blk, DC, kTokens, false, issue);
            umma_product_w<true, true, DB>(tKV, aRest, blk, tC, blk, DC, kTokens, true, issue);
            umma_commit_w(&bar_kv[n & 1], issue);
        }
        umma_commit_w(&bar_end, issue);                           // leaves when its products have come to their end, whatever has expired
        mbar_drain(&bar_end, 0);
    } else if (lane == 0) {
        // ---------------------------------- loads ----------------------------------
        const int tiles = chunks * kPer;
        for (int m = 0; m < tiles; ++m, ++loads) {
            if (m >= kRing) {
                const int old = m - kRing, on = old / kPer;
                uint64_t* bar = !ENDS && old % kPer == kA ? &bar_af[on & 1] : &bar_kv[on & 1];
                if (!wait(bar, (on >> 1) & 1)) break;
            }
            const int n = m / kPer, j = m % kPer, t0 = token0(n);
            const CUtensorMap* map = j == 0 ? &maps.b[walk] : j == kC ? &maps.c[walk] : &maps.a[walk];
            const int width = j == kC ? DC : DB;
            uint64_t* bar = &bar_full[m % kRing];
            mbar_expect_tx(bar, kTokens * width * 2);
            for (int blk = 0; blk < width / 64; ++blk) tma_load_3d(slot(m) + blk * kTokens * 128, map, hh * width + blk * 64, t0, b, bar);
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

// Layer norm (norm.cu) together with what stands beside it in a layer:
//   gated    y = ((x - m) r w + b) f(z),  f = SiLU or the logistic function             (a read-out per head)
//            dn = dy f, dz = dy ((x - m) r w + b) f'(z), then as a norm's backward with dn for dy
//   added    t = e + s x (residual and scale),  y = (t - m) r w + b                      (the residual stream)
//            d = norm's backward of dy at t, + dt;  de = d, dx = s d, ds = sum_rows d x    (t added up again: rounded to bf16 it costs dw, an
//            fp32 sum of terms of both signs, 1.6e-3 of its length)
// Backward of the norm, with g = dy w and x^ = (x - m) r:  dx = r (g - x^ mean(g x^) - mean(g))  (the last term not without the mean),
// dw = sum_rows dy x^, db = sum_rows dy.
//
// Bound by HBM, so the plan of a row decides:
//   k_fused_fwd, _bwd   rows of whole 16-byte (or 4-byte) groups: a row belongs to 2^k lanes or to a CTA and is in registers when its sums are taken; what
//                       the next rows need is on its way to shared memory, where each thread reads back only what it asked for (no barrier).
//                       CTAs stay; backward the sums over rows stay in registers, one partial per CTA, added up in a fixed order.
//   k_odd_fwd, _bwd     bf16 rows of an odd width, which begin anywhere: blocks of rows come to shared memory as the aligned 16-byte pieces that they lie in, and
//                       are read from there one element at a time, neighbouring columns to neighbouring lanes.
//   k_wide_sums, _cols  backward of rows too wide for registers: the sums of a row first, then everything else with a thread to a column
//                       and the rows in a loop, whose sums over rows need no more than the registers of one column.  Inputs are read twice.
#include "rows.cuh"

namespace qd {
namespace {

struct FusedP {
    long long rows;
    int width;
    const void *x, *e, *scale, *weight, *bias, *dy, *dt;      // e: gate or residual
    void *y, *t, *dx, *de;
    float* stats;                                              // [2][rows]: mean, r
    float* part;                                               // backward: [parts][sums][width]
    float* rowsum;                                             // wide backward: [2][rows]: mean(g x^), mean(g)
    float eps, inv;
    int step;                                                  // odd rows: rows that a group of lanes takes of a block; wide: rows of a CTA
    bool rms, silu;
};
constexpr __host__ __device__ int fused_threads(int tpr) { return tpr > 256 ? tpr : 256; }
constexpr __host__ __device__ int fused_sums(bool added) { return added ? 3 : 2; }

// sums over the TPR threads of a row, the same bits in each; as in norm.cu
template <int TPR, int M>
__device__ __forceinline__ void row_sum(float (&v)[M], float (*red)[M][32], int& turn) {
#pragma unroll
    for (int w = (TPR < 32 ? TPR : 32) / 2; w > 0; w >>= 1)
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], w);
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0)
#pragma unroll
            for (int m = 0; m < M; ++m) red[turn][m][threadIdx.x >> 5] = v[m];
        __syncthreads();
        const int first = threadIdx.x / TPR * (TPR / 32);
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = red[turn][m][first + threadIdx.x % (TPR / 32)];
        turn ^= 1;
#pragma unroll
        for (int w = TPR / 64; w > 0; w >>= 1)
#pragma unroll
            for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], w);
    }
}
// the gate and its slope
__device__ __forceinline__ float gate_value(float z, bool silu) { const float s = gate_sigmoid(z); return silu ? z * s : s; }
__device__ __forceinline__ float2 gate_slope(float z, bool silu) {
    const float s = gate_sigmoid(z);
    return silu ? make_float2(z * s, s * fmaf(z, 1.f - s, 1.f)) : make_float2(s, s * (1.f - s));
}
// One element backward.  `in`: x, gate or residual, dy, dtotal.  Leaves x^ and g; adds to the row's sums and, where `cols`, to dw and db.
template <bool ADDED>
__device__ __forceinline__ void element(const FusedP& p, const float (&in)[4], float w, float v, float mean, float r, float& xh, float& g, float& dz,
                                        float (&s)[2], float* dw, float* db) {
    float x = in[0], d = in[2];
    if (ADDED) x = p.scale ? fmaf(v, x, in[1]) : x + in[1];
    xh = (x - mean) * r;
    if (!ADDED) {
        const float2 f = gate_slope(in[1], p.silu);
        dz = d * fmaf(xh, w, p.bias ? v : 0.f) * f.y;
        d *= f.x;
    }
    g = d * w;
    s[0] = fmaf(g, xh, s[0]);
    s[1] += g;
    if (dw) { *dw = fmaf(d, xh, *dw); *db += d; }
}

// ---- rows of whole groups -----------------------------------------------------------------------------------------------------
// A thread's K groups of STREAMS rows, DEPTH rows ahead: one forward (with three, 262144 x 128 gated takes 36.2 us for 33.6, added 54.6 for
// 49.8), three backward, where few threads have room (two gated rows ahead in registers instead: 74.7 for 64.7).
constexpr int depth_of(int stage, bool bwd) { return !bwd ? 1 : 3 * stage <= 49152 ? 3 : 2 * stage <= 65536 ? 2 : 1; }
template <typename IO, int V, int K, int TPR, int STREAMS, bool BWD>
struct Ahead {
    static constexpr int NT = fused_threads(TPR), B = V * sizeof(IO), kStage = STREAMS * K * NT * B, DEPTH = depth_of(kStage, BWD), kBytes = DEPTH * kStage;
    static_assert(B == 16 || B == 4, "what copies take");
    unsigned char* mine;
    __device__ __forceinline__ explicit Ahead(unsigned char* smem) : mine(smem + threadIdx.x * B) {}
    __device__ __forceinline__ unsigned char* at(int stage, int stream, int k) const { return mine + ((stage * STREAMS + stream) * K + k) * (NT * B); }
    __device__ __forceinline__ void fetch(int stage, const void* const (&src)[STREAMS], long long row, int width, bool live) const {
#pragma unroll
        for (int m = 0; m < STREAMS; ++m)
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + threadIdx.x % TPR) * V;
                const bool in = live && c < width && src[m];
                copy_bytes<B>(at(stage, m, k), in ? static_cast<const IO*>(src[m]) + row * width + c : static_cast<const IO*>(src[0]), in ? B : 0);
            }
        copy_commit();
    }
    __device__ __forceinline__ Pack<IO, V> take(int stage, int stream, int k) const {
        Pack<IO, V> r;
        if constexpr (B == 16) {
            const uint4 u = *reinterpret_cast<const uint4*>(at(stage, stream, k));
            r.w[0] = u.x; r.w[1] = u.y; r.w[2] = u.z; r.w[3] = u.w;
        } else {
            r.w[0] = *reinterpret_cast<const uint32_t*>(at(stage, stream, k));
        }
        return r;
    }
};
// CTAs to an SM that the registers are shared out for.  bf16 forward, 262144 x 128: gated 33.3 us with three (35.5 with two, 40.4 with four),
// added, which writes as much as it reads, 44.3 with two (49.5, 54.2); backward 63.8 and 67.6 with two (70.8 and 84.0 with three).
constexpr __host__ __device__ int fused_resident(int k, int v, int tpr, bool bwd, bool added) {
    return tpr > 256 ? (k * v <= 16 && !bwd ? 2 : 1) : bwd ? (k * v <= 8 ? 2 : 1) : (k * v <= 8 ? 4 : k * v <= 16 ? (added ? 2 : 3) : 1);
}

template <typename IO, int V, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR), fused_resident(K, V, TPR, false, ADDED)) k_fused_fwd(const FusedP p) {
    constexpr int NT = fused_threads(TPR), RPC = NT / TPR;
    constexpr bool HELD = K * V <= 16;                       // scale, weight and bias stay in registers
    extern __shared__ __align__(16) unsigned char smem_rows[];
    __shared__ float red[2][1][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long row = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    int turn = 0, stage = 0;
    typedef Ahead<IO, V, K, TPR, 2, false> Rows;
    constexpr int DEPTH = Rows::DEPTH;
    const Rows ahead(smem_rows);
    const void* const src[2] = {p.x, p.e};
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) ahead.fetch(d, src, row + d * step, p.width, row + d * step < p.rows);
    auto param = [&](const void* base, int c) { return load_pack<IO, V>(static_cast<const IO*>(base) + c, V, true); };
    Pack<IO, V> ps[HELD && ADDED ? K : 1], pw[HELD ? K : 1], pb[HELD ? K : 1];
    if constexpr (HELD)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            const bool in = c < p.width;
            if constexpr (ADDED) ps[k] = p.scale && in ? param(p.scale, c) : zero_pack<IO, V>();
            pw[k] = p.weight && in ? param(p.weight, c) : zero_pack<IO, V>();
            pb[k] = p.bias && in ? param(p.bias, c) : zero_pack<IO, V>();
        }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        float f[K][V], s[1] = {0.f}, mean = 0.f;
        Pack<IO, V> e[K];
        copy_wait<DEPTH - 1>();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            const Pack<IO, V> x = ahead.take(stage, 0, k);
            e[k] = ahead.take(stage, 1, k);
            Pack<IO, V> sc;
            if (ADDED && p.scale) sc = HELD ? ps[HELD && ADDED ? k : 0] : c < p.width ? param(p.scale, c) : zero_pack<IO, V>();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                f[k][i] = !ADDED ? pick(x, i) : p.scale ? fmaf(pick(sc, i), pick(x, i), pick(e[k], i)) : pick(x, i) + pick(e[k], i);
                s[0] += f[k][i];
            }
        }
        ahead.fetch(stage, src, row + DEPTH * step, p.width, row + DEPTH * step < p.rows);
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
        if (ADDED && row < p.rows) {
            IO* t = static_cast<IO*>(p.t) + row * p.width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c < p.width) store_pack(t + c, narrow<IO, V>(f[k]), V, true);
            }
        }
        if (!p.rms) {
            row_sum<TPR>(s, red, turn);
            mean = s[0] * p.inv;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const bool in = (k * TPR + tr) * V < p.width;
#pragma unroll
                for (int i = 0; i < V; ++i) f[k][i] = in ? f[k][i] - mean : 0.f;
            }
        }
        s[0] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] = fmaf(f[k][i], f[k][i], s[0]);
        row_sum<TPR>(s, red, turn);
        const float r = rsqrtf(fmaf(s[0], p.inv, p.eps));
        if (row < p.rows) {
            if (tr == 0 && p.stats) { p.stats[row] = mean; p.stats[p.rows + row] = r; }
            IO* y = static_cast<IO*>(p.y) + row * p.width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c >= p.width) break;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = f[k][i] * r;
                if (p.weight) {
                    const Pack<IO, V> w = HELD ? pw[HELD ? k : 0] : param(p.weight, c);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] *= pick(w, i);
                }
                if (p.bias) {
                    const Pack<IO, V> b = HELD ? pb[HELD ? k : 0] : param(p.bias, c);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += pick(b, i);
                }
                if (!ADDED)
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] *= gate_value(pick(e[k], i), p.silu);
                store_pack(y + c, narrow<IO, V>(o), V, true);
            }
        }
    }
}

template <typename IO, int V, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR), fused_resident(K, V, TPR, true, ADDED)) k_fused_bwd(const FusedP p) {
    constexpr int NT = fused_threads(TPR), RPC = NT / TPR, SUMS = fused_sums(ADDED), STREAMS = ADDED ? 4 : 3;
    extern __shared__ __align__(16) unsigned char smem_rows[];
    __shared__ float red[2][2][32];
    __shared__ float cols[RPC > 1 ? NT * V * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long row = (long long)blockIdx.x * RPC + rg;
    int turn = 0, stage = 0;
    float sum[SUMS][K][V], nmean = 0.f, nr = 0.f;
#pragma unroll
    for (int m = 0; m < SUMS; ++m)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[m][k][i] = 0.f;
    typedef Ahead<IO, V, K, TPR, STREAMS, true> Rows;
    constexpr int DEPTH = Rows::DEPTH;
    const Rows ahead(smem_rows);
    const void* src[STREAMS];
    src[0] = p.x; src[1] = p.e; src[2] = p.dy;
    if constexpr (ADDED) src[3] = p.dt;
    const void* vec = ADDED ? p.scale : p.bias;
    auto stats = [&](long long at) {
        nmean = at < p.rows && !p.rms ? p.stats[at] : 0.f;
        nr = at < p.rows ? p.stats[p.rows + at] : 0.f;
    };
    stats(row);
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) ahead.fetch(d, src, row + d * step, p.width, row + d * step < p.rows);
    auto param = [&](const void* base, int c) { return load_pack<IO, V>(static_cast<const IO*>(base) + c, V, true); };
    Pack<IO, V> pw[K], pv[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + tr) * V;
        pw[k] = p.weight && c < p.width ? param(p.weight, c) : zero_pack<IO, V>();
        pv[k] = vec && c < p.width ? param(vec, c) : zero_pack<IO, V>();
    }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        const float r = nr, mean = nmean;
        Pack<IO, V> keep[K], kx[ADDED ? K : 1];                // dtotal, or dz as it will be written; x
        float xh[K][V], g[K][V], s[2] = {0.f, 0.f};
        copy_wait<DEPTH - 1>();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const bool in = (k * TPR + tr) * V < p.width;
            const Pack<IO, V> x = ahead.take(stage, 0, k), e = ahead.take(stage, 1, k), dy = ahead.take(stage, 2, k);
            float dz[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float v[4] = {pick(x, i), pick(e, i), pick(dy, i), 0.f};
                element<ADDED>(p, v, p.weight ? pick(pw[k], i) : 1.f, pick(pv[k], i), mean, in ? r : 0.f, xh[k][i], g[k][i], dz[i], s, &sum[0][k][i],
                               &sum[1][k][i]);
            }
            if constexpr (ADDED) { keep[k] = ahead.take(stage, 3, k); kx[k] = x; }
            else keep[k] = narrow<IO, V>(dz);
        }
        ahead.fetch(stage, src, row + DEPTH * step, p.width, row + DEPTH * step < p.rows);
        stage = stage + 1 == DEPTH ? 0 : stage + 1;
        stats(row + step);
        row_sum<TPR>(s, red, turn);
        const float m1 = s[0] * p.inv, m2 = p.rms ? 0.f : s[1] * p.inv;
        if (row < p.rows) {
            IO *dx = static_cast<IO*>(p.dx) + row * p.width, *de = static_cast<IO*>(p.de) + row * p.width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c >= p.width) break;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = r * (g[k][i] - m2 - xh[k][i] * m1);
                if constexpr (ADDED) {
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        o[i] += pick(keep[k], i);
                        sum[2][k][i] = fmaf(o[i], pick(kx[k], i), sum[2][k][i]);
                    }
                    store_pack(de + c, narrow<IO, V>(o), V, true);
                    if (vec) {
#pragma unroll
                        for (int i = 0; i < V; ++i) o[i] *= pick(pv[k], i);
                        store_pack(dx + c, narrow<IO, V>(o), V, true);
                    }
                } else {
                    store_pack(de + c, keep[k], V, true);
                    store_pack(dx + c, narrow<IO, V>(o), V, true);
                }
            }
        }
    }
    if (!p.part) return;
    float* part = p.part + (size_t)blockIdx.x * SUMS * p.width;
#pragma unroll
    for (int m = 0; m < SUMS; ++m) {
        if constexpr (RPC > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) cols[rg * (TPR * V * K) + (k * TPR + tr) * V + i] = sum[m][k][i];
            __syncthreads();
            for (int c = threadIdx.x; c < p.width; c += NT) {
                float t = 0.f;
                for (int q = 0; q < RPC; ++q) t += cols[q * (TPR * V * K) + c];
                part[(size_t)m * p.width + c] = t;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (k * TPR + tr) * V + i;
                    if (c < p.width) part[(size_t)m * p.width + c] = sum[m][k][i];
                }
        }
    }
}

// ---- rows that begin anywhere ---------------------------------------------------------------------------------------------------
// A block of rows: RPC groups of lanes, p.step rows each, one after the other in memory, two blocks under way.
template <typename IO, int TPR, int STREAMS>
struct Blocks {
    static constexpr int NT = fused_threads(TPR), RPC = NT / TPR;
    unsigned char* smem;
    int width, rows, stride;                                   // rows of a block, bytes of a stream in a stage
    __device__ __forceinline__ Blocks(unsigned char* s, const FusedP& p)
        : smem(s), width(p.width), rows(RPC * p.step), stride((int)(((size_t)RPC * p.step * p.width * sizeof(IO) + 31) & ~(size_t)15)) {}
    // bytes between an aligned address and the block's first element
    __device__ __forceinline__ int shift(long long block) const { return (int)((unsigned long long)(block * rows) * width * sizeof(IO) & 15); }
    __device__ __forceinline__ void fetch(int stage, const void* const (&src)[STREAMS], long long block, long long all) const {
        const long long first = block * rows;
        if (first < all) {
            const long long end = first + rows < all ? first + rows : all;
            const size_t from = (size_t)first * width * sizeof(IO) & ~(size_t)15, to = (size_t)end * width * sizeof(IO);
            const int pieces = (int)((to - from + 15) / 16);
#pragma unroll
            for (int m = 0; m < STREAMS; ++m)
                if (src[m])
                    for (int i = threadIdx.x; i < pieces; i += NT) {
                        const size_t at = from + (size_t)i * 16;
                        copy_bytes<16>(smem + (stage * STREAMS + m) * stride + i * 16, static_cast<const unsigned char*>(src[m]) + at,
                                       (int)(to - at < 16 ? to - at : 16));
                    }
        }
        copy_commit();
    }
    __device__ __forceinline__ const IO* row(int stage, int stream, long long block, int r) const {
        return reinterpret_cast<const IO*>(smem + (stage * STREAMS + stream) * stride + shift(block)) + r * width;
    }
};

template <typename IO, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR)) k_odd_fwd(const FusedP p) {
    extern __shared__ __align__(16) unsigned char smem_rows[];
    __shared__ float red[2][1][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    int turn = 0;
    const Blocks<IO, TPR, 2> blocks(smem_rows, p);
    const void* const src[2] = {p.x, p.e};
    float w[K], b[K], sc[K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = tr + TPR * k;
        const bool in = c < p.width;
        w[k] = p.weight && in ? ld(static_cast<const IO*>(p.weight), c) : 1.f;
        b[k] = p.bias && in ? ld(static_cast<const IO*>(p.bias), c) : 0.f;
        sc[k] = ADDED && p.scale && in ? ld(static_cast<const IO*>(p.scale), c) : 1.f;
    }
    long long block = blockIdx.x;
    blocks.fetch(0, src, block, p.rows);
    blocks.fetch(1, src, block + gridDim.x, p.rows);
    for (int stage = 0; block * blocks.rows < p.rows; block += gridDim.x, stage ^= 1) {
        copy_wait<1>();
        __syncthreads();
        for (int q = 0; q < p.step; ++q) {
            const int local = q * (fused_threads(TPR) / TPR) + rg;
            const long long row = block * blocks.rows + local;
            const bool live = row < p.rows;
            const IO *x = blocks.row(stage, 0, block, local), *e = blocks.row(stage, 1, block, local);
            float f[K], z[K], s[1] = {0.f}, mean = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = tr + TPR * k;
                const bool in = live && c < p.width;
                f[k] = in ? ld(x, c) : 0.f;
                z[k] = in ? ld(e, c) : 0.f;
                if (ADDED) {
                    f[k] = fmaf(sc[k], f[k], z[k]);
                    if (in) st(static_cast<IO*>(p.t), (size_t)(row * p.width + c), f[k]);
                }
                s[0] += f[k];
            }
            if (!p.rms) {
                row_sum<TPR>(s, red, turn);
                mean = s[0] * p.inv;
#pragma unroll
                for (int k = 0; k < K; ++k) f[k] = tr + TPR * k < p.width ? f[k] - mean : 0.f;
            }
            s[0] = 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) s[0] = fmaf(f[k], f[k], s[0]);
            row_sum<TPR>(s, red, turn);
            const float r = rsqrtf(fmaf(s[0], p.inv, p.eps));
            if (!live) continue;
            if (tr == 0 && p.stats) { p.stats[row] = mean; p.stats[p.rows + row] = r; }
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = tr + TPR * k;
                if (c >= p.width) break;
                float o = fmaf(f[k] * r, w[k], b[k]);
                if (!ADDED) o *= gate_value(z[k], p.silu);
                st(static_cast<IO*>(p.y), (size_t)(row * p.width + c), o);
            }
        }
        __syncthreads();
        blocks.fetch(stage, src, block + 2LL * gridDim.x, p.rows);
    }
}

template <typename IO, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR)) k_odd_bwd(const FusedP p) {
    constexpr int NT = fused_threads(TPR), RPC = NT / TPR, SUMS = fused_sums(ADDED), STREAMS = ADDED ? 4 : 3;
    extern __shared__ __align__(16) unsigned char smem_rows[];
    __shared__ float red[2][2][32];
    __shared__ float cols[RPC > 1 ? NT * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    int turn = 0;
    const Blocks<IO, TPR, STREAMS> blocks(smem_rows, p);
    const void* src[STREAMS];
    src[0] = p.x; src[1] = p.e; src[2] = p.dy;
    if constexpr (ADDED) src[3] = p.dt;
    const void* vec = ADDED ? p.scale : p.bias;
    float w[K], v[K], sum[SUMS][K];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = tr + TPR * k;
        w[k] = p.weight && c < p.width ? ld(static_cast<const IO*>(p.weight), c) : 1.f;
        v[k] = vec && c < p.width ? ld(static_cast<const IO*>(vec), c) : 1.f;
#pragma unroll
        for (int m = 0; m < SUMS; ++m) sum[m][k] = 0.f;
    }
    long long block = blockIdx.x;
    blocks.fetch(0, src, block, p.rows);
    blocks.fetch(1, src, block + gridDim.x, p.rows);
    for (int stage = 0; block * blocks.rows < p.rows; block += gridDim.x, stage ^= 1) {
        copy_wait<1>();
        __syncthreads();
        for (int q = 0; q < p.step; ++q) {
            const int local = q * RPC + rg;
            const long long row = block * blocks.rows + local;
            const bool live = row < p.rows;
            const float mean = live && !p.rms ? p.stats[row] : 0.f, r = live ? p.stats[p.rows + row] : 0.f;
            const IO *x = blocks.row(stage, 0, block, local), *e = blocks.row(stage, 1, block, local), *y = blocks.row(stage, 2, block, local),
                     *t = ADDED && p.dt ? blocks.row(stage, STREAMS - 1, block, local) : nullptr;
            float xh[K], g[K], dz[K], s[2] = {0.f, 0.f};
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = tr + TPR * k;
                const bool in = live && c < p.width;
                const float u[4] = {in ? ld(x, c) : 0.f, in ? ld(e, c) : 0.f, in ? ld(y, c) : 0.f, 0.f};
                element<ADDED>(p, u, w[k], v[k], mean, in ? r : 0.f, xh[k], g[k], dz[k], s, &sum[0][k], &sum[1][k]);
            }
            row_sum<TPR>(s, red, turn);
            const float m1 = s[0] * p.inv, m2 = p.rms ? 0.f : s[1] * p.inv;
            if (!live) continue;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = tr + TPR * k;
                if (c >= p.width) break;
                const size_t at = (size_t)(row * p.width + c);
                float o = r * (g[k] - m2 - xh[k] * m1);
                if constexpr (ADDED) {
                    if (t) o += ld(t, c);
                    sum[2][k] = fmaf(o, ld(x, c), sum[2][k]);
                    st(static_cast<IO*>(p.de), at, o);
                    if (vec) st(static_cast<IO*>(p.dx), at, o * v[k]);
                } else {
                    st(static_cast<IO*>(p.de), at, dz[k]);
                    st(static_cast<IO*>(p.dx), at, o);
                }
            }
        }
        __syncthreads();
        blocks.fetch(stage, src, block + 2LL * gridDim.x, p.rows);
    }
    if (!p.part) return;
    float* part = p.part + (size_t)blockIdx.x * SUMS * p.width;
#pragma unroll
    for (int m = 0; m < SUMS; ++m) {
        if constexpr (RPC > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k) cols[rg * (TPR * K) + k * TPR + tr] = sum[m][k];
            __syncthreads();
            for (int c = threadIdx.x; c < p.width; c += NT) {
                float t = 0.f;
                for (int q = 0; q < RPC; ++q) t += cols[q * (TPR * K) + c];
                part[(size_t)m * p.width + c] = t;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (tr + TPR * k < p.width) part[(size_t)m * p.width + tr + TPR * k] = sum[m][k];
        }
    }
}

// ---- wide rows, backward ----------------------------------------------------------------------------------------------------------
constexpr int kWideThreads = 256;
template <typename IO, int V, bool ADDED>
__device__ __forceinline__ void wide_load(const FusedP& p, long long row, int c, Pack<IO, V> (&u)[4]) {
    const void* const src[4] = {p.x, p.e, p.dy, ADDED ? p.dt : nullptr};
#pragma unroll
    for (int m = 0; m < 4; ++m) u[m] = src[m] ? load_pack<IO, V>(static_cast<const IO*>(src[m]) + row * p.width + c, V, V > 1) : zero_pack<IO, V>();
}
template <typename IO, int V, bool ADDED>
__global__ void __launch_bounds__(kWideThreads) k_wide_sums(const FusedP p) {
    __shared__ float red[2][2][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const void* vec = ADDED ? p.scale : p.bias;
    int turn = 0;
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const float mean = p.rms ? 0.f : p.stats[row], r = p.stats[p.rows + row];
        float s[2] = {0.f, 0.f};
#pragma unroll(V * sizeof(IO) == 16 ? 2 : 8)
        for (int c = threadIdx.x * V; c < p.width; c += kWideThreads * V) {
            Pack<IO, V> u[4];
            wide_load<IO, V, false>(p, row, c, u);
            const Pack<IO, V> w = p.weight ? load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, V, V > 1) : zero_pack<IO, V>(),
                              v = vec ? load_pack<IO, V>(static_cast<const IO*>(vec) + c, V, V > 1) : zero_pack<IO, V>();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float in[4] = {pick(u[0], i), pick(u[1], i), pick(u[2], i), 0.f};
                float xh, g, dz;
                element<ADDED>(p, in, p.weight ? pick(w, i) : 1.f, pick(v, i), mean, r, xh, g, dz, s, nullptr, nullptr);
            }
        }
        row_sum<kWideThreads>(s, red, turn);
        if (threadIdx.x == 0) { p.rowsum[row] = s[0] * p.inv; p.rowsum[p.rows + row] = p.rms ? 0.f : s[1] * p.inv; }
    }
}
template <typename IO, int V, bool ADDED>
__global__ void __launch_bounds__(kWideThreads) k_wide_cols(const FusedP p) {
    constexpr int SUMS = fused_sums(ADDED), U = V * sizeof(IO) == 16 ? 2 : 4;     // rows under way
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int c = (blockIdx.x * kWideThreads + threadIdx.x) * V;
    if (c >= p.width) return;
    const void* vec = ADDED ? p.scale : p.bias;
    const Pack<IO, V> w = p.weight ? load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, V, V > 1) : zero_pack<IO, V>(),
                      v = vec ? load_pack<IO, V>(static_cast<const IO*>(vec) + c, V, V > 1) : zero_pack<IO, V>();
    float sum[SUMS][V];
#pragma unroll
    for (int m = 0; m < SUMS; ++m)
#pragma unroll
        for (int i = 0; i < V; ++i) sum[m][i] = 0.f;
    const long long first = (long long)blockIdx.y * p.step, end = first + p.step < p.rows ? first + p.step : p.rows;
    for (long long row0 = first; row0 < end; row0 += U) {
        Pack<IO, V> u[U][4];
#pragma unroll
        for (int j = 0; j < U; ++j)
            if (row0 + j < end) wide_load<IO, V, ADDED>(p, row0 + j, c, u[j]);
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const long long row = row0 + j;
            if (row >= end) break;
            const float mean = p.rms ? 0.f : p.stats[row], r = p.stats[p.rows + row], m1 = p.rowsum[row], m2 = p.rowsum[p.rows + row];
            float o[V], dz[V], s[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float in[4] = {pick(u[j][0], i), pick(u[j][1], i), pick(u[j][2], i), pick(u[j][3], i)};
                float xh, g;
                element<ADDED>(p, in, p.weight ? pick(w, i) : 1.f, pick(v, i), mean, r, xh, g, dz[i], s, &sum[0][i], &sum[1][i]);
                o[i] = r * (g - m2 - xh * m1);
                if constexpr (ADDED) {
                    o[i] += in[3];
                    sum[2][i] = fmaf(o[i], in[0], sum[2][i]);
                }
            }
            IO *dx = static_cast<IO*>(p.dx) + row * p.width + c, *de = static_cast<IO*>(p.de) + row * p.width + c;
            if constexpr (ADDED) {
                store_pack(de, narrow<IO, V>(o), V, V > 1);
                if (vec) {
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] *= pick(v, i);
                    store_pack(dx, narrow<IO, V>(o), V, V > 1);
                }
            } else {
                store_pack(de, narrow<IO, V>(dz), V, V > 1);
                store_pack(dx, narrow<IO, V>(o), V, V > 1);
            }
        }
    }
    if (!p.part) return;
    float* part = p.part + (size_t)blockIdx.y * SUMS * p.width + c;
#pragma unroll
    for (int m = 0; m < SUMS; ++m)
#pragma unroll
        for (int i = 0; i < V; ++i) part[(size_t)m * p.width + i] = sum[m][i];
}

// out[m][c] = sum over p of part[p][m][c], in an order that depends on nothing but `parts`; absent outputs are skipped
struct SumOut { float* out[3]; };
__global__ void __launch_bounds__(32 * kSumRows) k_fused_sums(const float* part, int parts, int width, int sums, SumOut o) {
    __shared__ float s[kSumRows][33];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    float* out = o.out[blockIdx.y];
    if (!out) return;
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float a = 0.f;
    if (c < width)
#pragma unroll 8
        for (int p = y; p < parts; p += kSumRows) a += part[((long long)p * sums + blockIdx.y) * width + c];
    s[y][x] = a;
    __syncthreads();
    a = s[x][y];
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) a += __shfl_xor_sync(0xffffffffu, a, w);
    if (x == 0 && blockIdx.x * 32 + y < (unsigned)width) out[blockIdx.x * 32 + y] = a;
}

// ---- which plan ---------------------------------------------------------------------------------------------------------------------
enum Kind { WHOLE, ODD, WIDE };
struct FusedPlan {
    Kind kind;
    int v;                   // elements of a group: of 16 bytes where rows are whole groups of those, else of 4; 1 of an odd bf16 row
    int tpr, k;              // lanes of a row, groups of a lane
    int step;                // FusedP::step
    long long ctas;          // that write a partial each
    int tiles;               // wide: CTAs side by side
};
FusedPlan fused_plan(long long rows, int width, int dtype, bool bwd, bool added) {
    const int io = dtype == QD_BF16 ? 2 : 4;
    FusedPlan q{};
    q.v = width % (16 / io) == 0 ? 16 / io : width % (4 / io) == 0 ? 4 / io : 1;
    const bool odd = q.v * io < 4, big = q.v * io == 16;
    const int n = width / q.v;
    // what registers hold: 16 elements to a lane and one to three sums of each
    if (bwd && n > (big ? 1024 : 2048)) {
        q.kind = WIDE;
        q.tiles = (n + kWideThreads - 1) / kWideThreads;
        const long long slabs = (6 * kSMs + q.tiles - 1) / q.tiles;
        q.step = (int)((rows + slabs - 1) / slabs);
        q.ctas = (rows + q.step - 1) / q.step;
        return q;
    }
    q.kind = odd ? ODD : WHOLE;
    q.step = 1;
    if (odd) {
        q.k = width <= 32 ? 4 : width <= 4096 ? 8 : 32;
        q.tpr = width <= 32 ? 8 : width <= 4096 ? 32 : 512;
        while (q.tpr * q.k < width) q.tpr *= 2;
        const int rpc = fused_threads(q.tpr) / q.tpr, block = rpc * width * io;
        const long long share = rows / (rpc * 2LL * kSMs);                  // few rows: as many CTAs as there are SMs
        q.step = block >= 4096 ? 1 : 4096 / block;                          // 4 KB of a stream in a block, if rows are short
        if (q.step > share) q.step = share < 1 ? 1 : (int)share;
    } else {
        const int most = bwd ? 256 : 512;
        q.k = bwd ? (big ? 1 : 4) : (big ? 2 : 8);
        for (q.tpr = 1; q.tpr * q.k < n && q.tpr < most; q.tpr *= 2) {}
        if (bwd && q.tpr * q.k < n) { q.k *= 2; if (q.tpr * q.k < n) q.tpr = 512; }
        while (q.tpr * q.k < n) q.k *= 2;
    }
    const int rpc = fused_threads(q.tpr) / q.tpr * q.step;
    const int resident = odd ? (q.tpr > 256 ? 1 : 4) : fused_resident(q.k, q.v, q.tpr, bwd, added);
    const long long groups = (rows + rpc - 1) / rpc, all = kSMs * (long long)resident;
    q.ctas = groups < all ? groups : all;
    return q;
}

template <class K>
cudaError_t go(K kern, dim3 grid, int threads, size_t bytes, const FusedP& p, cudaStream_t stream) {
    const cudaError_t e = bytes > 32768 ? set_max_smem_once((const void*)kern, bytes) : cudaSuccess;
    return e != cudaSuccess ? e : launch_overlapped(kern, grid, dim3(threads), bytes, stream, p);
}
template <typename IO, int V, int K, int TPR, bool ADDED, bool BWD>
cudaError_t whole(const FusedP& p, dim3 grid, cudaStream_t stream) {
    constexpr int bytes = Ahead<IO, V, K, TPR, !BWD ? 2 : ADDED ? 4 : 3, BWD>::kBytes;
    if constexpr (BWD) return go(k_fused_bwd<IO, V, K, TPR, ADDED>, grid, fused_threads(TPR), bytes, p, stream);
    else return go(k_fused_fwd<IO, V, K, TPR, ADDED>, grid, fused_threads(TPR), bytes, p, stream);
}
template <typename IO, int V, bool ADDED, bool BWD>
cudaError_t whole(const FusedP& p, const FusedPlan& q, cudaStream_t stream) {
    const dim3 grid((unsigned)q.ctas);
    constexpr bool BIG = V * sizeof(IO) == 16;
    constexpr int L = BWD ? (BIG ? 1 : 4) : (BIG ? 2 : 8);
#define QD_FUSED(TPR, K) if (q.tpr == TPR && q.k == (K)) return whole<IO, V, (K), TPR, ADDED, BWD>(p, grid, stream);
    QD_FUSED(1, L) QD_FUSED(2, L) QD_FUSED(4, L) QD_FUSED(8, L) QD_FUSED(16, L) QD_FUSED(32, L) QD_FUSED(64, L) QD_FUSED(128, L) QD_FUSED(256, L)
    if constexpr (BWD) {
        QD_FUSED(256, 2 * L)
        if constexpr (BIG) QD_FUSED(512, 2 * L)
    } else {
        QD_FUSED(512, L) QD_FUSED(512, 2 * L)
        if constexpr (sizeof(IO) == 4) QD_FUSED(512, 4 * L)
    }
#undef QD_FUSED
    return cudaErrorInvalidValue;
}
template <int K, int TPR, bool ADDED, bool BWD>
cudaError_t odd(const FusedP& p, dim3 grid, cudaStream_t stream) {
    constexpr int NT = fused_threads(TPR), STREAMS = !BWD ? 2 : ADDED ? 4 : 3;
    const size_t bytes = 2 * STREAMS * (((size_t)NT / TPR * p.step * p.width * 2 + 31) & ~(size_t)15);
    if constexpr (BWD) return go(k_odd_bwd<__nv_bfloat16, K, TPR, ADDED>, grid, NT, bytes, p, stream);
    else return go(k_odd_fwd<__nv_bfloat16, K, TPR, ADDED>, grid, NT, bytes, p, stream);
}
template <typename IO, int V, bool ADDED>
cudaError_t wide(const FusedP& p, const FusedPlan& q, cudaStream_t stream) {
    const long long most = 8LL * kSMs;
    const cudaError_t e = go(k_wide_sums<IO, V, ADDED>, dim3((unsigned)(p.rows < most ? p.rows : most)), kWideThreads, 0, p, stream);
    return e != cudaSuccess ? e : go(k_wide_cols<IO, V, ADDED>, dim3((unsigned)q.tiles, (unsigned)q.ctas), kWideThreads, 0, p, stream);
}
template <typename IO, bool ADDED, bool BWD>
cudaError_t launch(FusedP p, cudaStream_t stream) {
    constexpr int BIG = 16 / sizeof(IO), SMALL = 4 / sizeof(IO);
    const FusedPlan q = fused_plan(p.rows, p.width, sizeof(IO) == 2 ? QD_BF16 : QD_F32, BWD, ADDED);
    p.step = q.step;
    if (q.kind == WHOLE) return q.v == BIG ? whole<IO, BIG, ADDED, BWD>(p, q, stream) : whole<IO, SMALL, ADDED, BWD>(p, q, stream);
    if constexpr (BWD)
        if (q.kind == WIDE) {
            if (q.v == BIG) return wide<IO, BIG, ADDED>(p, q, stream);
            if constexpr (SMALL > 1)
                if (q.v == SMALL) return wide<IO, SMALL, ADDED>(p, q, stream);
            return wide<IO, 1, ADDED>(p, q, stream);
        }
    if constexpr (sizeof(IO) == 2) {
        const dim3 grid((unsigned)q.ctas);
#define QD_ODD(TPR, K) if (q.tpr == TPR && q.k == K) return odd<K, TPR, ADDED, BWD>(p, grid, stream);
        QD_ODD(8, 4) QD_ODD(32, 8) QD_ODD(64, 8) QD_ODD(128, 8) QD_ODD(256, 8)
        if constexpr (!BWD) { QD_ODD(512, 8) QD_ODD(512, 32) }
#undef QD_ODD
    }
    return cudaErrorInvalidValue;
}
template <bool ADDED, bool BWD>
cudaError_t launch(const FusedP& p, int dtype, cudaStream_t stream) {
    return dtype == QD_BF16 ? launch<__nv_bfloat16, ADDED, BWD>(p, stream) : launch<float, ADDED, BWD>(p, stream);
}
FusedP fused(const FusedNormArgs& a) {
    FusedP p{};
    p.rows = a.rows; p.width = a.width; p.inv = 1.f / (float)a.width; p.eps = a.eps; p.rms = a.rms; p.silu = a.silu;
    p.x = a.x; p.scale = a.scale; p.weight = a.weight; p.bias = a.bias; p.dy = a.dy; p.dt = a.dtotal;
    p.y = a.y; p.t = a.total; p.stats = a.stats; p.dx = a.dx;
    p.e = a.added ? a.residual : a.gate;
    p.de = a.added ? a.dresidual : a.dgate;
    return p;
}
// the workspace: partial sums, then the rows' sums
size_t part_floats(const FusedPlan& q, int width) { return ((size_t)q.ctas * fused_sums(true) * width + 3) & ~(size_t)3; }

}  // namespace

size_t fused_norm_workspace(long long rows, int width, int dtype) {
    const FusedPlan q = fused_plan(rows, width, dtype, true, true);      // backward alike for both
    return (part_floats(q, width) + (q.kind == WIDE ? 2 * (size_t)rows : 0)) * sizeof(float);
}
bool fused_norm_needs_workspace(long long rows, int width, int dtype) { return fused_plan(rows, width, dtype, true, true).kind == WIDE; }

cudaError_t fused_norm_fwd(const FusedNormArgs& a) {
    const FusedP p = fused(a);
    return a.added ? launch<true, false>(p, a.dtype, a.stream) : launch<false, false>(p, a.dtype, a.stream);
}
cudaError_t fused_norm_bwd(const FusedNormArgs& a) {
    FusedP p = fused(a);
    const FusedPlan q = fused_plan(a.rows, a.width, a.dtype, true, a.added);
    const SumOut out{{a.dweight, a.dbias, a.added ? a.dscale : nullptr}};
    const bool sums = out.out[0] || out.out[1] || out.out[2];
    p.part = sums ? a.part : nullptr;
    p.rowsum = q.kind == WIDE ? a.part + part_floats(q, a.width) : nullptr;
    cudaError_t e = a.added ? launch<true, true>(p, a.dtype, a.stream) : launch<false, true>(p, a.dtype, a.stream);
    const int n = fused_sums(a.added);
    if (e == cudaSuccess && sums)
        e = launch_overlapped(k_fused_sums, dim3((unsigned)((a.width + 31) / 32), n), dim3(32 * kSumRows), 0, a.stream, p.part, (int)q.ctas, a.width, n,
                              out);
    // without a scale the kernels write dresidual alone: a caller who wants it in two places has it copied (a store of both, under a condition
    // of its own, made the call with a scale 1.5 % slower)
    if (e == cudaSuccess && a.added && !a.scale && a.dx)
        e = cudaMemcpyAsync(a.dx, a.dresidual, (size_t)a.rows * a.width * (a.dtype == QD_BF16 ? 2 : 4), cudaMemcpyDeviceToDevice, a.stream);
    return e;
}

}  // namespace qd

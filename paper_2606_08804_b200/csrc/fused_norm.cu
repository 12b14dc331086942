// Layer norm (norm.cu) together with what stands beside it in a layer:
//   gated    y = ((x - m) r w + b) f(z),  f = SiLU or the logistic function             (a read-out per head)
//            dn = dy f, dz = dy ((x - m) r w + b) f'(z), then as a norm's backward with dn for dy
//   added    t = e + s x (residual and scale),  y = (t - m) r w + b                      (the residual stream)
//            d = norm's backward of dy at t, + dt;  de = d, dx = s d, ds = sum_rows d x    (t added up again: rounded to bf16 it costs dw, an
//            fp32 sum of terms of both signs, 1.6e-3 of its length)
// Backward of the norm, with g = dy w and x^ = (x - m) r:  dx = r (g - x^ mean(g x^) - mean(g))  (the last term not without the mean),
// dw = sum_rows dy x^, db = sum_rows dy.
//
// Bound by HBM.  Rows belong to groups of lanes or to a CTA and are read once into registers, the next one on its way, as in norm.cu;
// backward the sums over rows stay in registers, one partial per CTA, added up in a fixed order.
#include "rows.cuh"

namespace qd {
namespace {

struct FusedP {
    long long rows;
    int width;
    const void *x, *e, *scale, *weight, *bias, *dy, *dt;      // e: gate or residual
    void *y, *t, *dx, *de;
    float* stats;                                              // [2][rows]: mean, r
    float* part;                                               // backward: [gridDim.x][sums][width]
    float eps, inv;
    bool rms, silu;
};
constexpr __host__ __device__ int fused_threads(int tpr) { return tpr > 256 ? tpr : 256; }
constexpr __host__ __device__ int fused_resident(int k, int v, int tpr, bool bwd) {
    return tpr > 256 ? 1 : bwd ? (k * v <= 8 ? 2 : 1) : (k * v <= 8 ? 4 : k * v <= 16 ? 2 : 1);
}
constexpr __host__ __device__ int fused_sums(bool added) { return added ? 3 : 2; }

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
template <typename IO, int V, int K, int TPR>
__device__ __forceinline__ void columns(const void* base, long long row, int width, bool live, Pack<IO, V> (&v)[K]) {
    const IO* p = static_cast<const IO*>(base) + row * width;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + threadIdx.x % TPR) * V;
        v[k] = live && c < width ? load_pack<IO, V>(p + c, V, V > 1) : zero_pack<IO, V>();
    }
}
// the gate and its slope
__device__ __forceinline__ float gate_value(float z, bool silu) { const float s = gate_sigmoid(z); return silu ? z * s : s; }
__device__ __forceinline__ float2 gate_slope(float z, bool silu) {
    const float s = gate_sigmoid(z);
    return silu ? make_float2(z * s, s * fmaf(z, 1.f - s, 1.f)) : make_float2(s, s * (1.f - s));
}

template <typename IO, int V, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR), fused_resident(K, V, TPR, false)) k_fused_fwd(const FusedP p) {
    constexpr int RPC = fused_threads(TPR) / TPR;
    constexpr bool HELD = K * V <= 16;                       // scale, weight and bias stay in registers
    __shared__ float red[2][1][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long row = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    int turn = 0;
    Pack<IO, V> nx[K], ne[K], ps[HELD && ADDED ? K : 1], pw[HELD ? K : 1], pb[HELD ? K : 1];
    auto ahead = [&](long long at) {
        columns<IO, V, K, TPR>(p.x, at, p.width, at < p.rows, nx);
        columns<IO, V, K, TPR>(p.e, at, p.width, at < p.rows, ne);
    };
    auto param = [&](const void* base, int c) { return load_pack<IO, V>(static_cast<const IO*>(base) + c, V, V > 1); };
    ahead(row);
    if constexpr (HELD) {
        if (ADDED && p.scale) columns<IO, V, K, TPR>(p.scale, 0, p.width, true, reinterpret_cast<Pack<IO, V>(&)[K]>(ps));
        if (p.weight) columns<IO, V, K, TPR>(p.weight, 0, p.width, true, pw);
        if (p.bias) columns<IO, V, K, TPR>(p.bias, 0, p.width, true, pb);
    }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        float f[K][V], s[1] = {0.f}, mean = 0.f;
        Pack<IO, V> e[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            e[k] = ne[k];
            Pack<IO, V> sc;
            if (ADDED && p.scale) sc = HELD ? ps[HELD ? k : 0] : c < p.width ? param(p.scale, c) : zero_pack<IO, V>();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x = pick(nx[k], i);
                f[k][i] = !ADDED ? x : p.scale ? fmaf(pick(sc, i), x, pick(ne[k], i)) : x + pick(ne[k], i);
                s[0] += f[k][i];
            }
        }
        if (first + step < p.rows) ahead(row + step);
        if (ADDED && row < p.rows) {
            IO* t = static_cast<IO*>(p.t) + row * p.width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c < p.width) store_pack(t + c, narrow<IO, V>(f[k]), V, V > 1);
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
                store_pack(y + c, narrow<IO, V>(o), V, V > 1);
            }
        }
    }
}

template <typename IO, int V, int K, int TPR, bool ADDED>
__global__ void __launch_bounds__(fused_threads(TPR), fused_resident(K, V, TPR, true)) k_fused_bwd(const FusedP p) {
    constexpr int NT = fused_threads(TPR), RPC = NT / TPR, SUMS = fused_sums(ADDED);
    constexpr bool HELD = K * V <= 16;
    __shared__ float red[2][2][32];
    __shared__ float cols[RPC > 1 ? NT * V * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long row = (long long)blockIdx.x * RPC + rg;
    int turn = 0;
    float sum[SUMS][K][V], nmean = 0.f, nr = 0.f;
#pragma unroll
    for (int m = 0; m < SUMS; ++m)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) sum[m][k][i] = 0.f;
    // x, gate or residual, dy, and dtotal of the sum
    Pack<IO, V> n0[K], n1[K], n2[K], n3[ADDED ? K : 1], pw[HELD ? K : 1], pv[HELD ? K : 1];
    const void* vec = ADDED ? p.scale : p.bias;
    auto ahead = [&](long long at) {
        const bool live = at < p.rows;
        columns<IO, V, K, TPR>(p.x, at, p.width, live, n0);
        columns<IO, V, K, TPR>(p.e, at, p.width, live, n1);
        columns<IO, V, K, TPR>(p.dy, at, p.width, live, n2);
        if constexpr (ADDED) columns<IO, V, K, TPR>(p.dt, at, p.width, live && p.dt, n3);
        nmean = live && !p.rms ? p.stats[at] : 0.f;
        nr = live ? p.stats[p.rows + at] : 0.f;
    };
    auto param = [&](const void* base, int c) { return load_pack<IO, V>(static_cast<const IO*>(base) + c, V, V > 1); };
    ahead(row);
    if constexpr (HELD) {
        if (p.weight) columns<IO, V, K, TPR>(p.weight, 0, p.width, true, pw);
        if (vec) columns<IO, V, K, TPR>(vec, 0, p.width, true, pv);
    }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        const float r = nr;
        Pack<IO, V> keep[K], kx[ADDED ? K : 1];                // dtotal, or dz as it will be written; x
        float xh[K][V], g[K][V], s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            const bool in = c < p.width;
            Pack<IO, V> w, v;
            if (p.weight) w = HELD ? pw[HELD ? k : 0] : in ? param(p.weight, c) : zero_pack<IO, V>();
            if (vec) v = HELD ? pv[HELD ? k : 0] : in ? param(vec, c) : zero_pack<IO, V>();
            float dz[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float x = pick(n0[k], i);
                if (ADDED) x = vec ? fmaf(pick(v, i), x, pick(n1[k], i)) : x + pick(n1[k], i);
                xh[k][i] = in ? (x - nmean) * r : 0.f;
                float d = pick(n2[k], i);
                const float wi = p.weight ? pick(w, i) : 1.f;
                if (!ADDED) {
                    const float2 fz = gate_slope(pick(n1[k], i), p.silu);
                    dz[i] = d * fmaf(xh[k][i], wi, vec ? pick(v, i) : 0.f) * fz.y;
                    d *= fz.x;
                }
                g[k][i] = d * wi;
                s[0] = fmaf(g[k][i], xh[k][i], s[0]);
                s[1] += g[k][i];
                sum[0][k][i] = fmaf(d, xh[k][i], sum[0][k][i]);
                sum[1][k][i] += d;
            }
            if constexpr (ADDED) { keep[k] = n3[k]; kx[k] = n0[k]; }
            else keep[k] = narrow<IO, V>(dz);
        }
        if (first + step < p.rows) ahead(row + step);
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
                    store_pack(de + c, narrow<IO, V>(o), V, V > 1);
                    if (vec) {
                        const Pack<IO, V> v = HELD ? pv[HELD ? k : 0] : param(vec, c);
#pragma unroll
                        for (int i = 0; i < V; ++i) o[i] *= pick(v, i);
                        store_pack(dx + c, narrow<IO, V>(o), V, V > 1);
                    }
                } else {
                    store_pack(de + c, keep[k], V, V > 1);
                    store_pack(dx + c, narrow<IO, V>(o), V, V > 1);
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

int fused_vector(int width, int dtype) {
    const int v = dtype == QD_BF16 ? 8 : 4;
    return width % v == 0 ? v : 1;
}
struct FusedShape { int tpr, k; };
FusedShape fused_shape(int n, bool bwd) {
    const int k = bwd ? 1 : 2;
    for (int tpr = 1; tpr <= 32; tpr *= 2)
        if (n <= k * tpr) return {tpr, k};
    if (n <= 256) return {256, 1};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 4096) return {1024, 4};
    return {1024, 16};
}
long long fused_ctas(long long rows, const FusedShape& s, int resident) {
    const int rpc = fused_threads(s.tpr) / s.tpr;
    const long long groups = (rows + rpc - 1) / rpc, most = kSMs * (long long)resident;
    return groups < most ? groups : most;
}

template <typename IO, int V, bool ADDED, bool BWD>
cudaError_t launch(const FusedP& p, cudaStream_t stream) {
    const FusedShape s = fused_shape((p.width + V - 1) / V, BWD);
#define QD_FUSED(TPR, K)                                                                                                            \
    if (s.tpr == TPR && s.k == K) {                                                                                                   \
        const dim3 grid((unsigned)fused_ctas(p.rows, s, fused_resident(K, V, TPR, BWD)));                                              \
        if constexpr (BWD) return launch_overlapped(k_fused_bwd<IO, V, K, TPR, ADDED>, grid, dim3(fused_threads(TPR)), 0, stream, p);   \
        else return launch_overlapped(k_fused_fwd<IO, V, K, TPR, ADDED>, grid, dim3(fused_threads(TPR)), 0, stream, p);                 \
    }
    constexpr int L = BWD ? 1 : 2;
    QD_FUSED(1, L) QD_FUSED(2, L) QD_FUSED(4, L) QD_FUSED(8, L) QD_FUSED(16, L) QD_FUSED(32, L)
    QD_FUSED(256, 1) QD_FUSED(256, 2) QD_FUSED(256, 4) QD_FUSED(1024, 4)
    if constexpr (V == 1) QD_FUSED(1024, 16)
#undef QD_FUSED
    return cudaErrorInvalidValue;
}
template <bool ADDED, bool BWD>
cudaError_t launch(const FusedP& p, int dtype, cudaStream_t stream) {
    const bool vec = fused_vector(p.width, dtype) > 1;
    if (dtype == QD_BF16) return vec ? launch<__nv_bfloat16, 8, ADDED, BWD>(p, stream) : launch<__nv_bfloat16, 1, ADDED, BWD>(p, stream);
    return vec ? launch<float, 4, ADDED, BWD>(p, stream) : launch<float, 1, ADDED, BWD>(p, stream);
}
long long fused_bwd_ctas(long long rows, int width, int dtype) {
    const int V = fused_vector(width, dtype);
    const FusedShape s = fused_shape((width + V - 1) / V, true);
    return fused_ctas(rows, s, fused_resident(s.k, V, s.tpr, true));
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

}  // namespace

size_t fused_norm_workspace(long long rows, int width, int dtype) {
    return (size_t)fused_bwd_ctas(rows, width, dtype) * fused_sums(true) * width * sizeof(float);
}
cudaError_t fused_norm_fwd(const FusedNormArgs& a) {
    const FusedP p = fused(a);
    return a.added ? launch<true, false>(p, a.dtype, a.stream) : launch<false, false>(p, a.dtype, a.stream);
}
cudaError_t fused_norm_bwd(const FusedNormArgs& a) {
    FusedP p = fused(a);
    const SumOut out{{a.dweight, a.dbias, a.added ? a.dscale : nullptr}};
    const bool sums = out.out[0] || out.out[1] || out.out[2];
    p.part = sums ? a.part : nullptr;
    const cudaError_t e = a.added ? launch<true, true>(p, a.dtype, a.stream) : launch<false, true>(p, a.dtype, a.stream);
    if (e != cudaSuccess || !sums) return e;
    const int n = fused_sums(a.added);
    return launch_overlapped(k_fused_sums, dim3((unsigned)((a.width + 31) / 32), n), dim3(32 * kSumRows), 0, a.stream, p.part,
                             (int)fused_bwd_ctas(a.rows, a.width, a.dtype), a.width, n, out);
}

}  // namespace qd

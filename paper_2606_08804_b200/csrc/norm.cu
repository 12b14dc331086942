// Layer norm over the last dimension, with or without the mean (rms), optional weight and bias:
//   m = mean(x) (0 for rms), r = 1 / sqrt(mean((x - m)^2) + eps), x^ = (x - m) r, y = x^ w + b.
// Backward, with g = dy w:  dx = r (g - x^ mean(g x^) - mean(g))  (the last term not for rms),  dw = sum_rows dy x^,  db = sum_rows dy.
//
// Bound by HBM: 262144 rows of 128 bf16 take 24.5 us forward (5.5 TB/s) and 39.5 backward (5.1 TB/s), 16384 rows of 2048 27 and 42; 256
// rows are one launch.  A row is read once into registers, where the mean is taken before the squares of what it leaves.  A row belongs to a
// group of 2^k lanes, or to a CTA where it is too wide for a warp; a lane has several groups of columns, since what is done once a row
// (sums over lanes, the root, addresses) otherwise is more than what is done with the columns.  CTAs stay and take every gridDim-th row
// group, the next one on its way while this one is worked on; backward dw and db so add up in registers (a thread has the same columns
// in every row) and one partial per CTA is left, which k_sum_parts adds in a fixed order.
#include "rows.cuh"

namespace qd {
namespace {

struct NormP {
    long long rows;
    int width;
    const void *x, *weight, *bias, *dy;
    void *y, *dx;
    float *stats;                            // [2][rows]: mean, r
    float* part;                             // backward: [gridDim.x][2][width]
    float eps, inv;                          // inv = 1 / width
    bool rms;
};

constexpr __host__ __device__ int norm_threads(int tpr) { return tpr > 256 ? tpr : 256; }
// CTAs to an SM that the register budget is made for, for K groups of V columns to a thread
constexpr __host__ __device__ int norm_resident(int k, int v, int tpr, bool bwd) {
    return tpr > 256 ? 1 : bwd ? (k * v < 8 ? 3 : k * v <= 16 ? 2 : 1) : (k * v <= 8 ? 4 : k * v <= 16 ? 3 : 2);
}

// Sums of v[0 .. M) over the TPR threads of a row, the same bits in each of them.  One barrier: `turn` alternates between two halves of red,
// and who writes a half again has passed the barrier after everybody read it.
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
        const int first = threadIdx.x / TPR * (TPR / 32);      // warps of this row
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = red[turn][m][first + threadIdx.x % (TPR / 32)];
        turn ^= 1;
#pragma unroll
        for (int w = TPR / 64; w > 0; w >>= 1)
#pragma unroll
            for (int m = 0; m < M; ++m) v[m] += __shfl_xor_sync(0xffffffffu, v[m], w);
    }
}
// This thread's columns of a row; V > 1 only where rows are whole groups.
template <typename IO, int V, int K, int TPR>
__device__ __forceinline__ void load_columns(const IO* row, int width, bool live, Pack<IO, V> (&v)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + threadIdx.x % TPR) * V;
        v[k] = live && c < width ? load_pack<IO, V>(row + c, V, V > 1) : zero_pack<IO, V>();
    }
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(norm_threads(TPR), norm_resident(K, V, TPR, false)) k_norm_fwd(const NormP p) {
    constexpr int RPC = norm_threads(TPR) / TPR;
    constexpr bool HELD = K * V <= 32;                       // weight and bias stay in registers
    __shared__ float red[2][1][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR;
    const long long step = (long long)gridDim.x * RPC;       // rows that all groups take at a time
    long long row = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    int turn = 0;
    const IO* x = static_cast<const IO*>(p.x) + row * p.width;
    IO* y = static_cast<IO*>(p.y) + row * p.width;
    Pack<IO, V> next[K], pw[HELD ? K : 1], pb[HELD ? K : 1];
    load_columns<IO, V, K, TPR>(x, p.width, row < p.rows, next);
    if constexpr (HELD) {
        if (p.weight) load_columns<IO, V, K, TPR>(static_cast<const IO*>(p.weight), p.width, true, pw);
        if (p.bias) load_columns<IO, V, K, TPR>(static_cast<const IO*>(p.bias), p.width, true, pb);
    }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        float f[K][V], s[1] = {0.f}, mean = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            widen(next[k], f[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += f[k][i];
        }
        x += step * p.width;
        if (first + step < p.rows) load_columns<IO, V, K, TPR>(x, p.width, row + step < p.rows, next);
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
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c >= p.width) break;
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = f[k][i] * r;
                if (p.weight) {
                    const Pack<IO, V> w = HELD ? pw[HELD ? k : 0] : load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, V, V > 1);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] *= pick(w, i);
                }
                if (p.bias) {
                    const Pack<IO, V> b = HELD ? pb[HELD ? k : 0] : load_pack<IO, V>(static_cast<const IO*>(p.bias) + c, V, V > 1);
#pragma unroll
                    for (int i = 0; i < V; ++i) o[i] += pick(b, i);
                }
                store_pack(y + c, narrow<IO, V>(o), V, V > 1);
            }
        }
        y += step * p.width;
    }
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(norm_threads(TPR), norm_resident(K, V, TPR, true)) k_norm_bwd(const NormP p) {
    constexpr int NT = norm_threads(TPR), RPC = NT / TPR;
    constexpr bool HELD = K * V <= 16;
    __shared__ float red[2][2][32];
    __shared__ float cols[RPC > 1 ? NT * V * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    long long row = (long long)blockIdx.x * RPC + rg;
    int turn = 0;
    const IO *x = static_cast<const IO*>(p.x) + row * p.width, *dy = static_cast<const IO*>(p.dy) + row * p.width;
    IO* dx = static_cast<IO*>(p.dx) + row * p.width;
    float dw[K][V], db[K][V], nmean = 0.f, nr = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) { dw[k][i] = 0.f; db[k][i] = 0.f; }
    Pack<IO, V> nx[K], ny[K], pw[HELD ? K : 1];
    auto ahead = [&](long long at) {
        const bool live = at < p.rows;
        load_columns<IO, V, K, TPR>(x, p.width, live, nx);
        load_columns<IO, V, K, TPR>(dy, p.width, live, ny);
        nmean = live && !p.rms ? p.stats[at] : 0.f;
        nr = live ? p.stats[p.rows + at] : 0.f;
    };
    ahead(row);
    if constexpr (HELD)
        if (p.weight) load_columns<IO, V, K, TPR>(static_cast<const IO*>(p.weight), p.width, true, pw);
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step, row += step) {
        const float r = nr;
        Pack<IO, V> py[K];
        float xh[K][V], s[2] = {0.f, 0.f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            py[k] = ny[k];
#pragma unroll
            for (int i = 0; i < V; ++i) xh[k][i] = (pick(nx[k], i) - nmean) * r;         // not used past the row's end
        }
        x += step * p.width;
        dy += step * p.width;
        if (first + step < p.rows) ahead(row + step);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            if (c >= p.width) break;
            Pack<IO, V> w;
            if (p.weight) w = HELD ? pw[HELD ? k : 0] : load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, V, V > 1);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = pick(py[k], i), g = p.weight ? d * pick(w, i) : d;
                s[0] = fmaf(g, xh[k][i], s[0]);
                s[1] += g;
                dw[k][i] = fmaf(d, xh[k][i], dw[k][i]);
                db[k][i] += d;
            }
        }
        row_sum<TPR>(s, red, turn);
        const float s1 = s[0] * p.inv, s2 = p.rms ? 0.f : s[1] * p.inv;
        if (row < p.rows) {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c >= p.width) break;
                Pack<IO, V> w;
                if (p.weight) w = HELD ? pw[HELD ? k : 0] : load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, V, V > 1);
                float o[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float d = pick(py[k], i), g = p.weight ? d * pick(w, i) : d;
                    o[i] = r * (g - s2 - xh[k][i] * s1);
                }
                store_pack(dx + c, narrow<IO, V>(o), V, V > 1);
            }
        }
        dx += step * p.width;
    }
    if (!p.part) return;
    float* part = p.part + (size_t)blockIdx.x * 2 * p.width;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        if constexpr (RPC > 1) {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) cols[rg * (TPR * V * K) + (k * TPR + tr) * V + i] = h ? db[k][i] : dw[k][i];
            __syncthreads();
            for (int c = threadIdx.x; c < p.width; c += NT) {
                float t = 0.f;
                for (int g = 0; g < RPC; ++g) t += cols[g * (TPR * V * K) + c];
                part[(size_t)h * p.width + c] = t;
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int c = (k * TPR + tr) * V + i;
                    if (c < p.width) part[(size_t)h * p.width + c] = h ? db[k][i] : dw[k][i];
                }
        }
    }
}

// Columns that a thread loads at a time: 16 bytes where rows are whole groups of them.
int norm_vector(int width, int dtype) {
    const int v = dtype == QD_BF16 ? 8 : 4;
    return width % v == 0 ? v : 1;
}
// Threads per row (TPR) and groups of V columns per thread (K) for a row of n groups: four groups to a lane forward, and eight rather than
// a CTA to a row (no barrier) where there are rows enough to fill the GPU so; two backward, where a column's two sums are registers too.
struct NormShape { int tpr, k; };
NormShape norm_shape(int n, long long rows, bool bwd) {
    const int k = bwd ? 2 : 4;
    for (int tpr = 1; tpr <= 32; tpr *= 2)
        if (n <= k * tpr) return {tpr, k};
    if (bwd && n <= 128) return {32, 4};
    if (n <= 256) return bwd ? NormShape{128, 2} : rows >= kSMs * 16 ? NormShape{32, 8} : NormShape{256, 1};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 4096) return {1024, 4};
    return {1024, 16};
}
// CTAs that stay: no more than are resident at once, of which each leaves one partial of the weights' gradients.
long long norm_ctas(long long rows, const NormShape& s, int resident) {
    const int rpc = norm_threads(s.tpr) / s.tpr;
    const long long groups = (rows + rpc - 1) / rpc, most = kSMs * (long long)resident;
    return groups < most ? groups : most;
}
long long norm_bwd_ctas(long long rows, int width, int dtype) {
    const int V = norm_vector(width, dtype);
    const NormShape s = norm_shape((width + V - 1) / V, rows, true);
    return norm_ctas(rows, s, norm_resident(s.k, V, s.tpr, true));
}

template <typename IO, int V, bool BWD>
cudaError_t launch(const NormP& p, cudaStream_t stream) {
    const NormShape s = norm_shape((p.width + V - 1) / V, p.rows, BWD);
#define QD_NORM(TPR, K)                                                                                                     \
    if (s.tpr == TPR && s.k == K) {                                                                                           \
        const dim3 grid((unsigned)norm_ctas(p.rows, s, norm_resident(K, V, TPR, BWD)));                                        \
        if constexpr (BWD) return launch_overlapped(k_norm_bwd<IO, V, K, TPR>, grid, dim3(norm_threads(TPR)), 0, stream, p);    \
        else return launch_overlapped(k_norm_fwd<IO, V, K, TPR>, grid, dim3(norm_threads(TPR)), 0, stream, p);                  \
    }
    constexpr int L = BWD ? 2 : 4;
    QD_NORM(1, L) QD_NORM(2, L) QD_NORM(4, L) QD_NORM(8, L) QD_NORM(16, L) QD_NORM(32, L)
    if constexpr (BWD) {
        QD_NORM(32, 4) QD_NORM(128, 2)
    } else {
        QD_NORM(32, 8) QD_NORM(256, 1)
    }
    QD_NORM(256, 2) QD_NORM(256, 4) QD_NORM(1024, 4)
    if constexpr (V == 1) QD_NORM(1024, 16)                  // 16384 columns are no more than 4096 groups of more
#undef QD_NORM
    return cudaErrorInvalidValue;
}

}  // namespace

size_t norm_bwd_workspace(long long rows, int width, int dtype) {
    return (size_t)norm_bwd_ctas(rows, width, dtype) * 2 * width * sizeof(float);
}

cudaError_t norm_fwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* bias, void* y, float* stats,
                     float eps, bool rms, cudaStream_t stream) {
    NormP p{};
    p.rows = rows; p.width = width; p.x = x; p.weight = weight; p.bias = bias; p.y = y; p.stats = stats;
    p.eps = eps; p.inv = 1.f / (float)width; p.rms = rms;
    const bool vec = norm_vector(width, dtype) > 1;
    if (dtype == QD_BF16) return vec ? launch<__nv_bfloat16, 8, false>(p, stream) : launch<__nv_bfloat16, 1, false>(p, stream);
    return vec ? launch<float, 4, false>(p, stream) : launch<float, 1, false>(p, stream);
}

cudaError_t norm_bwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* dy, const float* stats, void* dx,
                     float* dweight, float* dbias, float* part, bool rms, cudaStream_t stream) {
    NormP p{};
    p.rows = rows; p.width = width; p.x = x; p.weight = weight; p.dy = dy; p.dx = dx; p.stats = const_cast<float*>(stats);
    p.inv = 1.f / (float)width; p.rms = rms;
    const bool vec = norm_vector(width, dtype) > 1;
    p.part = dweight || dbias ? part : nullptr;
    const long long ctas = norm_bwd_ctas(rows, width, dtype);
    const cudaError_t e = dtype == QD_BF16
                              ? (vec ? launch<__nv_bfloat16, 8, true>(p, stream) : launch<__nv_bfloat16, 1, true>(p, stream))
                              : (vec ? launch<float, 4, true>(p, stream) : launch<float, 1, true>(p, stream));
    if (e != cudaSuccess || !p.part) return e;
    return sum_parts(p.part, (int)ctas, 2LL * width, width, width, 1, dweight, dbias, stream);
}

}  // namespace qd

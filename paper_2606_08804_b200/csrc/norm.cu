// Layer norm over the last dimension, with or without the mean (rms), optional weight and bias:
//   m = mean(x) (0 for rms), r = 1 / sqrt(mean((x - m)^2) + eps), x^ = (x - m) r, y = x^ w + b.
// Backward, with g = dy w:  dx = r (g - x^ mean(g x^) - mean(g))  (the last term not for rms),  dw = sum_rows dy x^,  db = sum_rows dy.
//
// Bound by HBM: a row is read once into registers, where the mean is taken before the squares of what it leaves.  A row belongs to a
// group of 2^k lanes, or to a CTA where it is too wide for a warp.  The backward's CTAs stay and take every gridDim-th row group, so
// that dw and db add up in registers (a thread has the same columns in every row) and one partial per CTA is left, which
// k_sum_parts adds in a fixed order.
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
    bool rms, vec;
};

// Sum over the TPR threads of a row, the same bits in each of them.
template <int TPR>
__device__ __forceinline__ float row_sum(float v, float* red) {
#pragma unroll
    for (int w = (TPR < 32 ? TPR : 32) / 2; w > 0; w >>= 1) v += __shfl_xor_sync(0xffffffffu, v, w);
    if constexpr (TPR > 32) {
        __syncthreads();                                     // red may still be read from the sum before
        if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
        __syncthreads();
        v = threadIdx.x % 32 < TPR / 32 ? red[threadIdx.x % 32] : 0.f;
#pragma unroll
        for (int w = TPR / 64; w > 0; w >>= 1) v += __shfl_xor_sync(0xffffffffu, v, w);
        v = __shfl_sync(0xffffffffu, v, 0);
    }
    return v;
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) k_norm_fwd(const NormP p) {
    constexpr int NT = TPR > 256 ? TPR : 256, RPC = NT / TPR;
    __shared__ float red[32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR;
    const long long row = (long long)blockIdx.x * RPC + threadIdx.x / TPR;
    const bool live = row < p.rows;
    const IO* x = static_cast<const IO*>(p.x) + (live ? row : 0) * p.width;
    float f[K][V];
    float s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + tr) * V;
        widen(live && c < p.width ? load_pack<IO, V>(x + c, p.width - c, p.vec) : zero_pack<IO, V>(), f[k]);
#pragma unroll
        for (int i = 0; i < V; ++i) s += f[k][i];
    }
    float mean = 0.f;
    if (!p.rms) {
        mean = row_sum<TPR>(s, red) * p.inv;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) f[k][i] = (k * TPR + tr) * V + i < p.width ? f[k][i] - mean : 0.f;
    }
    s = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) s = fmaf(f[k][i], f[k][i], s);
    const float r = 1.f / sqrtf(row_sum<TPR>(s, red) * p.inv + p.eps);
    if (!live) return;
    if (tr == 0 && p.stats) { p.stats[row] = mean; p.stats[p.rows + row] = r; }
    IO* y = static_cast<IO*>(p.y) + row * p.width;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + tr) * V;
        if (c >= p.width) break;
        float w[V], b[V], o[V];
        if (p.weight) widen(load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, p.width - c, p.vec), w);
        if (p.bias) widen(load_pack<IO, V>(static_cast<const IO*>(p.bias) + c, p.width - c, p.vec), b);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            o[i] = f[k][i] * r;
            if (p.weight) o[i] *= w[i];
            if (p.bias) o[i] += b[i];
        }
        store_pack(y + c, narrow<IO, V>(o), p.width - c, p.vec);
    }
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(TPR > 256 ? TPR : 256) k_norm_bwd(const NormP p) {
    constexpr int NT = TPR > 256 ? TPR : 256, RPC = NT / TPR;
    __shared__ float red[32];
    __shared__ float cols[RPC > 1 ? NT * V * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    float dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) { dw[k][i] = 0.f; db[k][i] = 0.f; }
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += (long long)gridDim.x * RPC) {
        const long long row = first + rg;
        const bool live = row < p.rows;
        const IO *x = static_cast<const IO*>(p.x) + (live ? row : 0) * p.width, *dy = static_cast<const IO*>(p.dy) + (live ? row : 0) * p.width;
        Pack<IO, V> px[K], py[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            const bool in = live && c < p.width;
            px[k] = in ? load_pack<IO, V>(x + c, p.width - c, p.vec) : zero_pack<IO, V>();
            py[k] = in ? load_pack<IO, V>(dy + c, p.width - c, p.vec) : zero_pack<IO, V>();
        }
        const float mean = live && !p.rms ? p.stats[row] : 0.f, r = live ? p.stats[p.rows + row] : 0.f;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (k * TPR + tr) * V;
            float w[V];
            if (p.weight && c < p.width) widen(load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, p.width - c, p.vec), w);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (c + i >= p.width) continue;              // whatever x^ would be there, it does not count
                const float xh = (pick(px[k], i) - mean) * r, d = pick(py[k], i), g = p.weight ? d * w[i] : d;
                s1 = fmaf(g, xh, s1);
                s2 += g;
                dw[k][i] = fmaf(d, xh, dw[k][i]);
                db[k][i] += d;
            }
        }
        s1 = row_sum<TPR>(s1, red) * p.inv;
        s2 = p.rms ? 0.f : row_sum<TPR>(s2, red) * p.inv;
        if (live) {
            IO* dx = static_cast<IO*>(p.dx) + row * p.width;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = (k * TPR + tr) * V;
                if (c >= p.width) break;
                float w[V], o[V];
                if (p.weight) widen(load_pack<IO, V>(static_cast<const IO*>(p.weight) + c, p.width - c, p.vec), w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float xh = (pick(px[k], i) - mean) * r, d = pick(py[k], i), g = p.weight ? d * w[i] : d;
                    o[i] = r * (g - s2 - xh * s1);
                }
                store_pack(dx + c, narrow<IO, V>(o), p.width - c, p.vec);
            }
        }
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
#pragma unroll
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
// Threads per row (TPR) and groups of V columns per thread (K) for a row of n groups.
struct NormShape { int tpr, k; };
NormShape norm_shape(int n) {
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {32, 1};
    if (n <= 64) return {32, 2};
    if (n <= 128) return {32, 4};
    if (n <= 256) return {256, 1};
    if (n <= 512) return {256, 2};
    if (n <= 1024) return {256, 4};
    if (n <= 4096) return {1024, 4};
    return {1024, 16};
}
// CTAs of the backward: a partial each, so no more than fill the GPU; as many as there are row groups where those are few.
long long norm_bwd_ctas(long long rows, int width, int dtype) {
    const int V = norm_vector(width, dtype);
    const NormShape s = norm_shape((width + V - 1) / V);
    const int nt = s.tpr > 256 ? s.tpr : 256;
    const long long groups = (rows + nt / s.tpr - 1) / (nt / s.tpr), most = kSMs * (long long)(nt == 1024 ? 1 : 4);
    return groups < most ? groups : most;
}

template <typename IO, int V, bool BWD>
cudaError_t launch(const NormP& p, long long ctas, cudaStream_t stream) {
    const NormShape s = norm_shape((p.width + V - 1) / V);
#define QD_NORM(TPR, K)                                                                                                     \
    if (s.tpr == TPR && s.k == K) {                                                                                           \
        constexpr int NT = TPR > 256 ? TPR : 256;                                                                             \
        const long long grid = BWD ? ctas : (p.rows + NT / TPR - 1) / (NT / TPR);                                              \
        return launch_overlapped(BWD ? k_norm_bwd<IO, V, K, TPR> : k_norm_fwd<IO, V, K, TPR>, dim3((unsigned)grid), dim3(NT), 0, stream, p); \
    }
    QD_NORM(8, 1) QD_NORM(16, 1) QD_NORM(32, 1) QD_NORM(32, 2) QD_NORM(32, 4) QD_NORM(256, 1) QD_NORM(256, 2) QD_NORM(256, 4)
    QD_NORM(1024, 4)
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
    p.eps = eps; p.inv = 1.f / (float)width; p.rms = rms; p.vec = norm_vector(width, dtype) > 1;
    if (dtype == QD_BF16) return p.vec ? launch<__nv_bfloat16, 8, false>(p, 0, stream) : launch<__nv_bfloat16, 1, false>(p, 0, stream);
    return p.vec ? launch<float, 4, false>(p, 0, stream) : launch<float, 1, false>(p, 0, stream);
}

cudaError_t norm_bwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* dy, const float* stats, void* dx,
                     float* dweight, float* dbias, float* part, bool rms, cudaStream_t stream) {
    NormP p{};
    p.rows = rows; p.width = width; p.x = x; p.weight = weight; p.dy = dy; p.dx = dx; p.stats = const_cast<float*>(stats);
    p.inv = 1.f / (float)width; p.rms = rms; p.vec = norm_vector(width, dtype) > 1;
    p.part = dweight || dbias ? part : nullptr;
    const long long ctas = norm_bwd_ctas(rows, width, dtype);
    const cudaError_t e = dtype == QD_BF16
                              ? (p.vec ? launch<__nv_bfloat16, 8, true>(p, ctas, stream) : launch<__nv_bfloat16, 1, true>(p, ctas, stream))
                              : (p.vec ? launch<float, 4, true>(p, ctas, stream) : launch<float, 1, true>(p, ctas, stream));
    if (e != cudaSuccess || !p.part) return e;
    return sum_parts(p.part, (int)ctas, 2LL * width, width, width, 1, dweight, dbias, stream);
}

}  // namespace qd

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

__host__ __device__ constexpr int norm_threads(int tpr) { return tpr > 256 ? tpr : 256; }
// CTAs to an SM that the register budget is made for
__host__ __device__ constexpr int norm_fwd_ctas(int kv, int tpr) { return tpr > 256 ? 1 : kv <= 8 ? 5 : kv <= 16 ? 3 : 2; }
__host__ __device__ constexpr int norm_bwd_resident(int kv, int tpr) { return tpr > 256 ? 1 : kv <= 8 ? 3 : kv <= 16 ? 2 : 1; }

// Sums of a and b over the TPR threads of a row, the same bits in each of them.  One barrier: `turn` alternates between two halves of red,
// and who writes a half again has passed the barrier after everybody read it.
template <int TPR>
__device__ __forceinline__ float2 row_sum(float a, float b, float2 (*red)[32], int& turn) {
#pragma unroll
    for (int w = (TPR < 32 ? TPR : 32) / 2; w > 0; w >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, w);
        b += __shfl_xor_sync(0xffffffffu, b, w);
    }
    if constexpr (TPR > 32) {
        if ((threadIdx.x & 31) == 0) red[turn][threadIdx.x >> 5] = make_float2(a, b);
        __syncthreads();
        const float2 v = red[turn][threadIdx.x % (TPR / 32)];
        turn ^= 1;
        a = v.x;
        b = v.y;
#pragma unroll
        for (int w = TPR / 64; w > 0; w >>= 1) {
            a += __shfl_xor_sync(0xffffffffu, a, w);
            b += __shfl_xor_sync(0xffffffffu, b, w);
        }
    }
    return make_float2(a, b);
}
template <typename IO, int V, int K, int TPR>
__device__ __forceinline__ void load_norm_row(const NormP& p, const void* base, long long row, Pack<IO, V> (&v)[K]) {
    const IO* x = static_cast<const IO*>(base) + row * p.width;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (k * TPR + threadIdx.x % TPR) * V;
        v[k] = row < p.rows && c < p.width ? load_pack<IO, V>(x + c, p.width - c, p.vec) : zero_pack<IO, V>();
    }
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(norm_threads(TPR), norm_fwd_ctas(K * V, TPR)) k_norm_fwd(const NormP p) {
    constexpr int RPC = norm_threads(TPR) / TPR;
    constexpr bool AHEAD = K * V <= 32 && TPR <= 256;                      // the row after this one is on its way; more would not fit the registers
    __shared__ float2 red[2][32];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    int turn = 0;
    Pack<IO, V> next[K];
    load_norm_row<IO, V, K, TPR>(p, p.x, (long long)blockIdx.x * RPC + rg, next);
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step) {
        const long long row = first + rg;
        float f[K][V], s = 0.f, sq = 0.f;
        if (!AHEAD && first != (long long)blockIdx.x * RPC) load_norm_row<IO, V, K, TPR>(p, p.x, row, next);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            widen(next[k], f[k]);
#pragma unroll
            for (int i = 0; i < V; ++i) s += f[k][i];
        }
        if (AHEAD && first + step < p.rows) load_norm_row<IO, V, K, TPR>(p, p.x, row + step, next);
        float mean = 0.f;
        if (!p.rms) {
            mean = row_sum<TPR>(s, 0.f, red, turn).x * p.inv;
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) f[k][i] = (k * TPR + tr) * V + i < p.width ? f[k][i] - mean : 0.f;
        }
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) sq = fmaf(f[k][i], f[k][i], sq);
        const float r = 1.f / sqrtf(row_sum<TPR>(sq, 0.f, red, turn).x * p.inv + p.eps);
        if (row >= p.rows) continue;
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
}

template <typename IO, int V, int K, int TPR>
__global__ void __launch_bounds__(norm_threads(TPR), norm_bwd_resident(K * V, TPR)) k_norm_bwd(const NormP p) {
    constexpr int NT = norm_threads(TPR), RPC = NT / TPR;
    constexpr bool AHEAD = K * V <= 16 && TPR <= 256;
    __shared__ float2 red[2][32];
    __shared__ float cols[RPC > 1 ? NT * V * K : 1];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int tr = threadIdx.x % TPR, rg = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * RPC;
    int turn = 0;
    float dw[K][V], db[K][V];
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) { dw[k][i] = 0.f; db[k][i] = 0.f; }
    Pack<IO, V> px[K], py[K], nx[AHEAD ? K : 1], ny[AHEAD ? K : 1];
    float2 st = {0.f, 0.f}, nst = {0.f, 0.f};
    auto stats = [&](long long row) {
        return row < p.rows ? make_float2(p.rms ? 0.f : p.stats[row], p.stats[p.rows + row]) : make_float2(0.f, 0.f);
    };
    auto ahead = [&](long long row) {
        if constexpr (AHEAD) {
            load_norm_row<IO, V, K, TPR>(p, p.x, row, nx);
            load_norm_row<IO, V, K, TPR>(p, p.dy, row, ny);
            nst = stats(row);
        }
    };
    ahead((long long)blockIdx.x * RPC + rg);
    for (long long first = (long long)blockIdx.x * RPC; first < p.rows; first += step) {
        const long long row = first + rg;
        if constexpr (AHEAD) {
#pragma unroll
            for (int k = 0; k < K; ++k) { px[k] = nx[k]; py[k] = ny[k]; }
            st = nst;
            if (first + step < p.rows) ahead(row + step);
        } else {
            load_norm_row<IO, V, K, TPR>(p, p.x, row, px);
            load_norm_row<IO, V, K, TPR>(p, p.dy, row, py);
            st = stats(row);
        }
        const float mean = st.x, r = st.y;
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
        const float2 sums = row_sum<TPR>(s1, s2, red, turn);
        s1 = sums.x * p.inv;
        s2 = p.rms ? 0.f : sums.y * p.inv;
        if (row >= p.rows) continue;
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
// Threads per row (TPR) and groups of V columns per thread (K) for a row of n groups.  Forward, a warp a row up to eight groups to a lane (no
// barrier) where there are rows enough to fill the GPU so; backward, where a thread's columns each need two sums, four.
struct NormShape { int tpr, k; };
NormShape norm_shape(int n, long long rows, bool bwd) {
    if (n <= 8) return {8, 1};
    if (n <= 16) return {16, 1};
    if (n <= 32) return {32, 1};
    const bool many = rows >= kSMs * 16;
    if (many || bwd) {
        if (n <= 64) return {32, 2};
        if (n <= 128) return {32, 4};
        if (n <= 256 && !bwd) return {32, 8};
    }
    if (n <= 256) return {256, 1};
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
    return norm_ctas(rows, s, norm_bwd_resident(s.k * V, s.tpr));
}

template <typename IO, int V, bool BWD>
cudaError_t launch(const NormP& p, cudaStream_t stream) {
    const NormShape s = norm_shape((p.width + V - 1) / V, p.rows, BWD);
#define QD_NORM(TPR, K)                                                                                                     \
    if (s.tpr == TPR && s.k == K) {                                                                                           \
        constexpr int resident = BWD ? norm_bwd_resident(K * V, TPR) : norm_fwd_ctas(K * V, TPR);                              \
        const dim3 grid((unsigned)norm_ctas(p.rows, s, resident));                                                             \
        if constexpr (BWD) return launch_overlapped(k_norm_bwd<IO, V, K, TPR>, grid, dim3(norm_threads(TPR)), 0, stream, p);    \
        else return launch_overlapped(k_norm_fwd<IO, V, K, TPR>, grid, dim3(norm_threads(TPR)), 0, stream, p);                  \
    }
    QD_NORM(8, 1) QD_NORM(16, 1) QD_NORM(32, 1) QD_NORM(32, 2) QD_NORM(32, 4) QD_NORM(256, 1) QD_NORM(256, 2) QD_NORM(256, 4)
    QD_NORM(1024, 4)
    if constexpr (!BWD) QD_NORM(32, 8)
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
    if (dtype == QD_BF16) return p.vec ? launch<__nv_bfloat16, 8, false>(p, stream) : launch<__nv_bfloat16, 1, false>(p, stream);
    return p.vec ? launch<float, 4, false>(p, stream) : launch<float, 1, false>(p, stream);
}

cudaError_t norm_bwd(long long rows, int width, int dtype, const void* x, const void* weight, const void* dy, const float* stats, void* dx,
                     float* dweight, float* dbias, float* part, bool rms, cudaStream_t stream) {
    NormP p{};
    p.rows = rows; p.width = width; p.x = x; p.weight = weight; p.dy = dy; p.dx = dx; p.stats = const_cast<float*>(stats);
    p.inv = 1.f / (float)width; p.rms = rms; p.vec = norm_vector(width, dtype) > 1;
    p.part = dweight || dbias ? part : nullptr;
    const long long ctas = norm_bwd_ctas(rows, width, dtype);
    const cudaError_t e = dtype == QD_BF16
                              ? (p.vec ? launch<__nv_bfloat16, 8, true>(p, stream) : launch<__nv_bfloat16, 1, true>(p, stream))
                              : (p.vec ? launch<float, 4, true>(p, stream) : launch<float, 1, true>(p, stream));
    if (e != cudaSuccess || !p.part) return e;
    return sum_parts(p.part, (int)ctas, 2LL * width, width, width, 1, dweight, dbias, stream);
}

}  // namespace qd

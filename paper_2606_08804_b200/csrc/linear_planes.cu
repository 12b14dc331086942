// Linear attention, fp32-accurate: a walk (linear.cuh) per CTA over chunks of 64 tokens, for 32 columns of the state.  All products are
// products of bf16 planes on the warp-level tensor instruction (planes.cuh), an fp32 matrix three planes; the state stays in fp32 registers,
// to which a chunk's sum is added, and is written as planes for the next chunk's a S.
// A chunk of 64 x 128 x 32 takes 7.6 us: its 1.2 million products of elements, six times over for the planes, keep the tensor pipe busy half of
// that, what is written as planes and the barriers in between is the rest; a b^T is made once for every 32 columns.  2 x 2048 tokens, 16 heads
// of 128 x 128: forward 247 us, backward 722 (bytes 21 and 36); 2 x 1000, 4 heads of 64 x 64 in segments: 21 and 46, latency.
#include "linear.cuh"
#include "planes.cuh"
#include "split_common.cuh"

namespace qd {
namespace {

constexpr int kRows = 64, kCols = 32, kPlanesThreads = 256;

// four neighbours of a tile from global memory, rows >= live as zeros; on their way in registers, then into planes
template <int W>
struct Rows4 {
    static constexpr int kN = kRows * W / 4 / kPlanesThreads;
    float4 r[kN];
    __device__ __forceinline__ void get(const float* src, size_t stride, int live) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int id = i * kPlanesThreads + threadIdx.x, row = id / (W / 4), c = id % (W / 4) * 4;
            r[i] = row < live ? *reinterpret_cast<const float4*>(src + row * stride + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
    }
    // zeros for elements that are infinite or NaN, which f(row, column) hears of
    template <class F> __device__ __forceinline__ void settle(F f) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            float* const x = &r[i].x;
            const float sum = 0.f * x[0] + 0.f * x[1] + 0.f * x[2] + 0.f * x[3];
            if (sum == 0.f) continue;
            const int id = i * kPlanesThreads + threadIdx.x;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!(fabsf(x[e]) < INFINITY)) {
                    x[e] = 0.f;
                    f(id / (W / 4), id % (W / 4) * 4 + e);
                }
        }
    }
    template <class P> __device__ __forceinline__ void put(const P& d) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int id = i * kPlanesThreads + threadIdx.x;
            d.st4(id / (W / 4), id % (W / 4) * 4, r[i]);
        }
    }
    template <class P> __device__ __forceinline__ void put(const P& d, const float* factor) const {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int id = i * kPlanesThreads + threadIdx.x;
            const float f = factor[id / (W / 4)];
            d.st4(id / (W / 4), id % (W / 4) * 4, make_float4(f * r[i].x, f * r[i].y, f * r[i].z, f * r[i].w));
        }
    }
};

// acc += A B as pmm does (planes.cuh), of three planes each.  The tensor instruction cuts as it adds, so the products go to three sums by their
// size, and none of them adds small products to a large sum; for all columns before the next product, so that none waits for the one before.
// Of 128 x 128, outputs are 2e-7 of their length off for 1.1e-6 with one sum; 244 us for 235 at 2 x 2048 tokens of 16 heads, 154 for 169 at 4 x 2048
// tokens of 16 heads of 64 x 64.
template <bool AT, bool BT, int NTL, class MA, class MB>
__device__ __forceinline__ void product(float (&acc)[1][NTL][4], const MA& A, const MB& B, int m0, int n0, int k1, int kb = 0) {
    static_assert(MA::NP == 3 && MB::NP == 3 && NTL % 2 == 0, "three planes, columns in pairs of 8");
    const int lane = threadIdx.x & 31;
    const __nv_bfloat16* pa = A.p + (AT ? ((lane & 7) + (lane >> 4) * 8) * MA::LD + m0 + ((lane >> 3) & 1) * 8 : (m0 + (lane & 15)) * MA::LD + (lane >> 4) * 8);
    const __nv_bfloat16* pb = B.p + (BT ? (lane & 15) * MB::LD + n0 + (lane >> 4) * 8 : (n0 + (lane & 7) + (lane >> 4) * 8) * MB::LD + ((lane >> 3) & 1) * 8);
    float less[2][NTL][4];
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int j = 0; j < NTL; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) less[s][j][e] = 0.f;
#pragma unroll 2
    for (int k0 = kb; k0 < k1; k0 += 16) {
        uint32_t a[3][4], b[NTL / 2][3][4];
#pragma unroll
        for (int x = 0; x < 3; ++x) sm100::ldsm4<AT>(pa + x * MA::PS + (AT ? k0 * MA::LD : k0), a[x]);
#pragma unroll
        for (int j = 0; j < NTL / 2; ++j)
#pragma unroll
            for (int y = 0; y < 3; ++y) sm100::ldsm4<BT>(pb + y * MB::PS + (BT ? k0 * MB::LD + 16 * j : 16 * j * MB::LD + k0), b[j][y]);
        auto all = [&](float (&to)[NTL][4], int x, int y) {
#pragma unroll
            for (int j = 0; j < NTL; ++j) mma_bf16(to[j], a[x], b[j / 2][y] + 2 * (j & 1));
        };
        all(less[1], 0, 2);
        all(less[0], 0, 1);
        all(acc[0], 0, 0);
        all(less[1], 1, 1);
        all(less[0], 1, 0);
        all(less[1], 2, 0);
    }
#pragma unroll
    for (int j = 0; j < NTL; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[0][j][e] += less[0][j][e] + less[1][j][e];
}

template <int DB>
struct PlanesLayout {
    typedef Planes<kRows, DB, 3> Wide;
    typedef Planes<kRows, kCols, 3> Slice;
    typedef Planes<kRows, kRows, 3> Square;
    typedef Planes<DB, kCols, 3> State;
    static constexpr int kA = 0, kB = kA + Wide::kBytes, kC = kB + Wide::kBytes, kCh = kC + Slice::kBytes, kP = kCh + Slice::kBytes,
                         kS = kP + Square::kBytes, kBytes = kS + State::kBytes;
};

template <int DB, int DC>
__global__ void __launch_bounds__(kPlanesThreads, 1) k_linear_planes(const LinearP p) {
    typedef PlanesLayout<DB> L;
    extern __shared__ __align__(16) unsigned char smem_planes[];
    __shared__ float s_d[kRows], s_rho[kRows], s_kappa[kRows];
    __shared__ int s_first[kCols];                             // of every column of c the first element that is infinite or NaN, in the walk's order
    __shared__ int s_unfit;
    const typename L::Wide A(smem_planes + L::kA), B(smem_planes + L::kB);
    const typename L::Slice Cc(smem_planes + L::kC);
    const typename L::Slice Ch(smem_planes + L::kCh);
    const typename L::Square P(smem_planes + L::kP);
    const typename L::State S(smem_planes + L::kS);
    constexpr int kSlices = DC / kCols;
    const int cta = blockIdx.x / p.walks, slice = cta % kSlices, segment = cta / kSlices % p.segments, bh = cta / kSlices / p.segments;
    const LinearWalk w = p.w[blockIdx.x % p.walks];
    const int b = bh / p.H, h = bh % p.H, j0 = slice * kCols, tid = threadIdx.x, warp = tid >> 5;
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const float g = p.g[h], g2 = g * 1.4426950408889634f;
    if (p.clear && blockIdx.x == 0 && tid == 0) *p.status = 0;
    // the sums of the segment that no other begins with are not asked for
    if (!w.out && segment == (w.reverse ? 0 : p.segments - 1)) return;

    // a warp's part of the state: 16 rows, 32 columns (16, where there are 64 rows)
    constexpr int NS = DB == 128 ? 4 : 2;
    const int sm = DB == 128 ? 16 * warp : 16 * (warp >> 1), sn = DB == 128 ? 0 : 16 * (warp & 1);
    float st[1][NS][4];
    const int size = DB * DC;
    auto place = [&](int r, int c) { return w.flip ? (j0 + c) * DB + r : r * DC + j0 + c; };
    const float* entry = w.s0 ? w.s0 + ((size_t)bh * p.segments + segment) * size : nullptr;
    each(st, sm, sn, [&](int r, int c, float& x, float& y) {
        x = entry ? __ldcg(entry + place(r, c)) : 0.f;
        y = entry ? __ldcg(entry + place(r, c + 1)) : 0.f;
        S.st2(r, c, x, y);
    });
    if (tid < kRows) s_d[tid] = p.scale * decay_power(g2, tid);
    if (tid < kCols) s_first[tid] = 0x7fffffff;
    if (tid == 0) s_unfit = 0;

    const int first = segment * p.length, end = min(p.T, first + p.length), chunks = (end - first + kRows - 1) / kRows;
    const size_t ld_b = (size_t)p.H * DB, ld_c = (size_t)p.H * DC;
    const float *ga = static_cast<const float*>(w.a), *gb = static_cast<const float*>(w.b), *gc = static_cast<const float*>(w.c);
    Rows4<DB> ra, rb;
    Rows4<kCols> rc;
    auto fetch = [&](int n) {
        const int t0 = first + (w.reverse ? chunks - 1 - n : n) * kRows, live = min(kRows, end - t0);
        const size_t row = (size_t)b * p.T + t0;
        if (w.out) ra.get(ga + row * ld_b + (size_t)h * DB, ld_b, live);
        rb.get(gb + row * ld_b + (size_t)h * DB, ld_b, live);
        rc.get(gc + row * ld_c + (size_t)h * DC + j0, ld_c, live);
    };
    fetch(0);
    for (int n = 0; n < chunks; ++n) {
        const int t0 = first + (w.reverse ? chunks - 1 - n : n) * kRows, live = min(kRows, end - t0);
        if (tid < kRows) {
            const float fall = tid < live ? decay_power(g2, live - 1 - tid) : 0.f, rise = tid < live ? p.scale * decay_power(g2, tid + 1) : 0.f;
            s_rho[tid] = w.reverse ? fall : rise;
            s_kappa[tid] = w.reverse ? rise : fall;
        }
        __syncthreads();                                       // and the chunk before has been read
        if (w.out) ra.put(A);
        rb.put(B);
        rc.put(Ch, s_kappa);
        // out's rows before a token take nothing of it, also where it is infinite or NaN; from there on its column of out is NaN
        rc.settle([&](int r, int c) {
            atomicMin(s_first + c, n * kRows + (w.reverse ? kRows - 1 - r : r));
            s_unfit = 1;
        });
        rc.put(Cc);
        __syncthreads();
        if (n + 1 < chunks) fetch(n + 1);
        if (w.out) {
            float acc[1][4][4];
            const int m0 = 16 * (warp >> 1), n0 = 32 * (warp & 1);
            zero(acc);
            product<false, false>(acc, A, B, m0, n0, DB);
            each(acc, m0, n0, [&](int r, int c, float& x, float& y) {
                const int u = w.reverse ? c - r : r - c, v = w.reverse ? u + 1 : u - 1;
                // past the end products are 0 and factors, of heads that grow, infinite
                P.st2(r, c, u >= 0 && c < live ? x * s_d[u] : 0.f, v >= 0 && c + 1 < live ? y * s_d[v] : 0.f);
            });
            __syncthreads();
            float in[1][2][4], out[1][2][4];
            const int o0 = 16 * (warp & 1);
            zero(in);
            zero(out);
            product<false, true>(in, P, Cc, m0, o0, w.reverse ? kRows : m0 + 16, w.reverse ? m0 : 0);
            product<false, true>(out, A, S, m0, o0, DB);
            float* o = static_cast<float*>(w.out) + ((size_t)b * p.T + t0) * ld_c + (size_t)h * DC + j0;
            each2(in, out, m0, o0, [&](int r, int c, float x, float y, float x2, float y2) {
                if (r >= live) return;
                const float f = s_rho[r];
                x = fmaf(f, x2, x);
                y = fmaf(f, y2, y);
                if (s_unfit) {
                    const int at = n * kRows + (w.reverse ? kRows - 1 - r : r);
                    if (at >= s_first[c]) x = NAN;
                    if (at >= s_first[c + 1]) y = NAN;
                }
                *reinterpret_cast<float2*>(o + r * ld_c + c) = make_float2(x, y);
            });
        }
        float add[1][NS][4];
        zero(add);
        product<true, true>(add, B, Ch, sm, sn, kRows);
        if (w.out) __syncthreads();                            // the state has been read
        const Keep keep = keep_power(g, live);
        each2(st, add, sm, sn, [&](int r, int c, float& x, float& y, float x2, float y2) {
            x = kept(keep, x, x2);
            y = kept(keep, y, y2);
            if (w.out) S.st2(r, c, x, y);
        });
    }
    float* left = w.out ? segment == (w.reverse ? 0 : p.segments - 1) && w.sT ? w.sT + (size_t)bh * size : nullptr
                        : w.ends + ((size_t)bh * p.segments + segment) * size;
    if (left)
        each(st, sm, sn, [&](int r, int c, float& x, float& y) {
            left[place(r, c)] = x;
            left[place(r, c + 1)] = y;
        });
}

template <int DB, int DC>
cudaError_t launch(const LinearP& p, cudaStream_t stream) {
    constexpr int bytes = PlanesLayout<DB>::kBytes;
    const auto kern = k_linear_planes<DB, DC>;
    const cudaError_t e = set_max_smem_once((const void*)kern, bytes);
    if (e != cudaSuccess) return e;
    return launch_overlapped(kern, dim3((unsigned)(p.BH * p.segments * (DC / kCols) * p.walks)), dim3(kPlanesThreads), bytes, stream, p);
}

}  // namespace

cudaError_t linear_planes(const LinearP& p, int db, int dc, cudaStream_t stream) {
    if (db == 128) return dc == 128 ? launch<128, 128>(p, stream) : launch<128, 64>(p, stream);
    return dc == 128 ? launch<64, 128>(p, stream) : launch<64, 64>(p, stream);
}

}  // namespace qd

// Single tokens of the selective scan (scan.cuh), state [B, D, N] updated in place; also several tokens per call, the state read and written
// once.  A lane has four states of a channel, 1 to 16 lanes (LN) a channel, in R sequences: with several, their states are on their way
// at once, A is read once for them, and what is per channel (softplus, gate) is shared out over the lanes.  A token's arithmetic depends
// neither on R nor on how many tokens a call has.
// Bound by HBM: 8 N bytes of state per channel, one exponential and five operations per state.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

struct StepsP {
    int B, S, D, N, G;
    const void *u, *dt, *Bm, *Cm, *z;
    const float *A, *skip, *bias;
    float* state;
    void* y;
    bool softplus, vecn;
};

template <typename IO, int LN, int R>
__global__ void __launch_bounds__(256, 4) k_scan_steps(const StepsP p) {
    constexpr int M = R > LN ? R / LN : 1;                 // sequences whose channel a lane does alone: l, l + LN, ..
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const long long i = (long long)blockIdx.x * (256 / LN) + threadIdx.x / LN;      // a channel of R sequences
    const long long rows = (p.B + R - 1) / R;
    const bool live = i < rows * p.D;
    const int l = threadIdx.x % LN, n0 = l * 4, b0 = live ? (int)(i / p.D) * R : 0, ch = live ? (int)(i % p.D) : 0, g = ch / (p.D / p.G);
    const int left = live ? p.N - n0 : 0;
    const IO *u = static_cast<const IO*>(p.u), *dt = static_cast<const IO*>(p.dt), *z = static_cast<const IO*>(p.z);
    const IO *Bm = static_cast<const IO*>(p.Bm), *Cm = static_cast<const IO*>(p.Cm);
    IO* y = static_cast<IO*>(p.y);
    float h[R][4], a2[4];
#pragma unroll
    for (int r = 0; r < R; ++r)
        widen(left > 0 && b0 + r < p.B ? load_pack<float, 4>(p.state + ((size_t)(b0 + r) * p.D + ch) * p.N + n0, left, p.vecn) : zero_pack<float, 4>(), h[r]);
    widen(left > 0 ? load_pack<float, 4>(p.A + (size_t)ch * p.N + n0, left, p.vecn) : zero_pack<float, 4>(), a2);
#pragma unroll
    for (float& a : a2) a *= kLog2e;
    const float bias = p.bias ? p.bias[ch] : 0.f, skip = p.skip ? p.skip[ch] : 0.f;
#pragma unroll 1
    for (int s = 0; s < p.S; ++s) {
        Pack<IO, 4> fb[R], fc[R];
        float uu[M], v[M], zz[M], x[M];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const size_t at = (((size_t)(b0 + r) * p.S + s) * p.G + g) * p.N + n0;
            const bool in = left > 0 && b0 + r < p.B;
            fb[r] = in ? load_pack<IO, 4>(Bm + at, left, p.vecn) : zero_pack<IO, 4>();
            fc[r] = in ? load_pack<IO, 4>(Cm + at, left, p.vecn) : zero_pack<IO, 4>();
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int r = (l + m * LN) % R;
            const size_t at = ((size_t)(b0 + r) * p.S + s) * p.D + ch;
            const bool in = live && b0 + r < p.B;
            uu[m] = in ? ld(u, at) : 0.f;
            v[m] = in ? ld(dt, at) + bias : 0.f;
            zz[m] = in && z ? ld(z, at) : 0.f;
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (p.softplus) v[m] = softplus(v[m], v[m]).x;
            x[m] = v[m] * uu[m];
        }
        float o[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const float vr = __shfl_sync(0xffffffffu, v[r / LN % M], r % LN, LN), xr = __shfl_sync(0xffffffffu, x[r / LN % M], r % LN, LN);
            o[r] = 0.f;
#pragma unroll
            for (int n = 0; n < 4; ++n) {
                h[r][n] = fmaf(exp2_unit(vr * a2[n]), h[r][n], xr * pick(fb[r], n));
                o[r] = fmaf(h[r][n], pick(fc[r], n), o[r]);
            }
        }
        // over the lanes of a channel, in the order 2, 1, 4, 8; with four sequences a lane ends with those that it does alone
        float k[M];
        if constexpr (R == 4 && LN >= 4) {
            const bool b1 = l & 2, b1_ = l & 1;
            float w[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) w[e] = (b1 ? o[2 + e] : o[e]) + __shfl_xor_sync(0xffffffffu, b1 ? o[e] : o[2 + e], 2);
            k[0] = (b1_ ? w[1] : w[0]) + __shfl_xor_sync(0xffffffffu, b1_ ? w[0] : w[1], 1);
        } else if constexpr (R == 4 && LN == 2) {
#pragma unroll
            for (int m = 0; m < 2; ++m) k[m] = (l ? o[2 * m + 1] : o[2 * m]) + __shfl_xor_sync(0xffffffffu, l ? o[2 * m] : o[2 * m + 1], 1);
        } else {
#pragma unroll
            for (int m = 0; m < M; ++m) k[m] = o[m];
            if constexpr (LN >= 4) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 2);
            if constexpr (LN >= 2) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 1);
        }
        if constexpr (LN >= 8) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 4);
        if constexpr (LN >= 16) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 8);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int r = l + m * LN;
            float e = fmaf(skip, uu[m], k[m]);
            if (z) e *= zz[m] * gate_sigmoid(zz[m]);
            if (live && r < R && b0 + r < p.B) st(y, ((size_t)(b0 + r) * p.S + s) * p.D + ch, e);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (left > 0 && b0 + r < p.B) store_pack(p.state + ((size_t)(b0 + r) * p.D + ch) * p.N + n0, narrow<float, 4>(h[r]), left, p.vecn);
}

template <typename IO, int LN, int R>
cudaError_t launch(const StepsP& p, cudaStream_t stream) {
    const long long channels = (long long)((p.B + R - 1) / R) * p.D, ctas = (channels + 256 / LN - 1) / (256 / LN);
    return launch_overlapped(k_scan_steps<IO, LN, R>, dim3((unsigned)ctas), dim3(256), 0, stream, p);
}
template <typename IO, int LN>
cudaError_t launch(const StepsP& p, cudaStream_t stream) {
    // four sequences to a lane where they fill the GPU all the same
    if (p.B >= 4 && (long long)p.B / 4 * p.D * LN >= kSMs * 1024LL) return launch<IO, LN, 4>(p, stream);
    return launch<IO, LN, 1>(p, stream);
}
template <typename IO>
cudaError_t launch(const StepsP& p, cudaStream_t stream) {
    const int lanes = (p.N + 3) / 4;
    return lanes <= 1   ? launch<IO, 1>(p, stream)
           : lanes <= 2 ? launch<IO, 2>(p, stream)
           : lanes <= 4 ? launch<IO, 4>(p, stream)
           : lanes <= 8 ? launch<IO, 8>(p, stream)
                        : launch<IO, 16>(p, stream);
}

}  // namespace

cudaError_t scan_steps(const ScanArgs& a) {
    StepsP p{};
    p.B = a.s.B; p.S = a.s.T; p.D = a.s.D; p.N = a.s.N; p.G = a.s.G;
    p.u = a.u; p.dt = a.dt; p.Bm = a.Bm; p.Cm = a.Cm; p.z = a.z; p.A = a.A; p.skip = a.D; p.bias = a.dt_bias;
    p.state = a.hT; p.y = a.y; p.softplus = a.softplus; p.vecn = a.s.N % 4 == 0;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.stream) : launch<float>(p, a.stream);
}

}  // namespace qd

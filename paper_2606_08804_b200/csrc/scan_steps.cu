// Single tokens of the selective scan (scan.cuh), state [B, D, N] updated in place; also several tokens per call, the state read and written
// once.  A lane has four states of a channel, 1 to 16 lanes a channel; a token's arithmetic does not depend on how many tokens a call has.
// Bound by HBM: 8 N bytes of state per channel, one exponential and five operations per state.
#include "scan.cuh"

namespace qd {
namespace {
using namespace scan;

template <typename IO, int LN>
__global__ void __launch_bounds__(256) k_scan_steps(int B, int S, int D, int N, int G, const IO* u, const IO* dt, const float* A, const IO* Bm,
                                                    const IO* Cm, const float* skip, const IO* z, const float* dt_bias, float* state, IO* y,
                                                    bool sp, bool vecn) {
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const long long i = (long long)blockIdx.x * (256 / LN) + threadIdx.x / LN;      // channel of a sequence
    const bool live = i < (long long)B * D;
    const int n0 = threadIdx.x % LN * 4, left = live ? N - n0 : 0;
    const int b = live ? (int)(i / D) : 0, ch = live ? (int)(i % D) : 0, g = ch / (D / G);
    float* hp = state + ((size_t)b * D + ch) * N + n0;
    float h[4] = {0.f, 0.f, 0.f, 0.f}, a2[4] = {0.f, 0.f, 0.f, 0.f};
    if (left > 0) {
        widen(load_pack<float, 4>(hp, left, vecn), h);
        widen(load_pack<float, 4>(A + (size_t)ch * N + n0, left, vecn), a2);
    }
    const float bias = live && dt_bias ? dt_bias[ch] : 0.f, sk = live && skip ? skip[ch] : 0.f;
#pragma unroll
    for (int n = 0; n < 4; ++n) a2[n] *= kLog2e;
    for (int s = 0; s < S; ++s) {
        const size_t row = (size_t)b * S + s, at = row * D + ch, bc = (row * G + g) * N + n0;
        float fb[4] = {0.f, 0.f, 0.f, 0.f}, fc[4] = {0.f, 0.f, 0.f, 0.f}, uu = 0.f, v = 0.f, zz = 0.f;
        if (left > 0) {
            widen(load_pack<IO, 4>(Bm + bc, left, vecn), fb);
            widen(load_pack<IO, 4>(Cm + bc, left, vecn), fc);
        }
        if (live) {
            uu = ld(u, at);
            v = ld(dt, at) + bias;
            if (z) zz = ld(z, at);
        }
        if (sp) v = softplus(v);
        const float x = v * uu;
        float o = 0.f;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
            h[n] = fmaf(exp2_unit(v * a2[n]), h[n], x * fb[n]);
            o = fmaf(h[n], fc[n], o);
        }
#pragma unroll
        for (int w = LN / 2; w > 0; w >>= 1) o += __shfl_xor_sync(0xffffffffu, o, w);
        o = fmaf(sk, uu, o);
        if (z) o *= zz * sigmoid(zz);
        if (live && n0 == 0) st(y, at, o);
    }
    if (left > 0) store_pack(hp, narrow<float, 4>(h), left, vecn);
}

template <typename IO, int LN>
cudaError_t launch(const ScanArgs& a) {
    const long long ctas = ((long long)a.s.B * a.s.D + 256 / LN - 1) / (256 / LN);
    return launch_overlapped(k_scan_steps<IO, LN>, dim3((unsigned)ctas), dim3(256), 0, a.stream, a.s.B, a.s.T, a.s.D, a.s.N, a.s.G,
                             static_cast<const IO*>(a.u), static_cast<const IO*>(a.dt), a.A, static_cast<const IO*>(a.Bm),
                             static_cast<const IO*>(a.Cm), a.D, static_cast<const IO*>(a.z), a.dt_bias, a.hT, static_cast<IO*>(a.y),
                             a.softplus, a.s.N % 4 == 0);
}
template <typename IO>
cudaError_t launch(const ScanArgs& a) {
    const int lanes = (a.s.N + 3) / 4;
    return lanes <= 1 ? launch<IO, 1>(a) : lanes <= 2 ? launch<IO, 2>(a) : lanes <= 4 ? launch<IO, 4>(a) : lanes <= 8 ? launch<IO, 8>(a) : launch<IO, 16>(a);
}

}  // namespace

cudaError_t scan_steps(const ScanArgs& a) { return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(a) : launch<float>(a); }

}  // namespace qd

// Single tokens of the selective scan (scan.cuh), state [B, D, N] updated in place; also several tokens per call, the state read and written
// once.  A lane has four states of a channel, 1 to 16 lanes (LN) a channel, in two sequences (R): both states are on their way at once, A is
// read once for them, and what is per channel (softplus, gate) is shared out over the lanes.  A token's arithmetic depends neither on R nor
// on how many tokens a call has.
// Bound by HBM: 8 N bytes of state per channel, one exponential and five operations per state; but these are 40 instructions a lane and
// sequence, and what a lane does once counts as much as they do: hence no division of 64-bit numbers, no loop for a single token, no lane
// that has nothing to do (it repeats what is there).  256 x 2048 channels of 16 states: 12.3 us, 5.8 TB/s; with four sequences a lane, of
// which not all fit in registers, 14 to 19, with one 17.
#include "scan.cuh"

#include <type_traits>

namespace qd {
namespace {
using namespace scan;

constexpr int kStepThreads = 128;

// Division of numbers below 2^31 by d <= 2^31: n m >> 31 + L for 2^L >= d and m = ceil(2^(31 + L) / d), whose error
// n (m d - 2^(31 + L)) / 2^(31 + L) d is below 1 / d; B D, and so the index of a channel, is 2^30 at most.  (A division of 64-bit numbers is
// 100 instructions, and a lane has 200 for its states.)
struct Divisor {
    uint32_t m;
    int shift;
};
Divisor divisor(uint32_t d) {
    int L = 0;
    while ((1ull << L) < d) ++L;
    return {(uint32_t)(((1ull << (31 + L)) + d - 1) / d), 31 + L};
}
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& d) { return (uint32_t)((uint64_t)n * d.m >> d.shift); }

struct StepsP {
    int B, S, D, N, G;
    const void *u, *dt, *Bm, *Cm, *z;
    const float *A, *skip, *bias;
    float* state;
    void* y;
    bool softplus;
    Divisor channels, group;                               // D, D / G
};

// N is 4 LN; a multiple of 4; any.  ONE: a single token.
enum States { kAll, kFours, kAny };
template <typename IO, int LN, int R, States STATES, bool ONE>
__global__ void __launch_bounds__(kStepThreads, 8) k_scan_steps(const StepsP p) {
    constexpr int M = R > LN ? R / LN : 1;                 // sequences whose channel a lane does alone: l, l + LN, ..
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const uint32_t i = blockIdx.x * (kStepThreads / LN) + threadIdx.x / LN;                  // a channel of R sequences
    const uint32_t row = quotient(i, p.channels);
    const int l = threadIdx.x % LN, n0 = STATES == kFours ? min(l * 4, p.N - 4) : l * 4, b0 = row * R, ch = i - row * p.D, g = quotient(ch, p.group);
    const bool own = STATES == kAll || l * 4 < p.N;                         // a lane behind the last states does the last ones once more, without their results
    const int left = p.N - n0;
    const IO *u = static_cast<const IO*>(p.u), *dt = static_cast<const IO*>(p.dt), *z = static_cast<const IO*>(p.z);
    IO* y = static_cast<IO*>(p.y);
    float* state[R];
    const IO *Bm[R], *Cm[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {                          // behind the last sequence: it once more, without its results
        const size_t b = min(b0 + r, p.B - 1), bc = (b * p.S * p.G + g) * p.N + n0;
        state[r] = p.state + (b * p.D + ch) * p.N + n0;
        Bm[r] = static_cast<const IO*>(p.Bm) + bc;
        Cm[r] = static_cast<const IO*>(p.Cm) + bc;
    }
    auto four = [&](const auto* from) {
        using T = std::remove_cv_t<std::remove_reference_t<decltype(*from)>>;
        if constexpr (STATES != kAny) return load_pack<T, 4>(from, 4, true);
        else return load_pack<T, 4>(from, left, false);
    };
    float h[R][4], a2[4];
#pragma unroll
    for (int r = 0; r < R; ++r) widen(four(state[r]), h[r]);
    widen(four(p.A + (size_t)ch * p.N + n0), a2);
#pragma unroll
    for (float& a : a2) a = no_lower(a * kLog2e);
    const float bias = p.bias ? p.bias[ch] : 0.f, skip = p.skip ? p.skip[ch] : 0.f;
#pragma unroll 1
    for (int s = 0; s < (ONE ? 1 : p.S); ++s) {
        Pack<IO, 4> fb[R], fc[R];
        float uu[M], v[M], zz[M], x[M];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            fb[r] = four(Bm[r]);
            fc[r] = four(Cm[r]);
            Bm[r] += (size_t)p.G * p.N;
            Cm[r] += (size_t)p.G * p.N;
        }
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int r = (l + m * LN) % R;
            const size_t at = ((size_t)min(b0 + r, p.B - 1) * p.S + s) * p.D + ch;
            uu[m] = ld(u, at);
            v[m] = ld(dt, at) + bias;
            zz[m] = z ? ld(z, at) : 0.f;
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
                h[r][n] = fmaf(exp2_unit(fmaf(vr, a2[n], kDecayShift)), h[r][n], xr * pick(fb[r], n));
                o[r] = fmaf(h[r][n], pick(fc[r], n), o[r]);
            }
            if (!own) o[r] = 0.f;
        }
        // over the lanes of a channel, in the order 1, 2, 4, 8; with two sequences a lane ends with those that it does alone
        float k[M];
        if constexpr (R == 2 && LN >= 2) k[0] = (l & 1 ? o[1] : o[0]) + __shfl_xor_sync(0xffffffffu, l & 1 ? o[0] : o[1], 1);
        else {
#pragma unroll
            for (int m = 0; m < M; ++m) k[m] = o[m];
            if constexpr (LN >= 2) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 1);
        }
        if constexpr (LN >= 4) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 2);
        if constexpr (LN >= 8) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 4);
        if constexpr (LN >= 16) k[0] += __shfl_xor_sync(0xffffffffu, k[0], 8);
#pragma unroll
        for (int m = 0; m < M; ++m) {
            const int r = l + m * LN;
            float e = fmaf(skip, uu[m], k[m]);
            if (z) e *= zz[m] * gate_sigmoid(zz[m]);
            if (r < R && b0 + r < p.B) st(y, ((size_t)(b0 + r) * p.S + s) * p.D + ch, e);
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
        if (own && b0 + r < p.B) {
            if constexpr (STATES != kAny) store_pack(state[r], narrow<float, 4>(h[r]), 4, true);
            else store_pack(state[r], narrow<float, 4>(h[r]), left, false);
        }
}

template <typename IO, int LN, int R>
cudaError_t launch(const StepsP& p, cudaStream_t stream) {
    const long long channels = (long long)((p.B + R - 1) / R) * p.D, ctas = (channels + kStepThreads / LN - 1) / (kStepThreads / LN);
    const auto kernel = p.N % 4         ? k_scan_steps<IO, LN, R, kAny, false>
                        : p.N != 4 * LN ? k_scan_steps<IO, LN, R, kFours, false>
                        : p.S > 1       ? k_scan_steps<IO, LN, R, kAll, false>
                                        : k_scan_steps<IO, LN, R, kAll, true>;
    return launch_overlapped(kernel, dim3((unsigned)ctas), dim3(kStepThreads), 0, stream, p);
}
template <typename IO, int LN>
cudaError_t launch(const StepsP& p, cudaStream_t stream) {
    return p.B > 1 ? launch<IO, LN, 2>(p, stream) : launch<IO, LN, 1>(p, stream);
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
    p.S = a.s.T; p.D = a.s.D; p.N = a.s.N; p.G = a.s.G;
    p.A = a.A; p.skip = a.D; p.bias = a.dt_bias; p.softplus = a.softplus;
    p.channels = divisor(p.D);
    p.group = divisor(p.D / p.G);
    p.B = a.s.B; p.u = a.u; p.dt = a.dt; p.z = a.z; p.Bm = a.Bm; p.Cm = a.Cm; p.y = a.y; p.state = a.hT;
    return a.s.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.stream) : launch<float>(p, a.stream);
}

}  // namespace qd

// Selective state space scan: what its kernels share.  Per sequence, with N states to a channel (u, dt, z per token and channel; B_t, C_t
// per token, shared by the D / G channels of a group),
//   dt = softplus(dt + dt_bias) or dt + dt_bias,  a_t = exp(dt_t A),  h_t = a_t h_{t-1} + dt_t u_t B_t,
//   y_t = (<C_t, h_t> + D u_t) SiLU(z_t)     (the factor only with z).
//
// Tiling.  A warp owns 16 channels x 16 states: lane = 4 c + q has channels 2c, 2c + 1 and states 4q .. 4q + 3, its eight states in
// registers from token to token, neighbouring channels side by side in the packed fp32 pairs of sm_100 (the pipe is not faster for them,
// but an instruction is issued for two).  Sums over the states (y, du, ddt) then are over 4 lanes, sums over the channels (dB, dC) over 8,
// and B_t, C_t, dt_t, u_t come from shared memory, where a CTA stages them for a tile of tokens in fp32.  N > 16 takes more warps for the
// same channels; states past N have A = B = C = 0 and channels past the group's last dt = u = 0, which leaves them at 0.  Tokens past T
// have dt = 0: the state passes through.
//
// Segments.  Where there are too few channels to fill the GPU, a sequence is cut into segments: each is first walked from a zero state
// (the first from h0) without outputs, the states at the segments' ends are joined (h = exp(A sum dt) h + local end), and then all
// segments run at once from their true states.  That walks all but the last twice, so one segment where channels suffice.
#pragma once
#include "rows.cuh"

namespace qd {
namespace scan {

constexpr int kWarpChannels = 16, kWarpStates = 16;
constexpr int kSave = 8;                     // tokens from one saved state to the next
constexpr int kTile = 16;                    // tokens that a CTA stages at a time, forward
constexpr size_t kWarpTile = kWarpChannels * kWarpStates;          // states of a warp, in the order [lane][state][channel of the pair]

// What both directions derive from the shape.
struct Dims {
    int B, T, D, N, G, K;                    // K = D / G channels of a group
    int nb;                                  // blocks of 16 states
    int cw;                                  // warps side by side in the channels of a CTA
    int tiles;                               // groups of 16 channels in a group
    int ctas;                                // CTAs to cover a group
    size_t states;                           // fp32 values of one state of one sequence in warp order
};
inline Dims dims(const qd_scan_shape& s) {
    Dims d{};
    d.B = s.B; d.T = s.T; d.D = s.D; d.N = s.N; d.G = s.G; d.K = s.D / s.G;
    d.nb = (s.N + kWarpStates - 1) / kWarpStates;
    d.cw = d.nb == 1 ? 4 : 2;
    d.tiles = (d.K + kWarpChannels - 1) / kWarpChannels;
    d.ctas = (d.tiles + d.cw - 1) / d.cw;
    d.states = (size_t)d.G * d.ctas * d.cw * d.nb * kWarpTile;
    return d;
}

struct P {
    Dims d;
    int segs, seglen;                        // segments of a sequence and tokens of one
    const void *u, *dt, *Bm, *Cm, *z, *dy;
    const float *A, *D, *dt_bias, *h0, *dhT;
    void *y, *du, *ddt, *dz;
    float *hT, *dh0;
    float *saved;                            // [B][ceil(T / kSave)][states]: state before every kSave-th token
    float *ends, *decays;                    // [segs - 1][B][states]: states (gradients) at segments' ends, exp(A sum dt) of segments
    float *pA, *pD;                          // partial gradients of A [segs][B][D N], of D and dt_bias [segs][B][2][D]
    float *pBC;                              // of B and C [ctas][2][B T G N]
    bool softplus, vec, vecn;                // rows are read 16 bytes at a time; so are those of B, C
};

#ifdef __CUDACC__
typedef unsigned long long f2;               // two fp32 in a register pair: channels 2c (low) and 2c + 1
__device__ __forceinline__ f2 pack2(float lo, float hi) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ float2 unpack2(f2 v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f2 exp2_pair(f2 x) {
    const float2 t = unpack2(x);
    return pack2(exp2_unit(t.x), exp2_unit(t.y));
}
struct alignas(16) f2x2 { f2 a, b; };

// softplus(x) = max(x, 0) + log1p(e), e = exp(-|x|) in (0, 1].  log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by the series
// s + s^3 / 3 + s^5 / 5 + ..., whose first dropped term is below 1e-8 of the sum: the relative error stays at a few 2^-24 where e is small.
__device__ __forceinline__ float softplus(float x) {
    const float e = expf(-fabsf(x)), s = __fdividef(e, 2.f + e), w = s * s;
    float t = fmaf(w, 1.f / 15, 1.f / 13);
    t = fmaf(w, t, 1.f / 11);
    t = fmaf(w, t, 1.f / 9);
    t = fmaf(w, t, 1.f / 7);
    t = fmaf(w, t, 1.f / 5);
    t = fmaf(w, t, 1.f / 3);
    const float l = 2.f * fmaf(s * w, t, s);
    return fmaxf(x, 0.f) + (x != x ? x : l);
}

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
#endif

cudaError_t join(float* ends, const float* decays, int n, int from, int step, size_t count, cudaStream_t stream);
int segments(const Dims& d, int slots, int shortest);
int segment_tokens(int T, int segs);

}  // namespace scan
}  // namespace qd

// Linear attention with a decay for each head, e^g = exp(log_decay[head]):
//     S_t = e^g S_{t-1} + k_t v_t^T ,   o_t = scale S_t^T q_t .
// Everything that is computed of a whole sequence is one kind of walk over its chunks, with a state S between them:
//     out_r = sum_{i <= r} D(r - i) (a_r . b_i) c_i  +  rho_r a_r S        D(m) = scale e^{g m}
//     S    <- e^{g n} S + sum_i kappa_i b_i c_i^T                          (n tokens in the chunk)
//   forward in time, rho_r = scale e^{g (r + 1)}, kappa_i = e^{g (n - 1 - i)}:
//     o  = walk(a = q,  b = k, c = v),  S = h          dq = walk(a = dO, b = v, c = k),  S = h^T
//   backward in time (i >= r), rho_r = e^{g (n - 1 - r)}, kappa_i = scale e^{g (i + 1)}:
//     dv = walk(a = k,  b = q, c = dO), S = dL/dh      dk = walk(a = v,  b = dO, c = q), S = (dL/dh)^T
// so a backward needs nothing of the forward but its inputs: no state of any chunk is ever in memory.  Where sequences and heads are
// few, a sequence is cut into segments: first the sums of each by itself (`ends`), which are then joined to the states that the segments
// begin with, then the walks from there.
#pragma once
#include "internal.h"
#include "sm100.cuh"

namespace qd {

struct LinearWalk {
    const void *a, *b, *c;
    void* out;               // NULL: the sums of every segment alone, to `ends`
    const float* s0;         // the states that the segments begin with, [B H][segments][state]; NULL: zeros
    float* sT;               // the state that the walk ends with; NULL: not returned
    float* ends;             // [B H][segments][state], written where out is NULL
    int reverse;
    int exact;               // the state is returned in fp32, so bf16 walks take three planes of what is added to it (see linear_tc.cu), not two
    int flip;                // s0, sT and ends hold S^T (as [DC][DB])
};
constexpr int kLinearWalks = 3;
struct LinearP {
    int T, H, BH, segments, length;      // tokens of a segment, whole chunks; the last one may be shorter
    const float* g;
    float scale;
    unsigned* status;
    int walks;                           // of this launch; CTAs of the walks that share a segment are neighbours
    int clear;                           // the first launch of a call: the status word starts at zero
    LinearWalk w[kLinearWalks];
};

// e^{g m} for a count m of tokens, g2 = g log2(e): 1 for m = 0 whatever g is (minus infinity: nothing is kept)
__device__ __forceinline__ float decay_power(float g2, int m) { return m == 0 ? 1.f : exp2f(g2 * (float)m); }

// e^{g m} = base + more, what a state keeps over m tokens.  A slow head has a base of 1: its factor, rounded, would be off by the same 2^-25 or more
// in every chunk, 1.4e-6 after 3000 tokens of chunks and worse token by token; e^{g m} - 1 is not.
struct Keep { float base, more; };
__device__ __forceinline__ Keep keep_power(float g, int m) {
    const float x = g * (float)m;
    return fabsf(x) < 0.5f ? Keep{1.f, expm1f(x)} : Keep{0.f, decay_power(g * 1.4426950408889634f, m)};
}
__device__ __forceinline__ float kept(const Keep& k, float h, float add) { return fmaf(k.more, h, fmaf(k.base, h, add)); }

}  // namespace qd

// Rotary positions of queries and keys, both in one launch: the pair (a, b) of frequency j becomes
//     (a cos - b sin, a sin + b cos) scale ,   angle = position * turns[j] / 2^64 turns .
// The product of a 64-bit position with a 64-bit fraction of a turn, modulo 2^64, is the angle without whole turns, exactly: no position is too
// far for it, and no floating point angle loses its last bits.  What is left is rounded to 2^-32 turns and brought to an eighth of a turn
// either way before it becomes a float.
//
// Bound by HBM.  A CTA computes the sines of a few tokens once, in shared memory, for all their heads, and then streams the heads through
// registers, 16 bytes at a time where rows allow it.
#include "rows.cuh"

namespace qd {
namespace {

constexpr int kRotaryThreads = 256, kRotaryPairs = 2048, kOpen = 2;      // sines in shared memory; units a thread has under way

struct RotaryP {
    const void *q, *k;
    void *qo, *ko;
    const long long *turns, *positions;
    long long start, tokens;
    int T, Hq, Hk, d, pairs, per;        // per: tokens of a CTA
    int units, rest;                     // of a head: of P pairs, and of the elements that are copied
    float scale;
    bool inverse, wide;                  // wide: packs are aligned
};

template <typename IO, int P, bool INTERLEAVED>
__global__ void __launch_bounds__(kRotaryThreads) k_rotary(const RotaryP p) {
    __shared__ __align__(16) float s_cos[kRotaryPairs], s_sin[kRotaryPairs];
    constexpr int N = INTERLEAVED ? 2 * P : P;               // elements of a pack
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const long long first = (long long)blockIdx.x * p.per;
    const int n = (int)min((long long)p.per, p.tokens - first);
    for (int i = threadIdx.x; i < n * p.pairs; i += kRotaryThreads) {
        const long long tok = first + i / p.pairs;
        const unsigned long long at = p.positions ? (unsigned long long)p.positions[tok] : (unsigned long long)p.start + (unsigned long long)(tok % p.T);
        const unsigned long long turn = at * (unsigned long long)p.turns[i % p.pairs];
        const uint32_t u = (uint32_t)((turn + 0x80000000ull) >> 32);
        const uint32_t quarter = (u + 0x20000000u) >> 30;                            // nearest quarter turn
        float s, c;
        sincospif((float)(int32_t)(u - (quarter << 30)) * 0x1p-31f, &s, &c);         // the rest, in half turns
        const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
        s_cos[i] = p.scale * ((quarter + 1) & 2 ? -x : x);
        s_sin[i] = p.scale * (((quarter & 2) != 0) != p.inverse ? -y : y);
    }
    __syncthreads();
    const int heads = p.Hq + p.Hk, all = p.units + p.rest, items = n * heads * all, stride = gridDim.y * kRotaryThreads;
    // a thread's next unit is `stride` further: unit, head and token of it without a division
    const int step_u = stride % all, step_h = stride / all % heads, step_t = stride / all / heads;
    int i0 = blockIdx.y * kRotaryThreads + threadIdx.x, nu = i0 % all, nh = i0 / all % heads, nt = i0 / all / heads;
    // kOpen units of a thread at a time: all loads, then all stores (which might be to where the next loads read)
    for (; i0 < items; i0 += kOpen * stride) {
        Pack<IO, N> x[kOpen], y[INTERLEAVED ? 1 : kOpen];
        IO* dst[kOpen];
        int unit[kOpen], at[kOpen];                            // unit of the head, and where its sines begin
#pragma unroll
        for (int o = 0; o < kOpen; ++o) {
            if (i0 + o * stride >= items) break;
            const int head = nh, t = nt;
            unit[o] = nu;
            at[o] = t * p.pairs + nu * P;
            nu += step_u; nh += step_h; nt += step_t;
            if (nu >= all) { nu -= all; ++nh; }
            if (nh >= heads) { nh -= heads; ++nt; }
            const bool is_q = head < p.Hq;
            const long long to = is_q ? ((first + t) * p.Hq + head) * p.d : ((first + t) * p.Hk + head - p.Hq) * p.d;
            const int c = unit[o] < p.units ? unit[o] * N : 2 * p.pairs + (unit[o] - p.units) * N;
            const IO* src = static_cast<const IO*>(is_q ? p.q : p.k) + to + c;
            dst[o] = static_cast<IO*>(is_q ? p.qo : p.ko) + to + c;
            const bool turned = unit[o] < p.units;
            x[o] = load_pack<IO, N>(src, turned ? N : p.d - c, p.wide);
            if constexpr (!INTERLEAVED)
                if (turned) y[o] = load_pack<IO, N>(src + p.pairs, N, p.wide);
        }
#pragma unroll
        for (int o = 0; o < kOpen; ++o) {
            if (i0 + o * stride >= items) break;
            if (unit[o] >= p.units) {                           // behind the pairs
                store_pack(dst[o], x[o], p.d - 2 * p.pairs - (unit[o] - p.units) * N, p.wide);
                continue;
            }
            float cs[P], sn[P];
            if constexpr (P % 4 == 0) {                         // pairs are a multiple of P, so at[o] is
#pragma unroll
                for (int j = 0; j < P; j += 4) {
                    const float4 c4 = *reinterpret_cast<const float4*>(s_cos + at[o] + j), s4 = *reinterpret_cast<const float4*>(s_sin + at[o] + j);
                    cs[j] = c4.x; cs[j + 1] = c4.y; cs[j + 2] = c4.z; cs[j + 3] = c4.w;
                    sn[j] = s4.x; sn[j + 1] = s4.y; sn[j + 2] = s4.z; sn[j + 3] = s4.w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < P; ++j) { cs[j] = s_cos[at[o] + j]; sn[j] = s_sin[at[o] + j]; }
            }
            if constexpr (INTERLEAVED) {
                float u[N];
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float a = pick(x[o], 2 * j), b = pick(x[o], 2 * j + 1);
                    u[2 * j] = a * cs[j] - b * sn[j];
                    u[2 * j + 1] = a * sn[j] + b * cs[j];
                }
                store_pack(dst[o], narrow<IO, N>(u), N, p.wide);
            } else {
                float u[N], v[N];
#pragma unroll
                for (int j = 0; j < P; ++j) {
                    const float a = pick(x[o], j), b = pick(y[o], j);
                    u[j] = a * cs[j] - b * sn[j];
                    v[j] = a * sn[j] + b * cs[j];
                }
                store_pack(dst[o], narrow<IO, N>(u), N, p.wide);
                store_pack(dst[o] + p.pairs, narrow<IO, N>(v), N, p.wide);
            }
        }
    }
}

template <typename IO, int P, bool INTERLEAVED>
cudaError_t launch(RotaryP p, bool in_place, cudaStream_t stream) {
    constexpr int N = INTERLEAVED ? 2 * P : P;
    p.units = p.pairs / P;
    p.rest = in_place ? 0 : (p.d - 2 * p.pairs + N - 1) / N;
    p.wide = p.d % N == 0 && (INTERLEAVED || p.pairs % N == 0) && 2 * p.pairs % N == 0;
    const long long items = (long long)(p.Hq + p.Hk) * (p.units + p.rest);
    // a CTA has work for eight passes of its threads, unless that leaves SMs without any
    long long per = 8 * kRotaryThreads / items;
    per = per > p.tokens / (4 * kSMs) ? p.tokens / (4 * kSMs) : per;
    per = per > kRotaryPairs / p.pairs ? kRotaryPairs / p.pairs : per;
    p.per = per < 1 ? 1 : (int)per;
    const long long ctas = (p.tokens + p.per - 1) / p.per;
    long long split = p.per * items / kRotaryThreads;
    split = ctas >= 2 * kSMs ? 1 : split > 2 * kSMs / ctas ? 2 * kSMs / ctas : split;
    return launch_overlapped(k_rotary<IO, P, INTERLEAVED>, dim3((unsigned)ctas, split < 1 ? 1 : (unsigned)split), dim3(kRotaryThreads), 0, stream, p);
}
// pairs of a unit: what makes packs of 16 bytes, or single ones
template <typename IO>
cudaError_t launch(const RotaryP& p, bool interleaved, bool in_place, cudaStream_t stream) {
    constexpr int V = 16 / sizeof(IO);
    if (interleaved)
        return p.d % V == 0 && p.pairs % (V / 2) == 0 ? launch<IO, V / 2, true>(p, in_place, stream) : launch<IO, 1, true>(p, in_place, stream);
    if (p.d % V == 0 && p.pairs % V == 0) return launch<IO, V, false>(p, in_place, stream);
    return p.d % 2 == 0 && p.pairs % 2 == 0 ? launch<IO, 2, false>(p, in_place, stream) : launch<IO, 1, false>(p, in_place, stream);
}

}  // namespace

cudaError_t rotary(const RotaryArgs& a) {
    RotaryP p{};
    p.q = a.q; p.k = a.k; p.qo = a.q_out; p.ko = a.k_out;
    p.turns = a.turns; p.positions = a.positions; p.start = a.start; p.tokens = (long long)a.B * a.T;
    p.T = a.T; p.Hq = a.Hq; p.Hk = a.Hk; p.d = a.d; p.pairs = a.pairs; p.scale = a.scale; p.inverse = a.inverse;
    const bool in_place = a.q == a.q_out && (!a.Hk || a.k == a.k_out);
    return a.dtype == QD_BF16 ? launch<__nv_bfloat16>(p, a.interleaved, in_place, a.stream) : launch<float>(p, a.interleaved, in_place, a.stream);
}

}  // namespace qd

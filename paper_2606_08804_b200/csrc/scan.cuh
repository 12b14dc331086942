// Selective state space scan: what its kernels share.  Per sequence, with N states to a channel (u, dt, z per token and channel; B_t, C_t
// per token, shared by the D / G channels of a group),
//   dt = softplus(dt + dt_bias) or dt + dt_bias,  a_t = exp(dt_t A),  h_t = a_t h_{t-1} + dt_t u_t B_t,
//   y_t = (<C_t, h_t> + D u_t) SiLU(z_t)     (the factor only with z).
//
// Tiling.  A warp owns 16 channels x 16 states: lane = 4 c + q has channels 2c, 2c + 1 and states 4q .. 4q + 3, its eight states in
// registers from token to token, neighbouring states side by side in the packed fp32 pairs of sm_100 (the pipe is not faster for them,
// but an instruction is issued for two).  dt, u, B, C of a token come from shared memory; that returns 128 bytes a clock and SM, however
// many lanes share a value, so a token costs a warp 12 clocks of it forward (20 with the channels packed instead of the states, B and C then
// being pairs of equal values).
// Sums over the states (y, du, ddt) are over 4 lanes, sums over the channels (dB, dC) over 8.  In such a sum a lane keeps a part and hands
// the rest on; so that it keeps the part that it has in the same register whichever lane it is, the channels of a pair are swapped where q
// is odd and, backward, the pairs of states where c & 2 (Map), and shared memory holds both orders.
//
// Roles.  Half of a CTA's warps walk the tokens.  The other half turns dt, u, z, dy of the tile after theirs into what the walk needs
// (softplus, products, gates) in shared memory, in fp32, and writes out what the tile before left there; what it reads is copied to shared
// memory two or three tiles ahead of that.
// One barrier a tile; the two halves share the issue slots of the four sub-partitions, of which the walk alone leaves many unused.  Backward
// the two loops together are as long as the instruction cache takes: with the preparing one twice in it, for two sets of registers, no
// instruction was there one time in eight, and 8 x 2048 tokens of 2048 channels took 681 us instead of 662.
//
// Segments.  Where there are too few channels to fill the GPU, a sequence is cut into segments: each is first walked from a zero state
// (the first from h0) without outputs, the states at the segments' ends are joined (h = exp(A sum dt) h + local end), and then all
// segments run at once from their true states.  That walks all but the last twice, so one segment where channels suffice (cut).
//
// States past N have A = B = C = 0 and channels past the group's last dt = u = 0, which leaves them at 0.  Tokens past T have dt = 0: the
// state passes through.
#pragma once
#include "rows.cuh"

#include <cfloat>

namespace qd {
namespace scan {

constexpr int kWarpChannels = 16, kWarpStates = 16;
constexpr int kWalkers = 4;                  // warps of a CTA that walk; as many prepare
constexpr int kThreads = 2 * 32 * kWalkers;
constexpr int kSave = 8;                     // tokens from one saved state to the next, and of a tile, backward
constexpr int kTile = 16;                    // tokens of a tile, forward
constexpr size_t kWarpTile = kWarpChannels * kWarpStates;          // states of a warp, in the order [lane][channel][state]

// Shared memory that two CTAs of an SM do not have: asked for where every CTA can have an SM for itself, which it would not get while the
// kernel before still holds some of them (backward of 128 CTAs, 4 x 2048 tokens of 2048 channels, call after call: 423 us, 459 without).
constexpr size_t kAloneSmem = 116 * 1024;

// What both directions derive from the shape.
struct Dims {
    int B, T, D, N, G, K;                    // K = D / G channels of a group
    int nb;                                  // blocks of 16 states: 1, 2 or 4, side by side in a CTA
    int ctas;                                // CTAs to cover a group's channels
    size_t states;                           // fp32 values of one state of one sequence in warp order
};
inline Dims dims(const qd_scan_shape& s) {
    Dims d{};
    d.B = s.B; d.T = s.T; d.D = s.D; d.N = s.N; d.G = s.G; d.K = s.D / s.G;
    d.nb = s.N <= 16 ? 1 : s.N <= 32 ? 2 : 4;
    const int cc = kWalkers / d.nb * kWarpChannels;
    d.ctas = (d.K + cc - 1) / cc;
    d.states = (size_t)d.G * d.ctas * kWalkers * kWarpTile;
    return d;
}

struct P {
    Dims d;
    int segs, first, seglen;                 // segments of a sequence, tokens of the first and of the others (Cut)
    const void *u, *dt, *Bm, *Cm, *z, *dy;
    const float *A, *D, *dt_bias, *h0, *dhT;
    void *y, *du, *ddt, *dz;
    float *hT, *dh0;
    float *saved;                            // [B][ceil(T / kSave)][states]: state before every kSave-th token
    float *ends, *decays;                    // [segs - 1][B][states]: states (gradients) at segments' ends, exp(A sum dt) of segments
    float *pA, *pD;                          // partial gradients of A [segs][B][D N], of D and dt_bias [segs][B][2][D]
    float *pBC;                              // of B and C [ctas][2][bcs]
    size_t bcs;                              // B T G N
    bool softplus;
    int rows, bc;                            // how rows and those of B, C are copied (Copy)
    bool joined;                             // the ends are those of the true states already
};

// How groups of a row are copied: whole and aligned; in words of 4 bytes (bf16: an even number of elements); one by one.
enum Copy { kSingle = 0, kWords = 1, kWhole = 2 };
inline int copy_of(int width, int group, int dtype) { return width % group == 0 ? kWhole : dtype == QD_F32 || width % 2 == 0 ? kWords : kSingle; }

// Segments of a sequence; tokens of the first and of each other, multiples of kTile.  Taken are those that need least time by what the two
// walks of a token cost, a walk taking the time of kBegin tokens more to begin, a second one kLaunch ns to launch.  CTAs beyond two an SM
// wait for those before.  Where one segment leaves some SMs a single CTA, the segment that is walked first, to be joined to the other, is a
// short one, for the places that are left over.
struct Cut { int segs, first, len; };
constexpr int kBegin = 24, kMostWaves = 5, kLaunch = 1500;
Cut cut(const Dims& d, bool backward);
// True states at the segments' ends from those of each walked alone, which they overwrite, where the walk does not join them itself.
constexpr int kMostJoined = 32;              // segments before one's own whose ends a CTA joins by itself
cudaError_t join(float* ends, const float* decays, int n, int from, int step, size_t count, cudaStream_t stream);

#ifdef __CUDACC__
struct alignas(16) f2x2 { f2 a, b; };

// softplus(x) = max(x, 0) + log1p(e), e = exp(-|x|) in (0, 1].  log1p(e) = 2 artanh(s), s = e / (2 + e) <= 1/3, by the series
// s + s^3 / 3 + s^5 / 5 + ..., whose first dropped term is below 1e-8 of the sum: the relative error stays at a few 2^-24 where e is
// small, but for that of e, 2^-24 |x|.
__device__ __forceinline__ float2 softplus(float x, float y) {
    const float e = exp2_unit(fabsf(x) * -kLog2e), f = exp2_unit(fabsf(y) * -kLog2e);
    const f2 ef = pack2(e, f), s = mul2(ef, pack2(reciprocal(2.f + e), reciprocal(2.f + f))), w = mul2(s, s), s2 = add2(s, s);
    f2 t = fma2(w, both(1.f / 15), both(1.f / 13));
    t = fma2(w, t, both(1.f / 11));
    t = fma2(w, t, both(1.f / 9));
    t = fma2(w, t, both(1.f / 7));
    t = fma2(w, t, both(1.f / 5));
    t = fma2(w, t, both(1.f / 3));
    return unpack2(add2(fma2(mul2(s2, w), t, s2), pack2(fmaxf(x, 0.f), fmaxf(y, 0.f))));
}
// Decay exp(dt A) with A2 = A log2(e).  The special function unit rounds down more often than up: 2^x comes out 5e-9 to 8e-9 too small on
// average for x in (-2^-8, 0), 2e-8 at -2^-7, 5e-8 from -2^-4 on (3e-8 to 6e-8 rms).  A decay of almost 1 is applied a thousand times, so
// it is the mean that counts: x is taken a little larger, which leaves 8e-9 too much in the first range, 6e-9 too little at -2^-7 and 3e-8 of
// either sign beyond; 2^0 stays 1 exactly.  (8 x 2048 tokens of 2048 channels: dA 0.76e-6 off, without it 1.8e-6, with 1.2e-8 1.04e-6, with
// 2.4e-8 0.77e-6; fp32 operations one by one 0.92e-6.)
constexpr float kDecayShift = 2e-8f;
// A log2(e) is taken no lower than the lowest number: minus infinity would make a step of 0, as that of the tokens past the last, 0 times
// infinity, where the state has to pass through.  Every step above 1e-36 forgets the state either way.  (NaN stays NaN.)
__device__ __forceinline__ float no_lower(float a) { return a < -FLT_MAX ? -FLT_MAX : a; }
__device__ __forceinline__ f2 decay(f2 dt, f2 A2) { return exp2_pair(fma2(dt, A2, both(kDecayShift))); }

// What a walking lane owns.  Registers [channel][pair of states], flat.
struct Map {
    int q, ch[2], order, swap;               // its channels in the warp's 16; which order of a record it reads, of channels and of pairs of states
    __device__ __forceinline__ Map(int lane, bool backward) {
        q = lane & 3;
        const int c = lane >> 2;
        order = q & 1;
        ch[0] = 2 * c + order;
        ch[1] = 2 * c + 1 - order;
        swap = backward ? c >> 1 & 1 : 0;
    }
    __device__ __forceinline__ int state(int pair, int e) const { return 4 * q + 2 * (pair ^ swap) + e; }       // in the warp's 16
};
// f(register, low half or high, offset in a [D, N] state, whether there is such a state)
template <class F>
__device__ __forceinline__ void each_state(const P& p, const Map& m, int g, int ch, int n0, F f) {
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int pr = 0; pr < 2; ++pr)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int k = ch + m.ch[c], n = n0 + m.state(pr, e);
                f(2 * c + pr, e, ((size_t)g * p.d.K + k) * p.d.N + n, k < p.d.K && n < p.d.N);
            }
}
__device__ __forceinline__ void load_state(const P& p, const Map& m, const float* s, int g, int ch, int n0, float scale, f2 (&h)[4]) {
    float v[4][2];
    each_state(p, m, g, ch, n0, [&](int r, int e, size_t at, bool in) { v[r][e] = in ? s[at] * scale : 0.f; });
#pragma unroll
    for (int r = 0; r < 4; ++r) h[r] = pack2(v[r][0], v[r][1]);
}
// A log2(e)
__device__ __forceinline__ void load_A(const P& p, const Map& m, int g, int ch, int n0, f2 (&A2)[4]) {
    load_state(p, m, p.A, g, ch, n0, kLog2e, A2);
#pragma unroll
    for (f2& a : A2) {
        const float2 v = unpack2(a);
        a = pack2(no_lower(v.x), no_lower(v.y));
    }
}
__device__ __forceinline__ void store_state(const P& p, const Map& m, float* s, int g, int ch, int n0, const f2 (&h)[4]) {
    each_state(p, m, g, ch, n0, [&](int r, int e, size_t at, bool in) {
        const float2 v = unpack2(h[r]);
        if (in) s[at] = e ? v.y : v.x;
    });
}
// the same in warp order
__device__ __forceinline__ void load_tile(const float* s, f2 (&h)[4]) {
    const f2x2 *v = reinterpret_cast<const f2x2*>(s), a = v[0], b = v[1];
    h[0] = a.a; h[1] = a.b; h[2] = b.a; h[3] = b.b;
}
__device__ __forceinline__ void store_tile(float* s, const f2 (&h)[4]) {
    f2x2* v = reinterpret_cast<f2x2*>(s);
    v[0] = {h[0], h[1]};
    v[1] = {h[2], h[3]};
}
// end of a segment walked alone: what it adds, and the decay of what was before it; sum: of dt, of both channels
__device__ __forceinline__ void store_end(const P& p, int k, int b, size_t lane, const f2 (&h)[4], const f2 (&A2)[4], const float (&sum)[2]) {
    const size_t at = ((size_t)k * p.d.B + b) * p.d.states + lane;
    f2 a[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) a[j] = exp2_pair(mul2(both(sum[j >> 1]), A2[j]));
    store_tile(p.ends + at, h);
    store_tile(p.decays + at, a);
}
// A segment's end from the state before it.  Where A is positive its decay may overflow, which a state of 0 does not notice.
__device__ __forceinline__ float joined(float decay, float before, float end) { return before == 0.f ? end : fmaf(decay, before, end); }
// the state behind segment ends[n - 1] of `from, from + step, ..`
__device__ __forceinline__ void load_end(const P& p, int from, int step, int n, int b, size_t lane, f2 (&h)[4]) {
    const size_t stride = (size_t)p.d.B * p.d.states, base = (size_t)b * p.d.states + lane;
    if (p.joined) return load_tile(p.ends + (size_t)(from + (n - 1) * step) * stride + base, h);
    load_tile(p.ends + (size_t)from * stride + base, h);
#pragma unroll 4
    for (int k = 1; k < n; ++k) {
        f2 a[4], e[4];
        load_tile(p.decays + (size_t)(from + k * step) * stride + base, a);
        load_tile(p.ends + (size_t)(from + k * step) * stride + base, e);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 x = unpack2(a[j]), y = unpack2(h[j]), z = unpack2(e[j]);
            h[j] = pack2(joined(x.x, y.x, z.x), joined(x.y, y.y, z.y));
        }
    }
}
// N neighbouring elements on their way to shared memory: those from `left` on are 0.  kSingle waits for them.
template <int N, typename IO>
__device__ __forceinline__ void copy_group(IO* dst, const IO* src, int left, int how) {
    constexpr int BYTES = N * sizeof(IO);
    if (how == kWhole) copy_bytes<BYTES>(dst, src, left > 0 ? BYTES : 0);
    else if (how == kWords) {
        constexpr int E = 4 / sizeof(IO);
#pragma unroll
        for (int o = 0; o < N; o += E) copy_bytes<4>(dst + o, src + (o < left ? o : 0), o < left ? 4 : 0);
    } else {
#pragma unroll
        for (int o = 0; o < N; ++o) st(dst, o, o < left ? ld(src, o) : 0.f);
    }
}
// Tiles of TT tokens (from tt, below `end`) x CC channels (from col, `left` of them) of NA tensors [T, D] (absent ones null), row major, by
// 128 threads, which share out the tensors where a tile is fewer than 128 groups of 16 bytes.
template <int TT, int CC, typename IO, int NA>
__device__ __forceinline__ void copy_tiles(IO* const (&dst)[NA], const void* const (&src)[NA], size_t row0, int D, int tt, int end, size_t col, int left,
                                           int how, int tid) {
    constexpr int E = 16 / sizeof(IO), CH = TT * CC / E, SETS = CH < 128 ? 128 / CH : 1;
#pragma unroll
    for (int j = 0; j < (CH + 127) / 128; ++j) {
        const int x = SETS > 1 ? tid % CH : tid + j * 128, t = tt + x / (CC / E), c = x % (CC / E) * E;
        const int have = t < end ? left - c : 0;
        const size_t at = have > 0 ? (row0 + t) * D + col + c : 0;
#pragma unroll
        for (int a = 0; a < NA; ++a)
            if (src[a] && (SETS == 1 || a % SETS == tid / CH)) copy_group<E>(dst[a] + x * E, static_cast<const IO*>(src[a]) + at, have, how);
    }
}
// The same of one tile after the other where groups are whole and all tokens there: a thread's addresses move on by a step a tile (computed
// anew for each they cost 3 % of 4 x 2048 x 2048 backward, 8 % forward).  `ring` is that of the first tensor, the others' are behind it.
template <int TT, int CC, int RING, typename IO, int NA>
struct TileRun {
    static constexpr int E = 16 / sizeof(IO), CH = TT * CC / E, SETS = CH < 128 ? 128 / CH : 1, PER = (NA + SETS - 1) / SETS, REP = (CH + 127) / 128;
    const IO* src[PER];                      // null: absent
    IO* dst;
    long long step;
    int bytes;                               // none where there are no channels
    __device__ __forceinline__ TileRun(IO* ring, const void* const (&from)[NA], size_t row, int D, size_t col, int channels, int by, int tid) {
        const int x = tid % CH, set = SETS > 1 ? tid / CH : 0, c = x % (CC / E) * E;
        const bool has = channels > c;
        bytes = has ? 16 : 0;
        step = has ? (long long)by * D : 0;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            src[j] = nullptr;
#pragma unroll
            for (int a = 0; a < NA; ++a)
                if (a == set + j * SETS && from[a]) src[j] = static_cast<const IO*>(from[a]) + (has ? (row + x / (CC / E)) * D + col + c : 0);
        }
        dst = ring + (set * RING * CH + x) * E;
    }
    __device__ __forceinline__ void copy(int slot, int D) const {
#pragma unroll
        for (int j = 0; j < PER; ++j)
#pragma unroll
            for (int r = 0; r < REP; ++r)
                if (src[j]) copy_bytes<16>(dst + ((j * SETS * RING + slot) * CH + r * 128) * E, src[j] + (bytes ? (size_t)(r * 128 / (CC / E)) * D : 0), bytes);
    }
    __device__ __forceinline__ void move() {
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (src[j]) src[j] += step;
    }
};
// And of B and C: four states of a token, of B by the first half of the threads that share a token (T tokens to a tile).
template <int NS, typename IO>
struct StateRun {
    const IO* src;
    size_t token;                            // elements from token to token
    long long step;
    int row, bytes;
    __device__ __forceinline__ StateRun(const P& p, size_t first, int g, bool with_B, bool with_C, int by, int tid) {
        const int r = tid % (NS / 2), s = r % (NS / 4) * 4;
        const bool is_B = r < NS / 4, has = s < p.d.N && (is_B ? with_B : with_C);
        row = tid / (NS / 2);
        bytes = has ? 4 * sizeof(IO) : 0;
        token = has ? (size_t)p.d.G * p.d.N : 0;
        step = (long long)token * by;
        src = static_cast<const IO*>(is_B ? p.Bm : p.Cm) + (has ? (first + row) * token + (size_t)g * p.d.N + s : 0);
    }
    template <int T, int J> __device__ __forceinline__ void copy(Pack<IO, 4> (&to)[J][128], int tid) const {
#pragma unroll
        for (int j = 0; j < J; ++j)
            if (row + j * (256 / NS) < T) copy_bytes<4 * sizeof(IO)>(&to[j][tid], src + j * (256 / NS) * token, bytes);
    }
    __device__ __forceinline__ void move() { src += step; }
};
__device__ __forceinline__ void prepare_barrier() { asm volatile("bar.sync 1, 128;" ::: "memory"); }     // the half that prepares
__device__ __forceinline__ float sum_pair(f2 v) {
    const float2 t = unpack2(v);
    return t.x + t.y;
}
#endif

}  // namespace scan
}  // namespace qd

// What the kernels around the delta rule (convolution, scan, norm) share: groups of channels in registers, the functions of the
// gates, and the sum of partial gradients.
#pragma once
#include "internal.h"
#include "sm100.cuh"

namespace qd {
namespace {

// N consecutive channels of a row.  `vec`: the row's groups are whole and aligned to their size (16 bytes at most); otherwise elements
// are read one at a time and those from `left` on are 0.  (Ordinary loads, not the read-only path: the kernel before may still be
// writing when a kernel begins, and a decode step writes the state that it read.)
template <typename IO, int N> struct Pack { uint32_t w[(N * sizeof(IO) + 3) / 4]; };

template <typename IO, int N>
__device__ __forceinline__ Pack<IO, N> load_pack(const IO* p, int left, bool vec) {
    Pack<IO, N> r;
    constexpr int W = sizeof(r.w) / 4;
    if (vec && left >= N) {
        if constexpr (W % 4 == 0) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const uint4 t = reinterpret_cast<const uint4*>(p)[i];
                r.w[4 * i] = t.x; r.w[4 * i + 1] = t.y; r.w[4 * i + 2] = t.z; r.w[4 * i + 3] = t.w;
            }
            return r;
        } else if constexpr (W == 2) {
            const uint2 t = *reinterpret_cast<const uint2*>(p);
            r.w[0] = t.x; r.w[1] = t.y;
            return r;
        } else if constexpr (N * sizeof(IO) == 4) {
            r.w[0] = *reinterpret_cast<const uint32_t*>(p);
            return r;
        }
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (sizeof(IO) == 4) {
            r.w[i] = i < left ? __float_as_uint(p[i]) : 0u;
        } else {
            const unsigned short* s = reinterpret_cast<const unsigned short*>(p);
            const uint32_t lo = 2 * i < left ? s[2 * i] : 0, hi = 2 * i + 1 < N && 2 * i + 1 < left ? s[2 * i + 1] : 0;
            r.w[i] = lo | hi << 16;
        }
    }
    return r;
}
template <typename IO, int N>
__device__ __forceinline__ Pack<IO, N> zero_pack() {
    Pack<IO, N> r;
#pragma unroll
    for (uint32_t& w : r.w) w = 0;
    return r;
}
template <typename IO, int N>
__device__ __forceinline__ float pick(const Pack<IO, N>& r, int i) {
    if constexpr (sizeof(IO) == 4) return __uint_as_float(r.w[i]);
    else return __uint_as_float(i & 1 ? r.w[i >> 1] & 0xffff0000u : r.w[i >> 1] << 16);
}
template <typename IO, int N>
__device__ __forceinline__ void widen(const Pack<IO, N>& r, float (&f)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = pick(r, i);
}
template <typename IO, int N>
__device__ __forceinline__ Pack<IO, N> narrow(const float (&f)[N]) {
    Pack<IO, N> r;
    if constexpr (sizeof(IO) == 4) {
#pragma unroll
        for (int i = 0; i < N; ++i) r.w[i] = __float_as_uint(f[i]);
    } else {
#pragma unroll
        for (int i = 0; i < (N + 1) / 2; ++i) {
            const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * i], 2 * i + 1 < N ? f[2 * i + 1 < N ? 2 * i + 1 : 0] : 0.f);
            r.w[i] = *reinterpret_cast<const uint32_t*>(&t);
        }
    }
    return r;
}
template <typename IO, int N>
__device__ __forceinline__ void store_pack(IO* p, const Pack<IO, N>& r, int left, bool vec) {
    constexpr int W = sizeof(r.w) / 4;
    if (vec && left >= N) {
        if constexpr (W % 4 == 0) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i)
                reinterpret_cast<uint4*>(p)[i] = make_uint4(r.w[4 * i], r.w[4 * i + 1], r.w[4 * i + 2], r.w[4 * i + 3]);
            return;
        } else if constexpr (W == 2) {
            *reinterpret_cast<uint2*>(p) = make_uint2(r.w[0], r.w[1]);
            return;
        } else if constexpr (N * sizeof(IO) == 4) {
            *reinterpret_cast<uint32_t*>(p) = r.w[0];
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) {
            if constexpr (sizeof(IO) == 4) p[i] = __uint_as_float(r.w[i]);
            else reinterpret_cast<unsigned short*>(p)[i] = (unsigned short)(i & 1 ? r.w[i >> 1] >> 16 : r.w[i >> 1]);
        }
}

// The logistic function.  e^{-x} overflows to infinity for x below -88, where the quotient is 0 as it should be.
__device__ __forceinline__ float sigmoid(float x) { return __fdividef(1.f, 1.f + expf(-x)); }

// 2^x on the special function unit: 2 ulp.
__device__ __forceinline__ float exp2_unit(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// BYTES on their way to shared memory, zeros where `bytes` is 0; committed in groups, of which all but the last N have come after a wait.
template <int BYTES>
__device__ __forceinline__ void copy_bytes(void* dst, const void* src, int bytes) {
    const uint32_t d = sm100::smem_u32(dst);
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(bytes) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(d), "l"(src), "n"(BYTES), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Whether any of many pairs of bf16 values is infinite or NaN, two pairs to an instruction: the sum of their products is then, too, whatever
// else is in it.  (Products that overflow raise it as well: who is told looks again.)
__device__ __forceinline__ void see_unfit(uint32_t& sum, uint32_t x, uint32_t y) {
    asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(x), "r"(y));
}
__device__ __forceinline__ bool seen_unfit(uint32_t sum) { return (sum & 0x7f80u) == 0x7f80u || (sum & 0x7f800000u) == 0x7f800000u; }

// A warpgroup's registers a thread, from here on: fewer, or more, as soon as others have given them.
template <int N> __device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float reciprocal(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// the logistic function, with the relative error of e^-x: 2^-24 |x|
__device__ __forceinline__ float gate_sigmoid(float x) { return reciprocal(1.f + exp2_unit(x * -kLog2e)); }

// ---- the packed fp32 instructions of sm_100: one issue for two (the pipe takes as long as for two) ----
typedef unsigned long long f2;               // two fp32 in a register pair
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
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ f2 both(float x) { return pack2(x, x); }
__device__ __forceinline__ f2 exp2_pair(f2 x) {
    const float2 t = unpack2(x);
    return pack2(exp2_unit(t.x), exp2_unit(t.y));
}

// out[col] = sum over p of part[p][col], col < cols, fp32, p in an order that depends on nothing but `parts`.  Column c of the
// partials is written to out0[c % inner * step0 + c / inner] while c < split, to out1[c - split] behind that.
constexpr int kSumRows = 32;                 // threads that share a column: many, since it is their loads' latency that counts
__global__ void __launch_bounds__(32 * kSumRows) k_sum_parts(const float* part, int parts, long long cols, long long split, long long inner,
                                                             int step0, float* out0, float* out1) {
    __shared__ float s[kSumRows][33];
    sm100::grid_dep_wait();
    sm100::grid_dep_launch();
    const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
    const long long c = (long long)blockIdx.x * 32 + x;
    float a = 0.f;
    if (c < cols)
#pragma unroll 8
        for (int p = y; p < parts; p += kSumRows) a += part[(long long)p * cols + c];
    s[y][x] = a;
    __syncthreads();
    a = s[x][y];                                            // a warp a column
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) a += __shfl_xor_sync(0xffffffffu, a, w);
    const long long o = (long long)blockIdx.x * 32 + y;
    if (x == 0 && o < cols) {
        if (o < split) { if (out0) out0[o % inner * step0 + o / inner] = a; }
        else if (out1) out1[o - split] = a;
    }
}
inline cudaError_t sum_parts(const float* part, int parts, long long cols, long long split, long long inner, int step0, float* out0,
                             float* out1, cudaStream_t stream) {
    return launch_overlapped(k_sum_parts, dim3((unsigned)((cols + 31) / 32)), dim3(32 * kSumRows), 0, stream, part, parts, cols, split, inner,
                             step0, out0, out1);
}

}  // namespace
}  // namespace qd

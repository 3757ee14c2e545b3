// Device code that the Newton-Schulz kernels of all sizes use: how a matrix element is read and written, and the fp16 pairs.
//
// The iteration (the odd quintic that Muon made common): X = G / (|G|_F + eps), then `steps` times
//     A = X X',   B = b A + c A^2,   X <- a X + B X.
// Its products run on tcgen05 with fp16 operands and fp32 sums, and keep fp32's accuracy: a matrix is a pair of fp16 matrices
// hi + lo (22 bits) times a power of two, and a product is hi hi' + hi lo' + lo hi' (lo lo' is below 2^-22 of it).
// Singular values of an estimated gradient are small against the Frobenius norm, and a step multiplies the small ones, and
// whatever rounding left beside them, by a (3.4): with 11 bits alone a matrix of low rank would come back with some percent of noise in
// its null space.  The scales are powers of two found on the host from the largest singular value that the steps can reach
// (an element is never larger), so nothing overflows; what lies below fp16's normal range is below 2^-29 of the largest, and
// its last bit below 2^-39.
//
// All matrices of the iteration are kept in panels: element (i, j) of a matrix with mp rows is half (j / 8 * mp + i) * 8 + j % 8.  A
// panel's 8 x 8 squares are the core matrices of an unswizzled tcgen05 operand both ways: with j as the contracted index (K-major) and
// with i (MN-major), so B X and X X' read the same X, and any tile is a set of contiguous runs.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
#include "newton_schulz.h"
#include "umma.cuh"

namespace evo {
namespace ns {

// kind::f16, fp16 x fp16 -> fp32, A K-major; B K-major or MN-major
__host__ __device__ constexpr uint32_t idesc_f16(uint32_t M, uint32_t N, bool b_mn)
{
    return (1u << 4) | (b_mn ? 1u << 16 : 0u) | ((N >> 3) << 17) | ((M >> 4) << 24);
}

// Waits of a kernel without a status block of its own: after one that ran out all others return at once.
struct Waits {
    volatile int* abort;
    const uint32_t* limit;               // log2 of the clocks (shared memory)
    uint32_t* sticky;
    __device__ __forceinline__ void wait(uint32_t bar, uint32_t parity) const
    {
        if (mbar_try_wait(bar, parity) || *abort) return;
        if (!mbar_wait_bounded(bar, parity, limit)) {
            *abort = 1;
            if (sticky) atomicOr(sticky, 1u << EVO_ERR_TIMEOUT);
        }
    }
};

// LATE: from L2, see Args
template <bool LATE, typename T>
__device__ __forceinline__ T fetch(const T* p)
{
    if constexpr (LATE) return __ldcg(p);
    else return *p;
}

// (1 - mu) g and mu m' are rounded once each
__device__ __forceinline__ float muon_direction(const Args& a, float gradient, float m, float* momentum)
{
    const float g = a.s.rest * gradient;
    *momentum = fmaf(a.s.mu, m, g);
    return a.s.nesterov ? fmaf(a.s.mu, *momentum, g) : *momentum;
}
template <uint32_t SRC, bool LATE>
__device__ __forceinline__ float load(const Args& a, uint64_t at, float* momentum)
{
    if constexpr (SRC == kF32) return static_cast<const float*>(a.in)[at];
    if constexpr (SRC == kBf16) return __bfloat162float(static_cast<const __nv_bfloat16*>(a.in)[at]);
    if constexpr (SRC == kF16) return __half2float(static_cast<const __half*>(a.in)[at]);
    if constexpr (SRC == kMuon) return muon_direction(a, fetch<LATE>(static_cast<const float*>(a.in) + at), fetch<LATE>(a.m_in + at), momentum);
}

// the momentum of a matrix element, and its second moment as it was (Adam's, which matrices do not use)
template <bool LATE>
__device__ __forceinline__ void store_moments(const Args& a, uint64_t at, float momentum)
{
    a.m_out[at] = momentum;
    if (a.v_out != a.v_in) a.v_out[at] = fetch<LATE>(a.v_in + at);
}

template <uint32_t SRC, bool LATE>
__device__ __forceinline__ void store(const Args& a, uint64_t at, float x, float gain)
{
    if constexpr (SRC == kF32) static_cast<float*>(a.out)[at] = x;
    if constexpr (SRC == kBf16) static_cast<__nv_bfloat16*>(a.out)[at] = __float2bfloat16_rn(x);
    if constexpr (SRC == kF16) static_cast<__half*>(a.out)[at] = __float2half_rn(x);
    if constexpr (SRC == kMuon) static_cast<float*>(a.out)[at] = fmaf(gain, x, a.s.keep * fetch<LATE>(a.c_in + at));
}

// Eight elements from `at` on, `step` apart, of which `count` exist (the others are 0).  UPDATE: what Muon updates on the way is updated.
template <uint32_t SRC, bool LATE, bool UPDATE>
__device__ __forceinline__ void load8(const Args& a, uint64_t at, uint32_t step, uint32_t count, float (&x)[8])
{
    if constexpr (SRC == kF32) {
        const float* const p = static_cast<const float*>(a.in) + at;
        if (step == 1u && count == 8u && (reinterpret_cast<uintptr_t>(p) & 15u) == 0u) {
            const float4 u = *reinterpret_cast<const float4*>(p), v = *reinterpret_cast<const float4*>(p + 4);
            x[0] = u.x; x[1] = u.y; x[2] = u.z; x[3] = u.w; x[4] = v.x; x[5] = v.y; x[6] = v.z; x[7] = v.w;
            return;
        }
    }
    float momentum[8];
    if constexpr (SRC == kMuon) {
        const float* const g = static_cast<const float*>(a.in) + at;
        const float* const m = a.m_in + at;
        if (step == 1u && count == 8u && ((reinterpret_cast<uintptr_t>(g) | reinterpret_cast<uintptr_t>(m) | reinterpret_cast<uintptr_t>(a.m_out + at)) & 15u) == 0u) {
#pragma unroll
            for (uint32_t h = 0; h < 8u; h += 4u) {
                const float4 u = fetch<LATE>(reinterpret_cast<const float4*>(g + h)), v = fetch<LATE>(reinterpret_cast<const float4*>(m + h));
                x[h] = muon_direction(a, u.x, v.x, &momentum[h]);
                x[h + 1u] = muon_direction(a, u.y, v.y, &momentum[h + 1u]);
                x[h + 2u] = muon_direction(a, u.z, v.z, &momentum[h + 2u]);
                x[h + 3u] = muon_direction(a, u.w, v.w, &momentum[h + 3u]);
            }
#pragma unroll
            for (uint32_t h = 0; UPDATE && h < 8u; h += 4u)
                *reinterpret_cast<float4*>(a.m_out + at + h) = make_float4(momentum[h], momentum[h + 1u], momentum[h + 2u], momentum[h + 3u]);
            if (UPDATE && a.v_out != a.v_in) {
                const float4* const v4 = reinterpret_cast<const float4*>(a.v_in + at);
                if (((reinterpret_cast<uintptr_t>(v4) | reinterpret_cast<uintptr_t>(a.v_out + at)) & 15u) == 0u) {
                    const float4 p = fetch<LATE>(v4), q = fetch<LATE>(v4 + 1);
                    *reinterpret_cast<float4*>(a.v_out + at) = p;
                    *reinterpret_cast<float4*>(a.v_out + at + 4u) = q;
                    return;
                }
                float v[8];
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e) v[e] = fetch<LATE>(a.v_in + at + e);
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e) a.v_out[at + e] = v[e];
            }
            return;
        }
    }
#pragma unroll
    for (uint32_t e = 0; e < 8u; ++e) x[e] = e < count ? load<SRC, LATE>(a, at + static_cast<uint64_t>(e) * step, &momentum[e]) : 0.f;
    if constexpr (SRC == kMuon && UPDATE) {
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e)
            if (e < count) store_moments<LATE>(a, at + static_cast<uint64_t>(e) * step, momentum[e]);
    }
}
// four neighbouring elements of the result, of which `count` (or more) exist
template <uint32_t SRC, bool LATE>
__device__ __forceinline__ void store4(const Args& a, uint64_t at, const float4& v, uint32_t count, float gain)
{
    if constexpr (SRC == kF32) {
        float* const p = static_cast<float*>(a.out) + at;
        if (count >= 4u && (reinterpret_cast<uintptr_t>(p) & 15u) == 0u) {
            *reinterpret_cast<float4*>(p) = v;
            return;
        }
    }
    if constexpr (SRC == kMuon) {
        float* const p = static_cast<float*>(a.out) + at;
        if (count >= 4u && ((reinterpret_cast<uintptr_t>(p) | reinterpret_cast<uintptr_t>(a.c_in + at)) & 15u) == 0u) {
            const float4 c = fetch<LATE>(reinterpret_cast<const float4*>(a.c_in + at));
            *reinterpret_cast<float4*>(p) = make_float4(fmaf(gain, v.x, a.s.keep * c.x), fmaf(gain, v.y, a.s.keep * c.y),
                                                        fmaf(gain, v.z, a.s.keep * c.z), fmaf(gain, v.w, a.s.keep * c.w));
            return;
        }
    }
    const float x[4] = { v.x, v.y, v.z, v.w };
#pragma unroll
    for (uint32_t e = 0; e < 4u; ++e)
        if (e < count) store<SRC, LATE>(a, at + e, x[e], gain);
}

// element (i, j) of the m x n matrix in the source or the result
__device__ __forceinline__ uint64_t in_index(const Group& g, uint32_t which, uint32_t i, uint32_t j)
{
    const uint32_t r = g.tall ? j : i, c = g.tall ? i : j;
    return g.in + which * g.in_stride + static_cast<uint64_t>(r) * g.in_ld + c;
}
__device__ __forceinline__ uint64_t out_index(const Group& g, uint32_t which, uint32_t i, uint32_t j)
{
    const uint32_t r = g.tall ? j : i, c = g.tall ? i : j;
    return g.out + which * g.out_stride + static_cast<uint64_t>(r) * g.out_ld + c;
}

// What the elements are multiplied with.  A matrix with an infinity or a NaN has no direction: the result is NaN throughout.
// One whose norm is not far above eps starts with small singular values; it is carried times a further 2^lift, so that fp16 pairs hold
// it as well, and a step takes `growth` back from that until nothing is left (see lift_at).
__device__ __forceinline__ double first_scale(const Scalars& s, double sum_of_squares, uint32_t* lift)
{
    *lift = 0u;
    if (!isfinite(sum_of_squares)) return __longlong_as_double(0x7FF8000000000000ll);
    const double norm = sqrt(sum_of_squares), f = norm / (norm + static_cast<double>(s.eps));
    if (f > 0.0 && f < 0.5) *lift = static_cast<uint32_t>(min(-1 - ilogb(f), 100));
    return ldexp(static_cast<double>(s.s_x) / (norm + static_cast<double>(s.eps)), static_cast<int>(*lift));
}
// lift of X in step k
__device__ __forceinline__ uint32_t lift_at(const Scalars& s, uint32_t first, uint32_t k)
{
    return first > k * s.growth ? first - k * s.growth : 0u;
}
__device__ __forceinline__ float power_of_two(int e) { return __int_as_float(e < -126 ? 0 : (e + 127) << 23); }

// x and y as pairs, packed (the difference to the high part by an instruction that takes it as it is)
__device__ __forceinline__ void split2(float x, float y, uint32_t& hi, uint32_t& lo)
{
    float u, v;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(y), "f"(x));
    asm("{\n\t.reg .b16 l, h;\n\tmov.b32 {l, h}, %2;\n\tadd.rn.f32.f16 %0, l, %3;\n\tadd.rn.f32.f16 %1, h, %4;\n\t}"
        : "=f"(u), "=f"(v) : "r"(hi ^ 0x80008000u), "f"(x), "f"(y));
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(lo) : "f"(v), "f"(u));
}
__device__ __forceinline__ void split8(const float (&x)[8], uint4& hi, uint4& lo)
{
    split2(x[0], x[1], hi.x, lo.x);
    split2(x[2], x[3], hi.y, lo.y);
    split2(x[4], x[5], hi.z, lo.z);
    split2(x[6], x[7], hi.w, lo.w);
}
__device__ __forceinline__ void join8(const uint4& hi, const uint4& lo, float (&x)[8])
{
    const uint32_t h[4] = { hi.x, hi.y, hi.z, hi.w }, l[4] = { lo.x, lo.y, lo.z, lo.w };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
        const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&l[i]));
        x[2 * i] = a.x + b.x;
        x[2 * i + 1] = a.y + b.y;
    }
}

// fixed-order sum over a block of T threads; every thread gets it
template <uint32_t T>
__device__ __forceinline__ double block_sum(double x, double* red)
{
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    if ((threadIdx.x & 31u) == 0u) red[threadIdx.x >> 5] = x;
    __syncthreads();
    double t = 0.0;
#pragma unroll
    for (uint32_t w = 0; w < T / 32u; ++w) t += red[w];
    __syncthreads();
    return t;
}

}  // namespace ns
}  // namespace evo

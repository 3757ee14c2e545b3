// Warp-level products of a weight tile (16 outputs) with rows of activations (8 columns of the MMA each).
//
// fp32 operands are two tf32 numbers each, x = hi + lo (hi rounded to 11 bits, of lo the first 11 count), and a product is
// hi hi' + hi lo' + lo hi': 2^-21 of it at worst, zero on average.  The tensor core cuts its sums off instead of rounding them, so the
// large products' accumulator is taken out every 64 of the contracted index and added up in fp32, and the small ones have their own.
//
// The order of the contracted index is free as long as both operands share it: a lane takes consecutive elements of its rows,
// which makes 128-bit loads of a weight row that lies in memory as it is.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstdint>

namespace evo {
namespace gm {

__device__ __forceinline__ void mma_tf32(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <typename T>
__device__ __forceinline__ void mma_16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (sizeof(T) == 2 && __is_same(T, __half))
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// hi is rounded to nearest by hand (cvt.rna.tf32 is a sequence of instructions: 4,096 members of 28-128-128-8 took 62 million warp
// instructions with it and 53 without).  Of an infinity the low part is a NaN, which only reaches the small products' sums: they do not
// count where the large ones' sum is no finite number, and then it is what the plain product would be.  A NaN that rounds to something else stays one
// in its low part.  (Numbers above 3.4011e38 round to an infinity.)
__device__ __forceinline__ void split(float x, uint32_t& hi, uint32_t& lo)
{
    hi = (__float_as_uint(x) + 0x1000u) & 0xFFFFE000u;
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ float join(float large, float small) { return isfinite(large) ? large + small : large; }

// tanh without branches: up to 1/2 the series of tanh to x^13 (what is left out is below 1e-7 of the result), beyond it
// 1 - 2 / (e^2|x| + 1) with the hardware's exponential (2^-22 relative) and reciprocal (2^-23): by these bounds 5.5e-7 of the result at worst, at 1/2.
// Measured over all multiples of 2^-18 up to 16: 2.2e-7, at 0.568
__device__ __forceinline__ float tanh32(float x)
{
    const float a = fabsf(x), s = x * x;
    float p = 21844.0f / 6081075.0f;
    p = fmaf(p, s, -1382.0f / 155925.0f);
    p = fmaf(p, s, 62.0f / 2835.0f);
    p = fmaf(p, s, -17.0f / 315.0f);
    p = fmaf(p, s, 2.0f / 15.0f);
    p = fmaf(p, s, -1.0f / 3.0f);
    const float near = fmaf(x * s, p, x);
    float e, r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(a * 2.885390082f));      // 2 log2(e)
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(e + 1.0f));
    return a < 0.5f ? near : copysignf(fmaf(-2.0f, r, 1.0f), x);
}

}  // namespace gm
}  // namespace evo

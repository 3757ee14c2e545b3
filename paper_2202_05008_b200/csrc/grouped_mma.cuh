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

// Of an infinity the low part is a NaN, which only reaches the small products' sums: they do not count where the large ones' sum is
// no finite number, and then it is what the plain product would be.  (Numbers above 3.4011e38 round to an infinity.)
__device__ __forceinline__ void split(float x, uint32_t& hi, uint32_t& lo)
{
    asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(hi) : "f"(x));
    lo = __float_as_uint(x - __uint_as_float(hi));
}
__device__ __forceinline__ float join(float large, float small) { return isfinite(large) ? large + small : large; }

}  // namespace gm
}  // namespace evo

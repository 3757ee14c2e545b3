// tcgen05 operands that TMA brings with the 128-byte swizzle, and the instruction's descriptor, for the products grouped by member and their gradients.
#pragma once
#include <type_traits>

#include "grouped.h"
#include "tma.h"
#include "umma.cuh"

namespace evo {

// K-major operand of rows of 128 bytes with the 128-byte swizzle, groups of 8 rows side by side
__device__ __forceinline__ uint64_t desc_sw128(uint32_t addr)
{
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(1) << 16 | static_cast<uint64_t>(64) << 32 |
           static_cast<uint64_t>(1) << 46 | static_cast<uint64_t>(2) << 61;
}
// MN-major operand: a row of 128 bytes is 64 of its rows (or columns) at one contracted index; the next 64 of them lie `apart` bytes further, 8 contracted indices 1,024
__device__ __forceinline__ uint64_t desc_sw128_mn(uint32_t addr, uint32_t apart)
{
    return static_cast<uint64_t>((addr & 0x3FFFFu) >> 4) | static_cast<uint64_t>(apart >> 4) << 16 | static_cast<uint64_t>(64) << 32 |
           static_cast<uint64_t>(1) << 46 | static_cast<uint64_t>(2) << 61;
}
// 128 x n, sums in fp32; A_MN, B_MN: operands that are MN-major
template <typename T, bool A_MN = false, bool B_MN = false>
__device__ __forceinline__ uint32_t idesc(uint32_t n)
{
    const uint32_t type = std::is_same<T, __half>::value ? 0u : 1u;
    return (1u << 4) | (type << 7) | (type << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((n >> 3) << 17) | ((128u >> 4) << 24);
}

__device__ __forceinline__ void copy2(uint32_t dst, const CUtensorMap* map, uint32_t c0, uint32_t c1, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
__device__ __forceinline__ void copy3(uint32_t dst, const CUtensorMap* map, uint32_t c0, uint32_t c1, uint32_t c2, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// Numbers as 16-bit parts whose sum they are: three bf16 ones of fp32 (24 bits, no exponent is lost), of which the six products down to 2^-16 of the largest
// count, the small ones first.  kPartW / kPartX: which parts (0 the largest) of the two operands a pass multiplies; an operand that has one part beside two: kPartOne, kPartTwo.
__constant__ const uint8_t kPartW[6] = { 0, 2, 1, 0, 1, 0 }, kPartX[6] = { 2, 0, 1, 1, 0, 0 }, kPartTwo[2] = { 1, 0 };

// An infinity or a NaN has no further parts (the product of an infinity's with a zero would be NaN); a number that would round to an infinity, from 3.396e38 on, is
// cut off instead.  (Without branches, so that the loads of several numbers run ahead.)
__device__ __forceinline__ void three_parts(float x, uint16_t* first, uint16_t* second, uint16_t* third)
{
    uint32_t part = __bfloat16_as_ushort(__float2bfloat16_rn(x));
    part -= (part & 0x7FFFu) == 0x7F80u && fabsf(x) <= 3.402823466e38f ? 1u : 0u;
    const float back = __uint_as_float(part << 16);
    const float rest = fabsf(back) <= 3.402823466e38f ? x - back : 0.f;
    const __nv_bfloat16 middle = __float2bfloat16_rn(rest);
    *first = static_cast<uint16_t>(part);
    *second = __bfloat16_as_ushort(middle);
    *third = __bfloat16_as_ushort(__float2bfloat16_rn(rest - __bfloat162float(middle)));
}

}  // namespace evo

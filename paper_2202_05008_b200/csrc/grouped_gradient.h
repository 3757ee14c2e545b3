// Arguments and launchers of the gradients of the products grouped by member (grouped_gradient.cu).
#pragma once
#include <cuda_fp16.h>

#include <type_traits>

#include "grouped.h"

namespace evo {

struct GradientArgs {
    GroupedArgs f;                       // the product: its b is unused, y is read
    const void* dy; void* dx; void* dw; void* db;
    uint64_t ld_dy, ld_dx, ld_dw, stride_dw, stride_db;
    uint32_t sum_w, sum_b;               // one gradient for all groups together
    float inverse;                       // 1 / scale
    uint32_t late;                       // see dep_begin
};

// dx, dW and db have nothing in common: a kernel that follows one of the others (which has waited for what both read before it let this one start) waits for it at its own
// end only, so that it fills the SMs that the one before leaves.
__device__ __forceinline__ void dep_begin(const GradientArgs& a)
{
    if (!a.late) dep_wait();
    dep_trigger();
}
__device__ __forceinline__ void dep_end(const GradientArgs& a)
{
    if (a.late) dep_wait();
}

// dz = dy scale act'(z), from y = scale act(z).  scale - y is exact close to the ends of tanh; scale + y is divided by scale before the two meet, since scale squared may be no number.
__device__ __forceinline__ float dz_of(const GradientArgs& a, float dy, float y)
{
    const float scale = a.f.scale;
    if (a.f.activation == EVO_ACT_TANH) return dy * ((scale - y) * ((scale + y) * a.inverse));
    if (a.f.activation == EVO_ACT_RELU) return (scale > 0.f ? y > 0.f : y < 0.f) ? dy * scale : 0.f;
    return dy * scale;
}

// dz / scale: no larger than dy
__device__ __forceinline__ float dz_unit(const GradientArgs& a, float dy, float y)
{
    if (a.f.activation == EVO_ACT_TANH) return dy * ((a.f.scale - y) * a.inverse) * ((a.f.scale + y) * a.inverse);
    if (a.f.activation == EVO_ACT_RELU) return (a.f.scale > 0.f ? y > 0.f : y < 0.f) ? dy : 0.f;
    return dy;
}
// dz / scale of 16-bit types in two numbers of the type, where it is not dy or 0: the second is what the first leaves, of fp16 times 2^kSecondUp, since what is left of small
// numbers lies below fp16's own (without that dz was off by up to 2^-25 whatever its size; so by 2^-22 of itself, or 2^-36).  Sums of second numbers are taken down again before those
// of the first ones join them.
constexpr uint32_t kSecondUp = 11;
template <typename T> constexpr float kUp = std::is_same<T, __half>::value ? static_cast<float>(1u << kSecondUp) : 1.f;
template <typename T> constexpr float kDown = 1.f / kUp<T>;
// Rows of a set (a group, or all of them together) between two offsets, inside [0, rows], of which split `split` of `splits` has its part, a multiple of 16 rows.
__device__ __forceinline__ void split_rows(const GradientArgs& a, int64_t p, int64_t q, uint32_t split, uint32_t splits, uint64_t* first, uint64_t* end)
{
    const int64_t top = static_cast<int64_t>(a.f.rows);
    p = p < 0 ? 0 : p > top ? top : p;
    q = q < p ? p : q > top ? top : q;
    *first = static_cast<uint64_t>(p);
    *end = static_cast<uint64_t>(q);
    if (splits == 1u) return;
    const uint64_t per = ((*end - *first + splits - 1u) / splits + 15u) / 16u * 16u;
    const uint64_t f = *first + split * per;
    *end = min(*end, f + per);
    *first = f;                                              // (behind the end: no rows)
}
__device__ __forceinline__ void set_rows(const GradientArgs& a, bool all, uint32_t set, uint32_t split, uint32_t splits, uint64_t* first, uint64_t* end)
{
    const uint32_t behind = all ? a.f.groups : set + 1u;
    if (a.f.wide_offsets) split_rows(a, static_cast<const int64_t*>(a.f.offsets)[set], static_cast<const int64_t*>(a.f.offsets)[behind], split, splits, first, end);
    else split_rows(a, static_cast<const int32_t*>(a.f.offsets)[set], static_cast<const int32_t*>(a.f.offsets)[behind], split, splits, first, end);
}

size_t grouped_gradient_bytes(uint32_t type, const GradientArgs& a, bool any_address);      // workspace; any_address: enough wherever the inputs lie
int launch_grouped_gradient(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work);

// grouped_gradient_tc.cu: dx and dW on tcgen05, and what has to be laid out in the workspace for that
struct TcPlan {
    bool dx, dw, lay_dz, lay_x, lay_w;
    uint32_t dz_parts, pitch_dz, pitch, long_rows;
    uint64_t dz_bytes, x_bytes, w_bytes, sum_bytes;
    uint64_t bytes() const { return dz_bytes + x_bytes + w_bytes + sum_bytes; }
};
TcPlan grouped_gradient_tc_plan(uint32_t type, const GradientArgs& a, bool dx, bool dw, uint32_t splits, bool any_address);
int launch_grouped_gradient_tc(cudaStream_t st, uint32_t type, const GradientArgs& a, const TcPlan& plan, uint32_t splits, float* part, void* work);

}  // namespace evo

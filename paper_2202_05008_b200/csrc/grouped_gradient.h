// Arguments and launchers of the gradients of the products grouped by member (grouped_gradient.cu).
#pragma once
#include "grouped.h"

namespace evo {

struct GradientArgs {
    GroupedArgs f;                       // the product: its b is unused, y is read
    const void* dy; void* dx; void* dw; void* db;
    uint64_t ld_dy, ld_dx, ld_dw, stride_dw, stride_db;
    uint32_t sum_w, sum_b;               // one gradient for all groups together
    float inverse;                       // 1 / scale
};

// dz = dy scale act'(z), from y = scale act(z).  scale - y is exact close to the ends of tanh.
__device__ __forceinline__ float dz_of(const GradientArgs& a, float dy, float y)
{
    const float scale = a.f.scale;
    if (a.f.activation == EVO_ACT_TANH) return dy * ((scale - y) * (scale + y) * a.inverse);
    if (a.f.activation == EVO_ACT_RELU) return (scale > 0.f ? y > 0.f : y < 0.f) ? dy * scale : 0.f;
    return dy * scale;
}

size_t grouped_gradient_bytes(uint32_t type, const GradientArgs& a);   // workspace; with addresses of 0, enough for any
int launch_grouped_gradient(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work);

}  // namespace evo

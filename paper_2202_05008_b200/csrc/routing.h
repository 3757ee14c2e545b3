// Arguments and launchers of the rows sorted by member (routing.cu, rows.cu).  Launchers: kernels launched, -1: a CUDA error, -2: more than 2^31 blocks.
#pragma once
#include "internal.h"

namespace evo {

struct RouteArgs {
    const void* members;
    uint64_t ld;
    uint32_t wide, choices, groups, pairs;
    int32_t* offsets; int32_t* source; int32_t* place;
};
size_t route_bytes(const RouteArgs& a);                      // workspace
int launch_route(cudaStream_t st, const RouteArgs& a, void* work);

struct RowSetArgs {
    const int32_t* place;
    const float* weights;                                    // or NULL: 1
    void* rows; void* sorted; void* d_sorted;
    float* d_weights;
    uint64_t count, ld_place, ld_weights, ld_rows, ld_sorted, ld_d_sorted, ld_d_weights;
    uint32_t sorted_rows, choices, cols;
};
int launch_take(cudaStream_t st, uint32_t type, const RowSetArgs& a);
int launch_combine(cudaStream_t st, uint32_t type, const RowSetArgs& a);
int launch_combine_backward(cudaStream_t st, uint32_t type, const RowSetArgs& a);

}  // namespace evo

// Arguments and launchers of the products grouped by member (grouped.cu, grouped_tc.cu).
#pragma once
#include "internal.h"

namespace evo {

// y[r] = scale act(W_g x[r] + b_g) for the rows offsets[g] <= r < offsets[g + 1] of every group
struct GroupedArgs {
    const void* x; const void* w; const void* b; void* y;
    const void* offsets;
    uint32_t wide_offsets;               // 64-bit ones
    uint32_t groups, n_in, n_out, activation;
    uint64_t rows, ld_x, ld_y, ld_w, stride_w, stride_b;
    float scale;
};

// First row and the one behind the last of a group, inside [0, rows] whatever the offsets hold.
__device__ __forceinline__ void group_rows(const GroupedArgs& a, uint32_t g, uint64_t* first, uint64_t* end)
{
    int64_t p, q;
    if (a.wide_offsets) {
        p = static_cast<const int64_t*>(a.offsets)[g];
        q = static_cast<const int64_t*>(a.offsets)[g + 1u];
    } else {
        p = static_cast<const int32_t*>(a.offsets)[g];
        q = static_cast<const int32_t*>(a.offsets)[g + 1u];
    }
    const int64_t top = static_cast<int64_t>(a.rows);
    p = p < 0 ? 0 : p > top ? top : p;
    q = q < p ? p : q > top ? top : q;
    *first = static_cast<uint64_t>(p);
    *end = static_cast<uint64_t>(q);
}

// The limit of a wait inside the kernels on tcgen05, and whether the first block leaves out a completion (evo_debug_grouped_waits): 31 and no but in the checked build.
struct Waits { uint32_t cycles_log2, drop; };
Waits grouped_waits();
constexpr uint32_t kLongestWait = 31;

size_t grouped_bytes(uint32_t type, const GroupedArgs& a);             // workspace
int launch_grouped(cudaStream_t st, uint32_t type, const GroupedArgs& a, void* work);
// grouped_tc.cu: 16-bit types whose rows TMA can address as they lie, where that pays, or (work) rows that are laid out for it first
bool grouped_tc_addressable(uint32_t type, const GroupedArgs& a);
bool grouped_tc_takes(uint32_t type, const GroupedArgs& a);
size_t grouped_tc_bytes(uint32_t type, const GroupedArgs& a);
int launch_grouped_tc(cudaStream_t st, uint32_t type, const GroupedArgs& a, void* work);
// Pieces of it, for the gradients.  Rows laid out: their pitch (fp32: of one of three parts), and the launch for the weights or (rows) x.
uint32_t grouped_tc_pitch(uint32_t type, uint32_t n);
int lay_out(cudaStream_t st, uint32_t type, const GroupedArgs& a, bool rows, uint32_t pitch, uint16_t* to);
// The product with weights [n_in][n_out], whose rows are the contracted index, of operands that TMA can address: `passes` 1; 2: x has two parts; 6: both three.
int launch_grouped_tc_transposed(cudaStream_t st, uint32_t type, const GroupedArgs& a, uint32_t passes, uint32_t pitch_w, uint32_t pitch_x, uint64_t span_w, uint64_t span_x);

}  // namespace evo

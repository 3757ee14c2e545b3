// Plan and launcher of the kernel that takes fp32 rows through the layers of their member's policy (member_rows.cu).
#pragma once
#include "grouped.h"

namespace evo {

struct MemberArgs {
    GroupedArgs g;                       // x, y, offsets, groups = members, rows, pitches of x and y, scale
    const float* theta;                  // of member 0, 16-byte aligned
    uint64_t stride;                     // from one member to the next, a multiple of 4
    uint32_t n_layers, chunks;           // chunks: parts of a single layer's outputs
    uint32_t sizes[EVO_MAX_LAYERS + 1], w_at[EVO_MAX_LAYERS], b_at[EVO_MAX_LAYERS];
    uint32_t aligned;                    // which layers' weight rows are 16-byte aligned
    uint32_t ld, row_tiles;
};
// Plan for layers of sizes[l] by sizes[l + 1] whose weights and biases lie at w_at and b_at: fills in what the kernel needs besides.  False where the activations
// of a layer do not fit.
bool member_plan(MemberArgs* a);
int launch_member_rows(cudaStream_t st, const MemberArgs& a);

}  // namespace evo

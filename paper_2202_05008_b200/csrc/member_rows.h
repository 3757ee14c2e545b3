// Plan and launcher of the kernel that takes fp32 rows through their member's layers (member_rows.cu): all of an MLP policy's, or one.
#pragma once
#include "grouped.h"

namespace evo {

struct MemberArgs {
    GroupedArgs g;                       // x, y, offsets, groups = members, rows, pitches of x and y, activation of the last layer, scale
    const float* w; const float* b;      // of member 0; b may be NULL
    uint64_t stride_w, stride_b;         // from one member to the next
    uint32_t n_layers, chunks;           // chunks: parts of the (single) layer's outputs
    uint32_t sizes[EVO_MAX_LAYERS + 1], w_at[EVO_MAX_LAYERS], b_at[EVO_MAX_LAYERS], ld_w[EVO_MAX_LAYERS];
    uint32_t aligned;                    // which layers' weight rows are 16-byte aligned
    uint32_t ld, row_tiles, team;        // team: warps that share an item
};
// Plan for layers of sizes[l] by sizes[l + 1] whose weights lie at w_at (rows ld_w apart) of members stride_w apart: fills in what the kernel
// needs besides.  False where the activations of a layer do not fit.
bool member_plan(MemberArgs* a);
int launch_member_rows(cudaStream_t st, const MemberArgs& a);

}  // namespace evo

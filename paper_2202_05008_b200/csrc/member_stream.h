// Plan and launcher of the kernel that streams members' fp32 weights (member_stream.cu): all layers of an MLP policy, or one layer.
#pragma once
#include "grouped.h"

namespace evo {

struct StreamArgs {
    GroupedArgs g;                       // x, y, offsets, groups = members, rows, pitches of x and y, activation of the last layer, scale
    const float* w; const float* b;      // of member 0; b may be NULL
    uint64_t stride_w, stride_b;         // from one member to the next
    uint64_t w_end;                      // floats that a member has from its first weight on
    uint32_t n_layers, chunks, shares;   // chunks: parts of the (single) layer's outputs; shares: of a member's rows
    uint32_t sizes[EVO_MAX_LAYERS + 1], w_at[EVO_MAX_LAYERS], b_at[EVO_MAX_LAYERS];
    uint32_t tiles_a_stage[EVO_MAX_LAYERS], aligned;     // sixteens of outputs that come together; which layers' weight rows are 16-byte aligned
    uint32_t stage_floats, stages, ld_in, ld_hidden, bias_floats, row_tiles;
};
// Plan for `n_layers` layers whose weights lie at w_at (rows of sizes[l] floats), members stride_w apart.  Fills in what the kernel needs besides the
// pointers; false where a stage of 16 weight rows or the activations do not fit a block.
bool stream_plan(StreamArgs* a, size_t* bytes);
int launch_stream(cudaStream_t st, const StreamArgs& a, size_t bytes);

}  // namespace evo

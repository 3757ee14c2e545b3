// Plan and launcher of the policy's actions (mlp_actions.cu).
#pragma once
#include "grouped.h"

namespace evo {

struct ActionsArgs {
    GroupedArgs g;                       // x = observations, y = actions, groups = members, scale
    const float* theta;
    uint64_t ld_theta;
    uint32_t n_layers, dim, aligned, ld_act, act_at, shares;
    uint32_t sizes[EVO_MAX_LAYERS + 1], layer_at[EVO_MAX_LAYERS], piece[EVO_MAX_LAYERS + 1];
};
// Layout of a block's shared memory; false where a member does not fit it.
bool actions_plan(const uint32_t* sizes, uint32_t n_layers, ActionsArgs* a, size_t* bytes);
int launch_actions(cudaStream_t st, const ActionsArgs& a, size_t bytes);

}  // namespace evo

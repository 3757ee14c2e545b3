// Arguments and launcher of the clipped policy loss (policy_loss.cu).
#pragma once
#include "internal.h"

namespace evo {

struct PolicyArgs {
    const void* logits; void* gradient;
    const void* action;
    const float* old_logp; const float* advantage; const float* ref_logp; const float* weights;      // the last two may be NULL
    float* logp; float* loss;
    double* row_loss;                                        // workspace, where the loss is wanted
    uint64_t rows, ld, ld_gradient;
    uint32_t n, wide;
    double clip_low, clip_high, kl, even;                    // even: the weight of a row without weights
    double log_low, log_high;                                // of 1 - clip_low and 1 + clip_high
};
size_t policy_loss_bytes(uint64_t rows);                  // workspace, where the loss is wanted
int launch_policy_loss(cudaStream_t st, uint32_t type, const PolicyArgs& a);

}  // namespace evo

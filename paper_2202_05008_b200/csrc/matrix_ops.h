// Launchers of the matrix operators (host side): lists of matrices for the Newton-Schulz kernels, and the Muon step.
#pragma once
#include <vector>

#include "internal.h"
#include "newton_schulz.h"

namespace evo {
namespace ns {

// `count` equal matrices of the caller
struct Matrix {
    uint64_t in, out, in_stride, out_stride;
    uint32_t rows, cols, in_ld, out_ld, count;
    float gain;
};

int launch_tiny(cudaStream_t st, uint32_t source, const Args& a, uint32_t row_tiles, uint32_t warps);
int launch_small(cudaStream_t st, uint32_t source, const Args& a, size_t smem);
int launch_large(cudaStream_t st, uint32_t source, const Args& a);

// Workspace of a list (0 where all matrices are small); ~0 if its blocks or tiles cannot be numbered in 32 bits
size_t workspace_bytes(const Matrix* list, size_t n);
// All matrices of the list.  `base` holds the pointers and scalars; the rest is filled in here.
int launch(cudaStream_t st, uint32_t source, const Matrix* list, size_t n, const Args& base, char* work);

}  // namespace ns

// the quintic and the eps that 0 selects
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f, kNsEps = 1e-7f;

struct MuonArgs {
    const float *center, *m, *v, *g;
    float *center_out, *m_out, *v_out;
    uint64_t dim;
    uint32_t step;                     // number of this step, from 1 ...
    const uint32_t* d_step;            // ... unless it stands here, on the device
    const double* skip;                // nothing is done where this is 0 (NULL: always)
    double lr, mu, decay, beta1, beta2, adam_eps;
    uint32_t nesterov, ns_steps;
    float a, b, c, ns_eps;
    char* work;
    uint32_t* sticky;
    uint32_t wait_log2, drop;
};
bool muon_scalars(const MuonArgs& a, ns::Scalars* s);       // false: an iteration that grows beyond fp16 pairs
size_t muon_workspace_bytes(const evo_matrix* list, size_t n);
int launch_muon(cudaStream_t st, const evo_matrix* list, size_t n, const MuonArgs& a);
// weight matrices of a solver's policy inside its parameter vector; returns how many
uint32_t policy_matrices(const evo_config& c, evo_matrix (&out)[EVO_MAX_LAYERS]);

}  // namespace evo

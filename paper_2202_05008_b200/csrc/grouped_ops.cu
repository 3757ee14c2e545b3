// C entry points of the products grouped by member and of the policy's actions.
#include <atomic>
#include <cmath>
#include <cstring>

#include "grouped.h"
#include "member_rows.h"

using namespace evo;

namespace {

constexpr uint64_t kMost = 1ull << 40;       // elements of a pitch or a stride, and rows

#ifdef EVO_DEBUG
std::atomic<uint32_t> test_waits { kLongestWait }, test_drop { 0u };
#endif

// the layers of a policy as the kernel for rows and layers takes them
void policy_layers(const evo_actions& p, MemberArgs* a)
{
    uint64_t at = 0;
    a->n_layers = p.n_layers;
    for (uint32_t l = 0; l <= p.n_layers; ++l) a->sizes[l] = p.layer_sizes[l];
    for (uint32_t l = 0; l < p.n_layers; ++l) {
        a->w_at[l] = static_cast<uint32_t>(at);
        at += static_cast<uint64_t>(p.layer_sizes[l]) * p.layer_sizes[l + 1];
        a->b_at[l] = static_cast<uint32_t>(at);
        at += p.layer_sizes[l + 1];
    }
    a->g.rows = p.rows;
    a->g.groups = p.members;
}

// rows of the layers between the first and the last, twice, for a policy that one block does not hold
size_t layers_bytes(const evo_actions& a)
{
    uint64_t widest = 0;
    for (uint32_t l = 1; l < a.n_layers; ++l) widest = a.layer_sizes[l] > widest ? a.layer_sizes[l] : widest;
    return static_cast<size_t>(2u * a.rows * ((widest + 3u) / 4u * 4u) * sizeof(float));
}

// Whether a launch per layer is the faster way: few rows a member and many weights, in layers that the kernel for one short layer takes (it reads
// them at 5.1 TB/s, the one for all layers at 2.5).  All layers / one after the other: 28-128-128-8, 300 members of 4 rows 15.5 / 19.6 us, 1,000 59.9 / 30.9,
// 4,096 140 / 107; 28-64-64-64-64-8, 1,000 47.8 / 31.6, 4,000 of 6 rows 112 / 99.5; 5-64-64-1, 1,000 28.4 / 21.8; 9-179-38-13 (not aligned), 4,000 145 / 177.
bool by_layers(const evo_actions& p)
{
    uint64_t dim = 0, at = 0;
    bool simple = p.n_layers > 1u;
    for (uint32_t l = 0; l < p.n_layers; ++l) {
        const uint64_t in = p.layer_sizes[l], out = p.layer_sizes[l + 1];
        if (in > 16u && (in > 128u || (in | at) % 4u)) simple = false;
        dim += in * out;
        at += (in + 1u) * out;
    }
    return simple && p.rows <= 8ull * p.members && dim * p.members >= (1u << 22);
}

evo_status check_actions(const evo_actions* a)
{
    if (!a || a->struct_size != sizeof(evo_actions) || a->members < 1u || a->n_layers < 1u || a->n_layers > EVO_MAX_LAYERS) return EVO_ERR_INVALID_ARG;
    uint64_t dim = 0;
    for (uint32_t l = 0; l <= a->n_layers; ++l)
        if (a->layer_sizes[l] < 1u || a->layer_sizes[l] > (1u << 20)) return EVO_ERR_INVALID_ARG;
    for (uint32_t l = 0; l < a->n_layers; ++l) dim += static_cast<uint64_t>(a->layer_sizes[l] + 1u) * a->layer_sizes[l + 1];
    if (dim > kMaxParamDim || a->ld_theta < dim || a->ld_theta > kMost || (a->ld_theta & 3u)) return EVO_ERR_INVALID_ARG;
    if (a->rows > kMost || a->members > 0x7FFFFFFFu || a->offsets_64 > 1u || !std::isfinite(a->action_scale)) return EVO_ERR_INVALID_ARG;
    return EVO_OK;
}

}  // namespace

#ifdef EVO_DEBUG
evo::Waits evo::grouped_waits() { return { test_waits.load(), test_drop.load() }; }
#else
evo::Waits evo::grouped_waits() { return { kLongestWait, 0u }; }
#endif

extern "C" {

evo_status evo_debug_grouped_waits(uint32_t wait_cycles_log2, uint32_t drop_completion)
{
    if (wait_cycles_log2 < 10u || wait_cycles_log2 > kLongestWait || drop_completion > 1u) return EVO_ERR_INVALID_ARG;
#ifdef EVO_DEBUG
    test_waits = wait_cycles_log2;
    test_drop = drop_completion;
    return EVO_OK;
#else
    return EVO_ERR_UNSUPPORTED;
#endif
}

static evo_status check_grouped(const evo_grouped* p)
{
    if (!p || p->struct_size != sizeof(evo_grouped) || p->type > EVO_F16 || p->activation > EVO_ACT_RELU || p->offsets_64 > 1u) return EVO_ERR_INVALID_ARG;
    if (p->groups < 1u || p->groups > 0x7FFFFFFFu || p->n_in < 1u || p->n_out < 1u || p->n_in > (1u << 20) || p->n_out > (1u << 20)) return EVO_ERR_INVALID_ARG;
    if (p->rows > kMost || p->ld_x > kMost || p->ld_y > kMost || p->ld_weight > kMost || p->weight_stride > kMost || p->bias_stride > kMost) return EVO_ERR_INVALID_ARG;
    if (!std::isfinite(p->scale)) return EVO_ERR_INVALID_ARG;
    if ((p->rows > 1u && (p->ld_x < p->n_in || p->ld_y < p->n_out)) || (p->n_out > 1u && p->ld_weight < p->n_in)) return EVO_ERR_INVALID_ARG;
    return EVO_OK;
}

static GroupedArgs grouped_args(const evo_grouped* p)
{
    GroupedArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = p->d_x; a.w = p->d_weight; a.b = p->d_bias; a.y = p->d_y; a.offsets = p->d_offsets; a.wide_offsets = p->offsets_64;
    a.groups = p->groups; a.n_in = p->n_in; a.n_out = p->n_out; a.activation = p->activation; a.scale = p->scale;
    // a pitch that is never taken may be anything
    a.rows = p->rows; a.ld_x = p->rows > 1u ? p->ld_x : 0u; a.ld_y = p->ld_y; a.ld_w = p->n_out > 1u ? p->ld_weight : 0u;
    a.stride_w = p->groups > 1u ? p->weight_stride : 0u; a.stride_b = p->bias_stride;
    return a;
}

evo_status evo_grouped_linear_bytes(const evo_grouped* p, size_t* bytes)
{
    const evo_status st = check_grouped(p);
    if (st != EVO_OK || !bytes) return EVO_ERR_INVALID_ARG;
    // (before the buffers exist: as much as they need wherever they lie)
    const GroupedArgs a = grouped_args(p);
    *bytes = p->rows == 0u ? 0u : p->d_x && p->d_weight ? grouped_bytes(p->type, a) : grouped_tc_bytes(p->type, a);
    return EVO_OK;
}

evo_status evo_grouped_linear(const evo_grouped* p, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    const evo_status st = check_grouped(p);
    if (st != EVO_OK) return st;
    if (p->rows == 0u) return EVO_OK;
    const uint64_t size = p->type == EVO_F32 ? 4u : 2u;
    const uintptr_t bits = reinterpret_cast<uintptr_t>(p->d_x) | reinterpret_cast<uintptr_t>(p->d_weight) | reinterpret_cast<uintptr_t>(p->d_bias) |
                           reinterpret_cast<uintptr_t>(p->d_y);
    if (!p->d_x || !p->d_weight || !p->d_y || !p->d_offsets || (bits & (size - 1u))) return EVO_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->d_offsets) & (p->offsets_64 ? 7u : 3u)) return EVO_ERR_INVALID_ARG;
    // (weights and biases may be shared by groups: stride 0)
    uint64_t x_bytes, y_bytes, set, w_bytes, b_bytes = 0;
    if (!extent(p->rows, p->ld_x, p->n_in, size, &x_bytes) || !extent(p->rows, p->ld_y, p->n_out, size, &y_bytes) ||
        !extent(p->n_out, p->ld_weight, p->n_in, 1u, &set) || !extent(p->groups, p->weight_stride, set, size, &w_bytes) ||
        (p->d_bias && !extent(p->groups, p->bias_stride, p->n_out, size, &b_bytes)))
        return EVO_ERR_INVALID_ARG;
    if (overlap(p->d_y, y_bytes, p->d_x, x_bytes) || overlap(p->d_y, y_bytes, p->d_weight, w_bytes) || (p->d_bias && overlap(p->d_y, y_bytes, p->d_bias, b_bytes)) ||
        overlap(p->d_y, y_bytes, p->d_offsets, (p->groups + 1ull) * (p->offsets_64 ? 8u : 4u)))
        return EVO_ERR_INVALID_ARG;
    const GroupedArgs a = grouped_args(p);
    const size_t need = grouped_bytes(p->type, a);
    if (need && (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255u))) return EVO_ERR_INVALID_ARG;
    if (workspace_bytes < need) return EVO_ERR_WORKSPACE;
    const int n = launch_grouped(static_cast<cudaStream_t>(cuda_stream), p->type, a, need ? d_workspace : nullptr);
    return n == -2 ? EVO_ERR_UNSUPPORTED : n < 0 ? EVO_ERR_CUDA : EVO_OK;
}

evo_status evo_mlp_actions_bytes(const evo_actions* p, size_t* bytes)
{
    const evo_status st = check_actions(p);
    if (st != EVO_OK || !bytes) return EVO_ERR_INVALID_ARG;
    MemberArgs a;
    std::memset(&a, 0, sizeof(a));
    policy_layers(*p, &a);
    *bytes = member_plan(&a) && !by_layers(*p) ? 0u : layers_bytes(*p);
    return EVO_OK;
}

evo_status evo_mlp_actions(const evo_actions* p, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    size_t need = 0;
    const evo_status st = evo_mlp_actions_bytes(p, &need);
    if (st != EVO_OK) return st;
    const uint32_t n_in = p->layer_sizes[0], n_out = p->layer_sizes[p->n_layers];
    if (p->rows == 0u) return EVO_OK;
    if (!p->d_theta || !p->d_observations || !p->d_actions || !p->d_offsets || (reinterpret_cast<uintptr_t>(p->d_theta) & 15u)) return EVO_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(p->d_observations) | reinterpret_cast<uintptr_t>(p->d_actions)) & 3u) return EVO_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p->d_offsets) & (p->offsets_64 ? 7u : 3u)) return EVO_ERR_INVALID_ARG;
    if (p->ld_observations > kMost || p->ld_actions > kMost || (p->rows > 1u && (p->ld_observations < n_in || p->ld_actions < n_out))) return EVO_ERR_INVALID_ARG;
    uint64_t dim = 0, in_bytes, out_bytes, theta_bytes;
    for (uint32_t l = 0; l < p->n_layers; ++l) dim += (p->layer_sizes[l] + 1ull) * p->layer_sizes[l + 1];
    if (!extent(p->rows, p->ld_observations, n_in, 4u, &in_bytes) || !extent(p->rows, p->ld_actions, n_out, 4u, &out_bytes) ||
        !extent(p->members, p->ld_theta, dim, 4u, &theta_bytes))
        return EVO_ERR_INVALID_ARG;
    if (overlap(p->d_actions, out_bytes, p->d_observations, in_bytes) || overlap(p->d_actions, out_bytes, p->d_theta, theta_bytes) ||
        overlap(p->d_actions, out_bytes, p->d_offsets, (p->members + 1ull) * (p->offsets_64 ? 8u : 4u)))
        return EVO_ERR_INVALID_ARG;
    if (need && (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255u))) return EVO_ERR_INVALID_ARG;
    if (workspace_bytes < need) return EVO_ERR_WORKSPACE;
    const cudaStream_t stream = static_cast<cudaStream_t>(cuda_stream);
    MemberArgs a;
    std::memset(&a, 0, sizeof(a));
    policy_layers(*p, &a);
    a.theta = p->d_theta; a.stride = p->ld_theta;
    GroupedArgs& g = a.g;
    g.x = p->d_observations; g.y = p->d_actions; g.offsets = p->d_offsets; g.wide_offsets = p->offsets_64;
    g.ld_x = p->rows > 1u ? p->ld_observations : 0u; g.ld_y = p->ld_actions; g.activation = EVO_ACT_TANH; g.scale = p->action_scale;
    if (need == 0u && member_plan(&a)) {
        const int n = launch_member_rows(stream, a);
        return n == -2 ? EVO_ERR_UNSUPPORTED : n < 0 ? EVO_ERR_CUDA : EVO_OK;
    }
    // a launch per layer, hidden rows in the workspace
    float* const hidden[2] = { static_cast<float*>(d_workspace), static_cast<float*>(d_workspace) + need / 8u };
    uint64_t at = 0;
    for (uint32_t l = 0; l < p->n_layers; ++l) {
        const bool last = l + 1u == p->n_layers;
        GroupedArgs b = g;
        b.n_in = p->layer_sizes[l]; b.n_out = p->layer_sizes[l + 1];
        if (l) { b.x = hidden[l & 1u]; b.ld_x = (b.n_in + 3u) / 4u * 4u; }
        if (!last) { b.y = hidden[(l + 1u) & 1u]; b.ld_y = (b.n_out + 3u) / 4u * 4u; b.scale = 1.f; }
        b.w = p->d_theta + at; b.ld_w = b.n_in; b.stride_w = p->ld_theta;
        at += static_cast<uint64_t>(b.n_in) * b.n_out;
        b.b = p->d_theta + at; b.stride_b = p->ld_theta;
        at += b.n_out;
        const int n = launch_grouped(stream, EVO_F32, b, nullptr);
        if (n < 0) return n == -2 ? EVO_ERR_UNSUPPORTED : EVO_ERR_CUDA;
    }
    return EVO_OK;
}

}  // extern "C"

// Host side of the orthogonalised updates: lists of matrices, the Muon step of a parameter vector, and their C entry points.
#include "matrix_ops.h"

#include <algorithm>
#include <cstring>
#include <new>

namespace evo {
namespace ns {

static uint32_t up(uint32_t x, uint32_t a) { return (x + a - 1u) / a * a; }

// blocks: of the cluster that takes a small matrix, 0: a large one
static Group group_for(const Matrix& x, uint32_t blocks)
{
    Group g = {};
    g.in = x.in; g.out = x.out; g.in_stride = x.in_stride; g.out_stride = x.out_stride; g.in_ld = x.in_ld; g.out_ld = x.out_ld;
    g.tall = x.rows > x.cols;
    g.m = g.tall ? x.cols : x.rows;
    g.n = g.tall ? x.rows : x.cols;
    g.mp = up(g.m, blocks ? 16u : kTile);
    g.np = blocks ? up((g.n + blocks - 1u) / blocks, 16u) : up(g.n, kPieceCols);
    g.count = x.count;
    g.gain = x.gain;
    return g;
}
static Choice choice_of(const Matrix& x) { return choose(std::min(x.rows, x.cols), std::max(x.rows, x.cols), x.count); }

// Lists the large matrices from *at on, as many as a launch takes; advances *at.  False where their numbers do not fit 32 bits.
static bool gather_large(const Matrix* list, size_t n, size_t* at, Args* a, size_t* bytes)
{
    uint64_t blocks = 0, pairs = 0, tiles = 0, matrices = 0;
    size_t off = 0;
    a->groups = 0;
    for (; *at < n && a->groups < kMaxLarge; ++*at) {
        if (choice_of(list[*at]).kind != kLarge) continue;
        Group g = group_for(list[*at], 0u);
        const uint64_t rows = g.mp / kTile;
        g.first_block = static_cast<uint32_t>(blocks); g.first_pair = static_cast<uint32_t>(pairs); g.first_tile = static_cast<uint32_t>(tiles);
        g.work = off;
        g.first_matrix = static_cast<uint32_t>(matrices);
        matrices += g.count;
        blocks += g.count * rows * (g.np / kPieceCols);
        pairs += g.count * (rows * (rows + 1u) / 2u);
        tiles += g.count * rows * ((g.np + kTile - 1u) / kTile);
        off += g.count * large_bytes(g.mp, g.np);
        if (blocks > 0x7FFFFFFFu || pairs > 0x7FFFFFFFu || tiles > 0x7FFFFFFFu) return false;
        a->g[a->groups++] = g;
    }
    a->blocks = static_cast<uint32_t>(blocks); a->pairs = static_cast<uint32_t>(pairs); a->tiles = static_cast<uint32_t>(tiles);
    a->partial_at = (off + 255u) / 256u * 256u;
    a->lift_at = a->partial_at + blocks * sizeof(double);
    *bytes = a->lift_at + matrices * sizeof(uint32_t);
    return true;
}

size_t workspace_bytes(const Matrix* list, size_t n)
{
    size_t most = 0, bytes = 0;
    Args a;
    for (size_t i = 0; i < n; ++i)
        if (static_cast<uint64_t>(choice_of(list[i]).blocks) * list[i].count > 0x7FFFFFFFu) return ~static_cast<size_t>(0);
    for (size_t at = 0; at < n;) {
        if (!gather_large(list, n, &at, &a, &bytes)) return ~static_cast<size_t>(0);
        most = std::max(most, bytes);
    }
    return most;
}

int launch(cudaStream_t st, uint32_t source, const Matrix* list, size_t n, const Args& base, char* work)
{
    int launches = 0;
    Args a = base;
    // the longest first: a launch for each kernel and size of cluster that the list needs
    for (int kind = kSmall; kind >= static_cast<int>(kTiny16); --kind)
        for (uint32_t cluster = kMostBlocks; cluster; cluster /= 2u)
            for (size_t at = 0; at < n;) {
                uint64_t blocks = 0;
                size_t smem = 0;
                uint32_t columns = 0;
                a.groups = 0;
                a.cluster = cluster;
                for (; at < n && a.groups < kMaxGroups; ++at) {
                    const Choice c = choice_of(list[at]);
                    if (static_cast<int>(c.kind) != kind || c.blocks != cluster) continue;
                    Group g = group_for(list[at], cluster);
                    g.first_block = static_cast<uint32_t>(blocks);
                    blocks += g.count;
                    if (blocks * cluster > 0x7FFFFFFFu) return -1;
                    smem = std::max(smem, small_bytes(g.mp, g.np, cluster));
                    columns = std::max(columns, g.np);
                    a.g[a.groups++] = g;
                }
                a.blocks = static_cast<uint32_t>(blocks);
                if (a.groups == 0u) continue;
                a.late = launches > 0;
                const int k = kind == kSmall ? launch_small(st, source, a, smem) : launch_tiny(st, source, a, kind + 1u, std::min(16u, columns / 16u));
                if (k < 0) return -1;
                launches += k;
            }
    for (size_t at = 0; at < n;) {
        size_t bytes = 0;
        if (!gather_large(list, n, &at, &a, &bytes)) return -1;
        if (a.groups == 0u) continue;
        a.work = work;
        a.partial = reinterpret_cast<double*>(work + a.partial_at);
        a.lift = reinterpret_cast<uint32_t*>(work + a.lift_at);
        const int k = launch_large(st, source, a);
        if (k < 0) return -1;
        launches += k;
    }
    return launches;
}

}  // namespace ns

// ---- Muon ----------------------------------------------------------------------------------------------------------------

// What lies between the matrices: Adam with the same decay.
constexpr uint32_t kMaxGaps = 64;
struct GapArgs {
    const float *c, *m, *v, *g;
    float *c_out, *m_out, *v_out;
    const double* skip;
    const uint32_t* d_step;
    uint32_t step, gaps, late;           // late: as in Args
    double beta1, beta2;
    float lr, keep, b1, b2, rest1, rest2, eps;      // (rest = 1 - beta)
    uint64_t start[kMaxGaps];
    uint64_t before[kMaxGaps + 1];       // elements of the gaps before this one
};

__device__ __forceinline__ void muon_rest(const GapArgs& a)
{
    if (a.skip && __ldcg(a.skip) == 0.0) return;
    const uint64_t at = static_cast<uint64_t>(blockIdx.x) * 256u + threadIdx.x;
    if (at >= a.before[a.gaps]) return;
    uint32_t lo = 0, hi = a.gaps - 1u;                          // the last gap that starts at or before `at`
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1u) / 2u;
        if (a.before[mid] <= at) lo = mid; else hi = mid - 1u;
    }
    const uint64_t d = a.start[lo] + (at - a.before[lo]);
    const double t = a.d_step ? __ldcg(a.d_step) : a.step;
    const float corr1 = static_cast<float>(1.0 / (1.0 - pow(a.beta1, t)));
    const float corr2 = static_cast<float>(1.0 / (1.0 - pow(a.beta2, t)));
    const float g = __ldcg(a.g + d), m = a.b1 * __ldcg(a.m + d) + a.rest1 * g, v = a.b2 * __ldcg(a.v + d) + a.rest2 * g * g;
    a.m_out[d] = m;
    a.v_out[d] = v;
    a.c_out[d] = a.keep * __ldcg(a.c + d) + a.lr * (m * corr1) / (sqrtf(v * corr2) + a.eps);
}

__global__ void __launch_bounds__(256) k_muon_rest(const __grid_constant__ GapArgs a)
{
    if (!a.late) dep_wait();
    dep_trigger();
    muon_rest(a);
    if (a.late) dep_wait();
}

static std::vector<ns::Matrix> muon_list(const evo_matrix* list, size_t n, double lr)
{
    std::vector<ns::Matrix> out(n);
    for (size_t i = 0; i < n; ++i) {
        const evo_matrix& x = list[i];
        out[i] = ns::Matrix{ x.offset, x.offset, 0, 0, x.rows, x.cols, x.cols, x.cols, 1u,
                             static_cast<float>(lr * 0.2 * std::sqrt(static_cast<double>(std::max(x.rows, x.cols)))) };
    }
    return out;
}

size_t muon_workspace_bytes(const evo_matrix* list, size_t n)
try {
    const std::vector<ns::Matrix> m = muon_list(list, n, 0.0);
    return ns::workspace_bytes(m.data(), m.size());
} catch (const std::bad_alloc&) {
    return ~static_cast<size_t>(0);
}

bool muon_scalars(const MuonArgs& a, ns::Scalars* s)
{
    std::memset(s, 0, sizeof(*s));
    s->a = a.a; s->b = a.b; s->c = a.c; s->eps = a.ns_eps; s->steps = a.ns_steps;
    s->mu = static_cast<float>(a.mu); s->rest = static_cast<float>(1.0 - a.mu); s->keep = static_cast<float>(1.0 - a.lr * a.decay); s->nesterov = a.nesterov;
    return ns::set_scales(s);
}

int launch_muon(cudaStream_t st, const evo_matrix* list, size_t n, const MuonArgs& a)
try {
    ns::Args args;
    std::memset(&args, 0, sizeof(args));
    if (!muon_scalars(a, &args.s)) return -1;
    args.in = a.g; args.out = a.center_out;
    args.m_in = a.m; args.m_out = a.m_out; args.v_in = a.v; args.v_out = a.v_out; args.c_in = a.center;
    args.skip = a.skip; args.sticky = a.sticky; args.wait_log2 = a.wait_log2; args.drop = a.drop;
    const std::vector<ns::Matrix> m = muon_list(list, n, a.lr);
    int launches = ns::launch(st, ns::kMuon, m.data(), n, args, a.work);
    if (launches < 0) return -1;
    GapArgs r;
    r.c = a.center; r.m = a.m; r.v = a.v; r.g = a.g; r.c_out = a.center_out; r.m_out = a.m_out; r.v_out = a.v_out;
    r.skip = a.skip; r.d_step = a.d_step; r.step = a.step;
    r.beta1 = a.beta1; r.beta2 = a.beta2; r.lr = static_cast<float>(a.lr); r.keep = args.s.keep;
    r.b1 = static_cast<float>(a.beta1); r.b2 = static_cast<float>(a.beta2); r.rest1 = static_cast<float>(1.0 - a.beta1);
    r.rest2 = static_cast<float>(1.0 - a.beta2); r.eps = static_cast<float>(a.adam_eps);
    uint64_t at = 0;
    for (size_t i = 0; i <= n;) {
        r.gaps = 0;
        r.before[0] = 0;
        for (; i <= n && r.gaps < kMaxGaps; ++i) {
            const uint64_t end = i < n ? list[i].offset : a.dim;
            if (end > at) {
                r.start[r.gaps] = at;
                r.before[r.gaps + 1u] = r.before[r.gaps] + (end - at);
                ++r.gaps;
            }
            if (i < n) at = list[i].offset + static_cast<uint64_t>(list[i].rows) * list[i].cols;
        }
        if (r.gaps == 0u) continue;
        const uint64_t blocks = (r.before[r.gaps] + 255u) / 256u;
        r.late = launches > 0;
        if (launch_dependent(k_muon_rest, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st, r) != cudaSuccess) return -1;
        ++launches;
    }
    return launches;
} catch (const std::bad_alloc&) {
    return -1;
}

uint32_t policy_matrices(const evo_config& c, evo_matrix (&out)[EVO_MAX_LAYERS])
{
    uint64_t at = 0;
    uint32_t n = 0;
    auto layer = [&](uint32_t rows, uint32_t cols, uint32_t bias) {
        out[n++] = evo_matrix{ at, rows, cols };
        at += static_cast<uint64_t>(rows) * cols + bias;
    };
    if (c.policy_kind == EVO_POLICY_MLP) {
        for (uint32_t l = 0; l < c.n_layers && l < EVO_MAX_LAYERS; ++l) layer(c.layer_sizes[l + 1], c.layer_sizes[l], c.layer_sizes[l + 1]);
    } else if (c.policy_kind == EVO_POLICY_CNN_28) {
        layer(8, 25, 8);
        layer(16, 200, 16);
        layer(10, 256, 10);
    } else if (c.policy_kind == EVO_POLICY_LSTM_SEQ2SEQ) {
        const uint32_t h = c.layer_sizes[0];
        for (int cell = 0; cell < 2; ++cell) {
            layer(4u * h, 12, 0);
            layer(4u * h, h, 4u * h);
        }
        layer(12, h, 12);
    }
    return n;
}

}  // namespace evo

using namespace evo;

static bool default_ns(const evo_newton_schulz* in, evo_newton_schulz* out)
{
    *out = evo_newton_schulz{ sizeof(evo_newton_schulz), 5u, kNsA, kNsB, kNsC, kNsEps };
    if (!in) return true;
    if (in->struct_size != sizeof(evo_newton_schulz)) return false;
    if (in->steps) out->steps = in->steps;
    if (in->a != 0.f || in->b != 0.f || in->c != 0.f) { out->a = in->a; out->b = in->b; out->c = in->c; }
    if (in->eps != 0.f) out->eps = in->eps;
    return out->steps <= 64u && out->eps >= 1e-30f && std::isfinite(out->eps);
}

static evo_status check_matrices(const evo_matrices* x)
{
    if (!x || x->type > EVO_F16 || x->batch < 1u || x->rows < 1u || x->cols < 1u) return EVO_ERR_INVALID_ARG;
    if (x->rows > (1u << 20) || x->cols > (1u << 20)) return EVO_ERR_INVALID_ARG;
    if (x->row_stride < x->cols && x->rows > 1u) return EVO_ERR_INVALID_ARG;
    if (x->row_stride > 0xFFFFFFFFull || x->batch_stride > (1ull << 40)) return EVO_ERR_INVALID_ARG;
    if (x->batch > 1u && x->batch_stride < (x->rows - 1u) * static_cast<uint64_t>(x->row_stride) + x->cols) return EVO_ERR_INVALID_ARG;
    if (!x->data || (reinterpret_cast<uintptr_t>(x->data) & (x->type == EVO_F32 ? 3u : 1u))) return EVO_ERR_INVALID_ARG;
    return EVO_OK;
}

extern "C" {

evo_status evo_orthogonalize_bytes(uint32_t batch, uint32_t rows, uint32_t cols, size_t* bytes)
{
    if (!bytes || batch < 1u || rows < 1u || cols < 1u || rows > (1u << 20) || cols > (1u << 20)) return EVO_ERR_INVALID_ARG;
    const ns::Matrix m{ 0, 0, 0, 0, rows, cols, cols, cols, batch, 0.f };
    const size_t need = ns::workspace_bytes(&m, 1);
    if (need == ~static_cast<size_t>(0)) return EVO_ERR_UNSUPPORTED;
    *bytes = need;
    return EVO_OK;
}

evo_status evo_orthogonalize(const evo_newton_schulz* ns_in, const evo_matrices* x, const evo_matrices* out, void* d_workspace,
                             size_t workspace_bytes, void* cuda_stream)
{
    evo_newton_schulz p;
    if (!default_ns(ns_in, &p)) return EVO_ERR_INVALID_ARG;
    evo_status st = check_matrices(x);
    if (st == EVO_OK) st = check_matrices(out);
    if (st != EVO_OK) return st;
    if (out->type != x->type || out->batch != x->batch || out->rows != x->rows || out->cols != x->cols) return EVO_ERR_INVALID_ARG;
    const size_t width = x->type == EVO_F32 ? 4u : 2u;
    uint64_t one, x_bytes, out_bytes;
    if (!extent(x->rows, x->row_stride, x->cols, 1u, &one) || !extent(x->batch, x->batch_stride, one, width, &x_bytes) ||
        !extent(out->rows, out->row_stride, out->cols, 1u, &one) || !extent(out->batch, out->batch_stride, one, width, &out_bytes))
        return EVO_ERR_INVALID_ARG;
    const bool same = x->data == out->data && (x->rows == 1u || x->row_stride == out->row_stride) && (x->batch == 1u || x->batch_stride == out->batch_stride);
    if (!same && overlap(x->data, x_bytes, out->data, out_bytes)) return EVO_ERR_INVALID_ARG;
    ns::Args a;
    std::memset(&a, 0, sizeof(a));
    a.s.a = p.a; a.s.b = p.b; a.s.c = p.c; a.s.eps = p.eps; a.s.steps = p.steps;
    if (!ns::set_scales(&a.s)) return EVO_ERR_UNSUPPORTED;
    size_t need = 0;
    st = evo_orthogonalize_bytes(x->batch, x->rows, x->cols, &need);
    if (st != EVO_OK) return st;
    if (need && (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255u))) return EVO_ERR_INVALID_ARG;
    if (workspace_bytes < need) return EVO_ERR_WORKSPACE;
    a.in = x->data; a.out = out->data; a.wait_log2 = 31u;
    const ns::Matrix m{ 0, 0, x->batch_stride, out->batch_stride, x->rows, x->cols, static_cast<uint32_t>(x->row_stride),
                        static_cast<uint32_t>(out->row_stride), x->batch, 0.f };
    return ns::launch(static_cast<cudaStream_t>(cuda_stream), x->type, &m, 1, a, static_cast<char*>(d_workspace)) < 0 ? EVO_ERR_CUDA : EVO_OK;
}

static evo_status check_list(const evo_matrix* list, uint32_t n, uint64_t dim)
{
    if (n && !list) return EVO_ERR_INVALID_ARG;
    uint64_t at = 0;
    for (uint32_t i = 0; i < n; ++i) {
        const evo_matrix& x = list[i];
        if (x.rows < 1u || x.cols < 1u || x.rows > (1u << 20) || x.cols > (1u << 20) || x.offset < at) return EVO_ERR_INVALID_ARG;
        const uint64_t size = static_cast<uint64_t>(x.rows) * x.cols;
        if (x.offset > dim || size > dim - x.offset) return EVO_ERR_INVALID_ARG;
        at = x.offset + size;
    }
    return EVO_OK;
}

evo_status evo_muon_bytes(const evo_matrix* list, uint32_t n, uint64_t param_dim, size_t* bytes)
{
    if (!bytes) return EVO_ERR_INVALID_ARG;
    const evo_status st = check_list(list, n, param_dim);
    if (st != EVO_OK) return st;
    const size_t need = muon_workspace_bytes(list, n);
    if (need == ~static_cast<size_t>(0)) return EVO_ERR_UNSUPPORTED;
    *bytes = need;
    return EVO_OK;
}

evo_status evo_muon_step(const evo_muon* cfg, const evo_matrix* list, uint32_t n, uint64_t param_dim, uint32_t step,
                         const float* d_center, const float* d_m, const float* d_v, const float* d_gradient,
                         float* d_center_out, float* d_m_out, float* d_v_out, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    if (!cfg || cfg->struct_size != sizeof(evo_muon) || step < 1u || param_dim < 1u || param_dim > (1ull << 38)) return EVO_ERR_INVALID_ARG;
    const void* ptrs[7] = { d_center, d_m, d_v, d_gradient, d_center_out, d_m_out, d_v_out };
    for (const void* p : ptrs)
        if (!p || (reinterpret_cast<uintptr_t>(p) & 3u)) return EVO_ERR_INVALID_ARG;
    // an output may be its own input; otherwise the outputs are apart from everything else
    for (int i = 4; i < 7; ++i)
        for (int j = 0; j < i; ++j) {
            const uintptr_t p = reinterpret_cast<uintptr_t>(ptrs[i]), q = reinterpret_cast<uintptr_t>(ptrs[j]);
            if (!(j == i - 4 && p == q) && p < q + 4u * param_dim && q < p + 4u * param_dim) return EVO_ERR_INVALID_ARG;
        }
    MuonArgs a;
    std::memset(&a, 0, sizeof(a));
    a.lr = cfg->lr; a.mu = cfg->momentum; a.decay = cfg->weight_decay; a.nesterov = cfg->plain_momentum ? 0u : 1u;
    a.beta1 = cfg->beta1 == 0.0 ? 0.9 : cfg->beta1;
    a.beta2 = cfg->beta2 == 0.0 ? 0.999 : cfg->beta2;
    a.adam_eps = cfg->adam_eps == 0.0 ? 1e-8 : cfg->adam_eps;
    if (!std::isfinite(a.lr) || !(a.mu >= 0.0 && a.mu < 1.0) || !(a.decay >= 0.0) || !std::isfinite(a.decay) || !(a.beta1 >= 0.0 && a.beta1 < 1.0) ||
        !(a.beta2 >= 0.0 && a.beta2 < 1.0) || !(a.adam_eps >= 0.0) || !std::isfinite(a.adam_eps))
        return EVO_ERR_INVALID_ARG;
    evo_newton_schulz p;
    if (!default_ns(&cfg->newton_schulz, &p)) return EVO_ERR_INVALID_ARG;
    a.a = p.a; a.b = p.b; a.c = p.c; a.ns_eps = p.eps; a.ns_steps = p.steps;
    ns::Scalars unused;
    if (!muon_scalars(a, &unused)) return EVO_ERR_UNSUPPORTED;
    size_t need = 0;
    const evo_status st = evo_muon_bytes(list, n, param_dim, &need);
    if (st != EVO_OK) return st;
    if (need && (!d_workspace || (reinterpret_cast<uintptr_t>(d_workspace) & 255u))) return EVO_ERR_INVALID_ARG;
    if (workspace_bytes < need) return EVO_ERR_WORKSPACE;
    a.center = d_center; a.m = d_m; a.v = d_v; a.g = d_gradient; a.center_out = d_center_out; a.m_out = d_m_out; a.v_out = d_v_out;
    a.dim = param_dim; a.step = step; a.work = static_cast<char*>(d_workspace); a.wait_log2 = 31u;
    return launch_muon(static_cast<cudaStream_t>(cuda_stream), list, n, a) < 0 ? EVO_ERR_CUDA : EVO_OK;
}

}  // extern "C"

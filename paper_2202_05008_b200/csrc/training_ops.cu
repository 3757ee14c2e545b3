// C entry points of what a mixture of members is trained with: routes, rows in sorted order and back, the gradients of the grouped products, the policy loss.
#include <cmath>
#include <cstring>

#include "grouped_gradient.h"
#include "policy_loss.h"
#include "routing.h"

using namespace evo;

namespace {

constexpr uint64_t kMost = 1ull << 40;       // elements of a pitch or a stride, and rows
constexpr uint32_t kMostWidth = 1u << 20;

bool misaligned(const void* p, uint64_t size) { return (reinterpret_cast<uintptr_t>(p) & (size - 1u)) != 0u; }
uint64_t size_of(uint32_t type) { return type == EVO_F32 ? 4u : 2u; }
evo_status status_of(int launches) { return launches == -2 ? EVO_ERR_UNSUPPORTED : launches < 0 ? EVO_ERR_CUDA : EVO_OK; }

// An array of a call: where it lies, and its bytes from the first to the last element.
struct Span { const void* p; uint64_t bytes; };
bool apart(const Span& a, const Span& b) { return !a.p || !b.p || !a.bytes || !b.bytes || !overlap(a.p, a.bytes, b.p, b.bytes); }
template <size_t N, size_t M>
bool apart(const Span (&outputs)[N], const Span (&inputs)[M])
{
    for (size_t i = 0; i < N; ++i) {
        for (size_t k = 0; k < M; ++k)
            if (!apart(outputs[i], inputs[k])) return false;
        for (size_t k = 0; k < i; ++k)
            if (!apart(outputs[i], outputs[k])) return false;
    }
    return true;
}
evo_status check_workspace(size_t need, const void* p, size_t bytes)
{
    if (need && (!p || misaligned(p, 256u))) return EVO_ERR_INVALID_ARG;
    return bytes < need ? EVO_ERR_WORKSPACE : EVO_OK;
}

// ---- routes ----
bool route_args(const evo_routes* p, RouteArgs* a)
{
    if (!p || p->struct_size != sizeof(evo_routes) || p->members_64 > 1u || p->groups < 1u || p->groups > kMostWidth || p->choices < 1u) return false;
    if (p->rows > kMost || (p->rows && p->choices > 0x7FFFFFFFull / p->rows) || p->ld_members > kMost || (p->rows > 1u && p->ld_members < p->choices)) return false;
    std::memset(a, 0, sizeof(*a));
    a->members = p->d_members; a->ld = p->rows > 1u ? p->ld_members : p->choices; a->wide = p->members_64;
    a->choices = p->choices; a->groups = p->groups; a->pairs = static_cast<uint32_t>(p->rows * p->choices);
    a->offsets = p->d_offsets; a->source = p->d_source; a->place = p->d_place;
    return true;
}

// ---- rows ----
enum { kTake, kCombine, kBackward };
evo_status row_set_args(const evo_row_sets* p, int what, RowSetArgs* a)
{
    if (!p || p->struct_size != sizeof(evo_row_sets) || p->type > EVO_F16 || p->choices < 1u || p->choices > kMostWidth || p->cols < 1u || p->cols > kMostWidth)
        return EVO_ERR_INVALID_ARG;
    if (p->rows > kMost || p->sorted_rows >= (1ull << 31)) return EVO_ERR_INVALID_ARG;
    const uint64_t size = size_of(p->type);
    const bool back = what == kBackward, many = p->rows > 1u, many_sorted = p->sorted_rows > 1u;
    // (a pitch that is never taken may be anything)
    const uint64_t ld_place = many ? p->ld_place : p->choices, ld_weights = many ? p->ld_weights : p->choices, ld_rows = many ? p->ld_rows : p->cols;
    const uint64_t ld_sorted = many_sorted ? p->ld_sorted : p->cols, ld_gradient = many_sorted ? p->ld_sorted_gradient : p->cols;
    const uint64_t ld_dw = many ? p->ld_weights_gradient : p->choices;
    if (ld_place < p->choices || (p->d_weights && ld_weights < p->choices) || ld_rows < p->cols || ld_sorted < p->cols) return EVO_ERR_INVALID_ARG;
    if (back && (ld_gradient < p->cols || ld_dw < p->choices)) return EVO_ERR_INVALID_ARG;
    if (ld_place > kMost || ld_weights > kMost || ld_rows > kMost || ld_sorted > kMost || (back && (ld_gradient > kMost || ld_dw > kMost))) return EVO_ERR_INVALID_ARG;
    std::memset(a, 0, sizeof(*a));
    a->place = p->d_place; a->weights = p->d_weights; a->rows = p->d_rows; a->sorted = p->d_sorted;
    a->count = p->rows; a->ld_place = ld_place; a->ld_weights = ld_weights; a->ld_rows = ld_rows; a->ld_sorted = ld_sorted;
    a->sorted_rows = static_cast<uint32_t>(p->sorted_rows); a->choices = p->choices; a->cols = p->cols;
    Span place = { p->d_place, 0 }, weights = { p->d_weights, 0 }, rows = { p->d_rows, 0 }, sorted = { p->d_sorted, 0 }, gradient = { nullptr, 0 }, dw = { nullptr, 0 };
    if (!extent(p->rows, ld_place, p->choices, 4u, &place.bytes) || !extent(p->rows, ld_weights, p->choices, 4u, &weights.bytes) ||
        !extent(p->rows, ld_rows, p->cols, size, &rows.bytes) || !extent(p->sorted_rows, ld_sorted, p->cols, size, &sorted.bytes))
        return EVO_ERR_INVALID_ARG;
    if (back) {
        a->d_sorted = p->d_sorted_gradient; a->ld_d_sorted = ld_gradient; a->d_weights = p->d_weights_gradient; a->ld_d_weights = ld_dw;
        gradient.p = p->d_sorted_gradient; dw.p = p->d_weights_gradient;
        if (!extent(p->sorted_rows, ld_gradient, p->cols, size, &gradient.bytes) || !extent(p->rows, ld_dw, p->choices, 4u, &dw.bytes)) return EVO_ERR_INVALID_ARG;
    }
    if (p->rows == 0u) return EVO_OK;
    if (!p->d_place || !p->d_rows || (!p->d_sorted && p->sorted_rows) || (back && (!p->d_weights || !p->d_weights_gradient || (!p->d_sorted_gradient && p->sorted_rows))))
        return EVO_ERR_INVALID_ARG;
    if (misaligned(p->d_place, 4u) || misaligned(p->d_weights, 4u) || misaligned(p->d_rows, size) || misaligned(p->d_sorted, size) ||
        (back && (misaligned(p->d_sorted_gradient, size) || misaligned(p->d_weights_gradient, 4u))))
        return EVO_ERR_INVALID_ARG;
    bool fine;
    if (what == kTake) { const Span out[] = { sorted }, in[] = { place, weights, rows }; fine = apart(out, in); }
    else if (what == kCombine) { const Span out[] = { rows }, in[] = { place, weights, sorted }; fine = apart(out, in); }
    else { const Span out[] = { gradient, dw }, in[] = { place, weights, rows, sorted }; fine = apart(out, in); }
    return fine ? EVO_OK : EVO_ERR_INVALID_ARG;
}

// ---- gradients of the grouped products ----
bool gradient_args(const evo_grouped* f, const evo_grouped_gradient* p, GradientArgs* a)
{
    if (!f || f->struct_size != sizeof(evo_grouped) || f->type > EVO_F16 || f->activation > EVO_ACT_RELU || f->offsets_64 > 1u) return false;
    if (f->groups < 1u || f->groups > 0x7FFFFFFFu || f->n_in < 1u || f->n_out < 1u || f->n_in > kMostWidth || f->n_out > kMostWidth || f->rows > kMost) return false;
    if (!p || p->struct_size != sizeof(evo_grouped_gradient) || p->sum_weight > 1u || p->sum_bias > 1u || !std::isfinite(f->scale)) return false;
    const bool act = f->activation != EVO_ACT_NONE;
    if (act && (f->scale == 0.f || !std::isfinite(1.f / f->scale))) return false;
    std::memset(a, 0, sizeof(*a));
    GroupedArgs& g = a->f;
    const bool many = f->rows > 1u, many_out = f->n_out > 1u, many_groups = f->groups > 1u;
    g.x = p->d_dweight ? f->d_x : nullptr; g.w = p->d_dx ? f->d_weight : nullptr; g.y = act ? f->d_y : nullptr; g.offsets = f->d_offsets;
    g.wide_offsets = f->offsets_64;
    g.groups = f->groups; g.n_in = f->n_in; g.n_out = f->n_out; g.activation = f->activation; g.scale = f->scale; g.rows = f->rows;
    // (a pitch that is never taken may be anything)
    g.ld_x = many ? f->ld_x : f->n_in; g.ld_y = many ? f->ld_y : f->n_out; g.ld_w = many_out ? f->ld_weight : f->n_in; g.stride_w = many_groups ? f->weight_stride : 0u;
    a->dy = p->d_dy; a->dx = p->d_dx; a->dw = p->d_dweight; a->db = p->d_dbias;
    a->ld_dy = many ? p->ld_dy : f->n_out; a->ld_dx = many ? p->ld_dx : f->n_in; a->ld_dw = many_out ? p->ld_dweight : f->n_in;
    a->stride_dw = many_groups ? p->dweight_stride : 0u; a->stride_db = many_groups ? p->dbias_stride : 0u;
    a->sum_w = p->sum_weight || !many_groups; a->sum_b = p->sum_bias || !many_groups;
    a->inverse = act ? 1.f / f->scale : 0.f;
    if (g.ld_x > kMost || g.ld_y > kMost || g.ld_w > kMost || g.stride_w > kMost || a->ld_dy > kMost || a->ld_dx > kMost || a->ld_dw > kMost || a->stride_dw > kMost || a->stride_db > kMost)
        return false;
    if (a->ld_dy < f->n_out || (act && g.ld_y < f->n_out) || (a->dw && (g.ld_x < f->n_in || a->ld_dw < f->n_in)) || (a->dx && (g.ld_w < f->n_in || a->ld_dx < f->n_in))) return false;
    return true;
}

// Gradients of weights and biases that lie between each other's groups, as in rows like theta's: neither reaches into the other.
bool interleaved(const GradientArgs& a, uint64_t size, uint64_t set_w, uint64_t w_sets, uint64_t b_sets, const Span& w, const Span& b)
{
    if (apart(w, b)) return true;
    const uint64_t period = a.stride_dw * size, set_b = static_cast<uint64_t>(a.f.n_out) * size;
    if (w_sets < 2u || b_sets < 2u || a.stride_dw != a.stride_db || period < set_w + set_b) return false;
    const int64_t distance = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(w.p));
    const int64_t q = static_cast<int64_t>(period), inside = (distance % q + q) % q;
    return static_cast<uint64_t>(inside) >= set_w && static_cast<uint64_t>(inside) + set_b <= period;
}

}  // namespace

extern "C" {

evo_status evo_route_rows_bytes(const evo_routes* p, size_t* bytes)
{
    RouteArgs a;
    if (!bytes || !route_args(p, &a)) return EVO_ERR_INVALID_ARG;
    *bytes = route_bytes(a);
    return EVO_OK;
}

evo_status evo_route_rows(const evo_routes* p, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    RouteArgs a;
    if (!route_args(p, &a) || !a.offsets || misaligned(a.offsets, 4u)) return EVO_ERR_INVALID_ARG;
    const uint64_t member = a.wide ? 8u : 4u;
    if (a.pairs && (!a.members || !a.place || misaligned(a.members, member) || misaligned(a.place, 4u) || misaligned(a.source, 4u))) return EVO_ERR_INVALID_ARG;
    Span in[] = { { a.members, 0 } };
    const Span out[] = { { a.offsets, 4u * (a.groups + 1ull) }, { a.source, 4ull * a.pairs }, { a.place, 4ull * a.pairs } };
    if (!extent(p->rows, a.ld, a.choices, member, &in[0].bytes) || !apart(out, in)) return EVO_ERR_INVALID_ARG;
    const evo_status st = check_workspace(route_bytes(a), d_workspace, workspace_bytes);
    return st != EVO_OK ? st : status_of(launch_route(static_cast<cudaStream_t>(cuda_stream), a, d_workspace));
}

evo_status evo_take_rows(const evo_row_sets* p, void* cuda_stream)
{
    RowSetArgs a;
    const evo_status st = row_set_args(p, kTake, &a);
    return st != EVO_OK || a.count == 0u || a.sorted_rows == 0u ? st : status_of(launch_take(static_cast<cudaStream_t>(cuda_stream), p->type, a));
}
evo_status evo_combine_rows(const evo_row_sets* p, void* cuda_stream)
{
    RowSetArgs a;
    const evo_status st = row_set_args(p, kCombine, &a);
    return st != EVO_OK || a.count == 0u ? st : status_of(launch_combine(static_cast<cudaStream_t>(cuda_stream), p->type, a));
}
evo_status evo_combine_rows_backward(const evo_row_sets* p, void* cuda_stream)
{
    RowSetArgs a;
    const evo_status st = row_set_args(p, kBackward, &a);
    return st != EVO_OK || a.count == 0u ? st : status_of(launch_combine_backward(static_cast<cudaStream_t>(cuda_stream), p->type, a));
}

evo_status evo_grouped_linear_backward_bytes(const evo_grouped* forward, const evo_grouped_gradient* p, size_t* bytes)
{
    GradientArgs a;
    if (!bytes || !gradient_args(forward, p, &a)) return EVO_ERR_INVALID_ARG;
    // (before the buffers exist: as much as they need wherever they lie)
    const bool known = a.dy && (!a.dw || a.f.x) && (!a.dx || a.f.w);
    *bytes = grouped_gradient_bytes(forward->type, a, !known);
    return EVO_OK;
}

evo_status evo_grouped_linear_backward(const evo_grouped* forward, const evo_grouped_gradient* p, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    GradientArgs a;
    if (!gradient_args(forward, p, &a)) return EVO_ERR_INVALID_ARG;
    if (!a.dx && !a.dw && !a.db) return EVO_OK;
    const GroupedArgs& g = a.f;
    const uint64_t size = size_of(forward->type), offset = g.wide_offsets ? 8u : 4u;
    if (!g.offsets || misaligned(g.offsets, offset)) return EVO_ERR_INVALID_ARG;
    if (g.rows && (!a.dy || (g.activation != EVO_ACT_NONE && !g.y) || (a.dw && !g.x) || (a.dx && !g.w))) return EVO_ERR_INVALID_ARG;
    const void* const arrays[] = { a.dy, g.y, g.x, g.w, a.dx, a.dw, a.db };
    for (const void* q : arrays)
        if (misaligned(q, size)) return EVO_ERR_INVALID_ARG;
    const uint64_t w_sets = a.sum_w ? 1u : g.groups, b_sets = a.sum_b ? 1u : g.groups;
    Span dy = { a.dy, 0 }, y = { g.y, 0 }, x = { g.x, 0 }, w = { g.w, 0 }, offsets = { g.offsets, (g.groups + 1ull) * offset }, dx = { a.dx, 0 }, dw = { a.dw, 0 }, db = { a.db, 0 };
    uint64_t set, set_dw = 0;
    if (!extent(g.rows, a.ld_dy, g.n_out, size, &dy.bytes) || (g.y && !extent(g.rows, g.ld_y, g.n_out, size, &y.bytes)) || (g.x && !extent(g.rows, g.ld_x, g.n_in, size, &x.bytes)) ||
        (g.w && (!extent(g.n_out, g.ld_w, g.n_in, 1u, &set) || !extent(g.groups, g.stride_w, set, size, &w.bytes))) || (a.dx && !extent(g.rows, a.ld_dx, g.n_in, size, &dx.bytes)) ||
        (a.dw && (!extent(g.n_out, a.ld_dw, g.n_in, 1u, &set_dw) || !extent(w_sets, a.stride_dw, set_dw, size, &dw.bytes))) ||
        (a.db && !extent(b_sets, a.stride_db, g.n_out, size, &db.bytes)))
        return EVO_ERR_INVALID_ARG;
    // (gradients of the groups lie one behind the other)
    if ((a.dw && w_sets > 1u && a.stride_dw < set_dw) || (a.db && b_sets > 1u && a.stride_db < g.n_out)) return EVO_ERR_INVALID_ARG;
    const Span in[] = { dy, y, x, w, offsets }, rows[] = { dx }, weights[] = { dw }, biases[] = { db }, out[] = { dw, db };
    if (!apart(rows, in) || !apart(weights, in) || !apart(biases, in) || !apart(rows, out) || !interleaved(a, size, set_dw * size, w_sets, b_sets, dw, db)) return EVO_ERR_INVALID_ARG;
    const evo_status st = check_workspace(grouped_gradient_bytes(forward->type, a, false), d_workspace, workspace_bytes);
    return st != EVO_OK ? st : status_of(launch_grouped_gradient(static_cast<cudaStream_t>(cuda_stream), forward->type, a, d_workspace));
}

evo_status evo_policy_loss_bytes(const evo_policy_rows* p, size_t* bytes)
{
    if (!p || !bytes || p->struct_size != sizeof(evo_policy_rows) || p->rows > kMost) return EVO_ERR_INVALID_ARG;
    *bytes = p->d_loss ? policy_loss_bytes(p->rows) : 0u;
    return EVO_OK;
}

evo_status evo_policy_loss(const evo_policy_rows* p, void* d_workspace, size_t workspace_bytes, void* cuda_stream)
{
    size_t need = 0;
    if (evo_policy_loss_bytes(p, &need) != EVO_OK || p->type > EVO_F16 || p->actions_64 > 1u || p->actions < 1u || p->actions > kMostWidth) return EVO_ERR_INVALID_ARG;
    if (!(p->clip_low >= 0.0 && p->clip_low <= 1.0 && p->clip_high >= 0.0 && p->kl >= 0.0) || !std::isfinite(p->clip_high) || !std::isfinite(p->kl) ||
        (!p->d_ref_logp && p->kl != 0.0))
        return EVO_ERR_INVALID_ARG;
    const uint64_t size = size_of(p->type), number = p->actions_64 ? 8u : 4u, ld = p->rows > 1u ? p->ld_logits : p->actions, ld_gradient = p->rows > 1u ? p->ld_gradient : p->actions;
    if (ld > kMost || ld < p->actions || (p->d_gradient && (ld_gradient > kMost || ld_gradient < p->actions))) return EVO_ERR_INVALID_ARG;
    if (p->rows && (!p->d_logits || !p->d_action || !p->d_old_logp || !p->d_advantage)) return EVO_ERR_INVALID_ARG;
    if (misaligned(p->d_logits, size) || misaligned(p->d_gradient, size) || misaligned(p->d_action, number) || misaligned(p->d_old_logp, 4u) || misaligned(p->d_advantage, 4u) ||
        misaligned(p->d_ref_logp, 4u) || misaligned(p->d_weights, 4u) || misaligned(p->d_loss, 4u) || misaligned(p->d_logp, 4u))
        return EVO_ERR_INVALID_ARG;
    Span logits = { p->d_logits, 0 }, gradient = { p->d_gradient, 0 };
    if (!extent(p->rows, ld, p->actions, size, &logits.bytes) || (p->d_gradient && !extent(p->rows, ld_gradient, p->actions, size, &gradient.bytes))) return EVO_ERR_INVALID_ARG;
    const uint64_t each = 4u * p->rows;
    const Span action = { p->d_action, number * p->rows }, old = { p->d_old_logp, each }, advantage = { p->d_advantage, each }, ref = { p->d_ref_logp, each },
               weights = { p->d_weights, each }, loss = { p->d_loss, 4u }, logp = { p->d_logp, each };
    const bool in_place = p->d_gradient == p->d_logits && ld == ld_gradient;
    const Span out[] = { loss, logp, gradient }, in[] = { action, old, advantage, ref, weights }, results[] = { loss, logp };
    const Span scores[] = { logits };
    if (!apart(out, in) || !apart(results, scores) || (!in_place && !apart(gradient, logits))) return EVO_ERR_INVALID_ARG;
    const evo_status st = check_workspace(need, d_workspace, workspace_bytes);
    if (st != EVO_OK) return st;
    PolicyArgs a;
    std::memset(&a, 0, sizeof(a));
    a.logits = p->d_logits; a.gradient = p->d_gradient; a.action = p->d_action; a.old_logp = p->d_old_logp; a.advantage = p->d_advantage; a.ref_logp = p->kl > 0.0 ? p->d_ref_logp : nullptr;
    a.weights = p->d_weights; a.logp = p->d_logp; a.loss = p->d_loss; a.row_loss = need ? static_cast<double*>(d_workspace) : nullptr;
    a.rows = p->rows; a.ld = ld; a.ld_gradient = ld_gradient; a.n = p->actions; a.wide = p->actions_64;
    a.clip_low = p->clip_low; a.clip_high = p->clip_high; a.kl = p->kl; a.even = p->rows ? 1.0 / static_cast<double>(p->rows) : 0.0;
    a.log_low = std::log1p(-p->clip_low); a.log_high = std::log1p(p->clip_high);      // (minus infinity for clip_low 1)
    if (!a.loss && !a.logp && !a.gradient) return EVO_OK;
    return status_of(launch_policy_loss(static_cast<cudaStream_t>(cuda_stream), p->type, a));
}

}  // extern "C"

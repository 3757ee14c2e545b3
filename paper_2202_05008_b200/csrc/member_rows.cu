// fp32 rows through the layers of the member that they belong to: an MLP policy's get_actions in one launch.
//
// A population's weights are read once, so their way from memory is the bound.  A warp takes a member (and 8 of its rows, or 16) through
// all layers by itself, without a barrier: weight rows go from memory straight into the operand registers of mma.sync (grouped_mma.cuh: pairs of tf32
// numbers), 16 outputs by 64 of the contracted index at a time, and the next such piece, be it of the next layer, is on its way while one is
// multiplied.  Activations stay in the warp's part of shared memory.  Where there are too few items to go round, eight warps share one and take the
// sixteens of outputs in turn.  4,096 members of 28-128-128-8 with 4 rows each: 140 us, 2.5 TB/s, 13,000 warp instructions a member, issued in 46 % of the
// cycles.  (A block of eight warps for a member took 20,000: its weights copied to shared memory ahead 162 us, loaded into registers before
// the barrier 136.)
#include <algorithm>

#include "grouped_mma.cuh"
#include "member_rows.h"

namespace evo {
namespace {

constexpr uint32_t kTeam = 8;                    // warps of an item that is shared
constexpr uint32_t kAlone = 4;                   // warps of a block that have an item each

// Eight or four numbers of the next piece: [step][row g, row g + 8]
struct Piece { float4 w[4][2]; };

// Where a warp stands: sixteen of outputs of a layer, and the first of up to four sixteens of the contracted index
struct Cursor {
    uint32_t layer, tile, tiles, step, steps;
    const float *w0, *w1;                        // this lane's two weight rows
};

template <uint32_t NT, uint32_t TEAM>
__global__ void __launch_bounds__(32 * (TEAM == 1u ? kAlone : TEAM), TEAM == 1u ? (NT == 1u ? 4 : 3) : (NT == 1u ? 2 : 1)) k_member_rows(const __grid_constant__ MemberArgs a)
{
    extern __shared__ __align__(16) float smem[];
    constexpr uint32_t kPass = 8u * NT;
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, g = lane >> 2, q = lane & 3u;
    const uint32_t rank = TEAM == 1u ? 0u : warp, team = TEAM == 1u ? blockIdx.x * kAlone + warp : blockIdx.x, teams = TEAM == 1u ? gridDim.x * kAlone : gridDim.x;
    float* const acts = smem + (TEAM == 1u ? warp * (a.n_layers == 1u ? 1u : 2u) * kPass * a.ld : 0u);      // two of [kPass][ld] (one layer: one)
    auto meet = [] { if constexpr (TEAM == 1u) __syncwarp(); else __syncthreads(); };
    dep_wait();
    dep_trigger();

    const uint32_t items = a.g.groups * a.chunks;
    for (uint32_t item = team; item < items; item += teams) {
        const uint32_t member = a.chunks == 1u ? item : item / a.chunks, chunk = a.chunks == 1u ? 0u : item - member * a.chunks;
        uint64_t row, end;
        group_rows(a.g, member, &row, &end);
        const float* const w = a.theta + member * a.stride;
        // (an item of one layer may have a part of its outputs)
        const uint32_t all = (a.sizes[1] + 15u) / 16u, per = a.chunks == 1u ? all : (all + a.chunks - 1u) / a.chunks;
        const uint32_t tile0 = min(chunk * per, all), tile1 = min(tile0 + per, all);
        auto rows_of = [&](Cursor& c) {                                     // what is beyond the last output is read as the last one, and not used
            const uint32_t o = c.tile * 16u + g, top = a.sizes[c.layer + 1u] - 1u;
            const float* const base = w + a.w_at[c.layer];
            c.w0 = base + static_cast<uint64_t>(min(o, top)) * a.sizes[c.layer] + 4u * q;
            c.w1 = base + static_cast<uint64_t>(min(o + 8u, top)) * a.sizes[c.layer] + 4u * q;
        };
        auto start = [&](Cursor& c, uint32_t layer) {                       // first tile of this warp in a layer, or in a later one where it has none
            for (c.layer = layer; c.layer < a.n_layers; ++c.layer) {
                const bool only = a.n_layers == 1u;
                c.tile = (only ? tile0 : 0u) + rank;
                c.tiles = only ? tile1 : (a.sizes[c.layer + 1u] + 15u) / 16u;
                c.step = 0u;
                c.steps = (a.sizes[c.layer] + 15u) / 16u;
                if (c.tile < c.tiles) { rows_of(c); return; }
            }
        };
        auto advance = [&](Cursor& c) {
            c.step += 4u;
            if (c.step < c.steps) return;
            c.step = 0u;
            c.tile += TEAM;
            if (c.tile < c.tiles) rows_of(c);
            else start(c, c.layer + 1u);
        };
        auto load = [&](const Cursor& c, Piece& p) {
            if (c.layer >= a.n_layers) return;
            const uint32_t n_in = a.sizes[c.layer];
            if (a.aligned >> c.layer & 1u) {
#pragma unroll
                for (uint32_t s = 0; s < 4u; ++s) {
                    const uint32_t k = 16u * (c.step + s);
                    const bool in = k + 4u * q < n_in;                      // (n_in is a multiple of 4)
                    p.w[s][0] = in ? __ldcs(reinterpret_cast<const float4*>(c.w0 + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
                    p.w[s][1] = in ? __ldcs(reinterpret_cast<const float4*>(c.w1 + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
                }
            } else {
#pragma unroll
                for (uint32_t s = 0; s < 4u; ++s) {
                    const uint32_t k = 16u * (c.step + s), kk = k + 4u * q;
                    p.w[s][0] = make_float4(kk < n_in ? c.w0[k] : 0.f, kk + 1u < n_in ? c.w0[k + 1u] : 0.f, kk + 2u < n_in ? c.w0[k + 2u] : 0.f, kk + 3u < n_in ? c.w0[k + 3u] : 0.f);
                    p.w[s][1] = make_float4(kk < n_in ? c.w1[k] : 0.f, kk + 1u < n_in ? c.w1[k + 1u] : 0.f, kk + 2u < n_in ? c.w1[k + 2u] : 0.f, kk + 3u < n_in ? c.w1[k + 3u] : 0.f);
                }
            }
        };
        // several items' passes over a member's rows go to several teams
        const uint32_t share = blockIdx.y, shares = gridDim.y;
        for (row += share * kPass; row < end; row += shares * kPass) {
            const uint32_t rows = static_cast<uint32_t>(min(static_cast<uint64_t>(kPass), end - row));
            Cursor next;
            Piece ahead;
            start(next, 0u);
            load(next, ahead);
            // observations: zeros behind the last row and up to 16 of the contracted index
            {
                const uint32_t in0 = a.sizes[0], pad0 = (in0 + 15u) / 16u * 16u;
                const float* const x = static_cast<const float*>(a.g.x) + row * a.g.ld_x;
                for (uint32_t r = rank; r < kPass; r += TEAM)
                    for (uint32_t k = lane; k < pad0; k += 32u) acts[r * a.ld + k] = r < rows && k < in0 ? x[r * a.g.ld_x + k] : 0.f;
            }
            meet();
            float large[NT][4], small[NT][4], less[NT][4], sum[NT][4];      // hi hi', hi lo', lo hi'; hi hi' of earlier pieces
            for (uint32_t layer = 0; layer < a.n_layers; ++layer) {
                const float* const x = acts + (layer & 1u) * kPass * a.ld + g * a.ld + 4u * q;
                float* const y = acts + (layer + 1u & 1u) * kPass * a.ld;
                const bool last_layer = layer + 1u == a.n_layers;
                while (next.layer == layer) {
                    const Cursor now = next;
                    const Piece p = ahead;
                    advance(next);
                    load(next, ahead);
                    if (now.step == 0u)
#pragma unroll
                        for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                            for (int i = 0; i < 4; ++i) sum[c][i] = small[c][i] = less[c][i] = 0.f;
#pragma unroll
                    for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) large[c][i] = 0.f;
#pragma unroll
                    for (uint32_t s = 0; s < 4u; ++s) {
                        if (now.step + s >= now.steps) break;
                        const float4 u = p.w[s][0], v = p.w[s][1];
                        uint32_t hi[2][4], lo[2][4];
                        gm::split(u.x, hi[0][0], lo[0][0]); gm::split(v.x, hi[0][1], lo[0][1]); gm::split(u.y, hi[0][2], lo[0][2]); gm::split(v.y, hi[0][3], lo[0][3]);
                        gm::split(u.z, hi[1][0], lo[1][0]); gm::split(v.z, hi[1][1], lo[1][1]); gm::split(u.w, hi[1][2], lo[1][2]); gm::split(v.w, hi[1][3], lo[1][3]);
#pragma unroll
                        for (uint32_t c = 0; c < NT; ++c) {
                            const float4 z = *reinterpret_cast<const float4*>(x + 8u * c * a.ld + 16u * (now.step + s));
                            uint32_t xh[4], xl[4];
                            gm::split(z.x, xh[0], xl[0]); gm::split(z.y, xh[1], xl[1]); gm::split(z.z, xh[2], xl[2]); gm::split(z.w, xh[3], xl[3]);
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                gm::mma_tf32(large[c], hi[h], xh[2 * h], xh[2 * h + 1]);
                                gm::mma_tf32(small[c], hi[h], xl[2 * h], xl[2 * h + 1]);
                                gm::mma_tf32(less[c], lo[h], xh[2 * h], xh[2 * h + 1]);
                            }
                        }
                    }
#pragma unroll
                    for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                        for (int i = 0; i < 4; ++i) sum[c][i] += large[c][i];
                    if (now.step + 4u < now.steps) continue;
#pragma unroll
                    for (uint32_t h = 0; h < 2u; ++h) {
                        const uint32_t out = now.tile * 16u + g + 8u * h;
                        const bool there = out < a.sizes[layer + 1u];
                        const float bias = there ? __ldg(w + a.b_at[layer] + out) : 0.f;
#pragma unroll
                        for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                            for (uint32_t i = 0; i < 2u; ++i) {
                                const uint32_t r = 8u * c + 2u * q + i;
                                const float s = gm::tanh32(gm::join(sum[c][2u * h + i], small[c][2u * h + i] + less[c][2u * h + i]) + bias);
                                if (!last_layer) {
                                    y[r * a.ld + out] = there ? s : 0.f;                    // (zeros up to 16: the next layer's contracted index)
                                } else if (there && r < rows) {
                                    static_cast<float*>(a.g.y)[(row + r) * a.g.ld_y + out] = a.g.scale * s;
                                }
                            }
                    }
                }
                meet();
            }
        }
    }
}

}  // namespace

bool member_plan(MemberArgs* a)
{
    // passes of 8 rows, or of 16 where members have more than 8 on average
    a->row_tiles = a->g.rows > 8ull * a->g.groups ? 2u : 1u;
    uint32_t widest = 16;
    a->aligned = 0;
    for (uint32_t l = 0; l < a->n_layers; ++l) {
        widest = std::max(widest, a->sizes[l]);
        if ((a->w_at[l] | a->sizes[l]) % 4u == 0u) a->aligned |= 1u << l;                   // (rows of theta are aligned)
    }
    if (widest > 512u) return false;
    // 4 more than a multiple of 32 floats: the eight rows of an MMA operand, 16 bytes a lane, fall on different banks
    a->ld = (widest + 31u) / 32u * 32u + 4u;
    return true;
}

int launch_member_rows(cudaStream_t st, const MemberArgs& in)
{
    MemberArgs a = in;
    const uint32_t pass = 8u * a.row_tiles;
    const uint64_t used = std::max<uint64_t>(1u, std::min<uint64_t>(a.g.groups, a.g.rows));
    // passes over a member's rows, on average, that can be worked on at the same time
    const uint64_t passes = std::max<uint64_t>(1u, (a.g.rows + pass - 1u) / pass / a.g.groups);
    const uint64_t tiles = (a.sizes[1] + 15u) / 16u, places = 12u * kSms;          // warps that run together, about
    const size_t each = (a.n_layers == 1u ? 1u : 2u) * pass * static_cast<size_t>(a.ld) * sizeof(float);
    // A warp an item where that gives most of them something to do and leaves room for three blocks of an SM; else eight warps an item.  A
    // single layer's outputs are dealt out in parts until there are two rounds of items.
    const bool fits = kAlone * each <= 72u * 1024u;
    const bool alone = fits && (a.n_layers == 1u || used * passes >= places / 2u);
    const uint64_t least = alone ? 1u : kTeam, wanted = 2u * places / (alone ? 1u : kTeam);
    a.chunks = a.n_layers == 1u ? static_cast<uint32_t>(std::max<uint64_t>(1u, std::min((tiles + least - 1u) / least, (wanted + used * passes - 1u) / (used * passes)))) : 1u;
    const uint64_t items = static_cast<uint64_t>(a.g.groups) * a.chunks;
    if (items > 0x7FFFFFFFull) return -2;
    const size_t bytes = alone ? kAlone * each : each;
    auto kernel = alone ? (a.row_tiles == 1u ? k_member_rows<1, 1> : k_member_rows<2, 1>) : (a.row_tiles == 1u ? k_member_rows<1, kTeam> : k_member_rows<2, kTeam>);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess) return -1;
    const uint64_t teams = alone ? (items + kAlone - 1u) / kAlone : items;
    const dim3 grid(static_cast<uint32_t>(std::min<uint64_t>(teams, 1u << 20)), static_cast<uint32_t>(std::min<uint64_t>(passes, 4096u)));
    return launch_dependent(kernel, grid, dim3(32u * (alone ? kAlone : kTeam)), bytes, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace evo

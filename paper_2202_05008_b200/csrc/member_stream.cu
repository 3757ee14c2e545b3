// Members' fp32 weights against the rows that belong to them: all layers of an MLP policy in one launch (get_actions), or one layer of
// any width (products grouped by member).
//
// A population's weights are read once, so their way from memory is the bound, and it must never pause.  A block stays and takes member
// after member; a warp of it copies weight rows, 16 outputs and more a stage, into a ring that goes on to the next member's while
// eight others still work on this one's.  A tile of 16 outputs by 8 (or four times 8) rows is a chain of mma.sync on pairs of tf32
// numbers (grouped_mma.cuh); activations pass from layer to layer through shared memory; the next rows of observations are on their way too.
// STREAM_TIME
#include <algorithm>

#include "async.cuh"
#include "grouped_mma.cuh"
#include "member_stream.h"

namespace evo {
namespace {

constexpr uint32_t kWarps = 8, kWorkers = kWarps * 32, kThreads = kWorkers + 32;
constexpr uint32_t kMostStages = 24;

__device__ __forceinline__ void copy_async4(uint32_t dst, const float* src, bool there)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(dst), "l"(src), "r"(there ? 4u : 0u) : "memory");
}

// Walks the items of a block: (member, part of its outputs, share of its rows) by (as many rows as a pass takes)
struct Walk {
    uint64_t item, row, end;
    uint32_t member, chunk;
    __device__ __forceinline__ bool find(const StreamArgs& a, uint32_t pass)          // from `item` on
    {
        const uint64_t items = static_cast<uint64_t>(a.g.groups) * a.chunks * a.shares;
        for (; item < items; item += gridDim.x) {
            const uint32_t share = static_cast<uint32_t>(item % a.shares);
            const uint64_t rest = item / a.shares;
            chunk = static_cast<uint32_t>(rest % a.chunks);
            member = static_cast<uint32_t>(rest / a.chunks);
            uint64_t first;
            group_rows(a.g, member, &first, &end);
            row = first + static_cast<uint64_t>(share) * pass;
            if (row < end) {
                // where the next item's rows are, for when it is asked for
                const uint64_t ahead = (item + gridDim.x) / (static_cast<uint64_t>(a.shares) * a.chunks);
                if (ahead < a.g.groups)
                    asm volatile("prefetch.global.L1 [%0];" :: "l"(static_cast<const char*>(a.g.offsets) + ahead * (a.g.wide_offsets ? 8u : 4u)));
                return true;
            }
        }
        return false;
    }
    __device__ __forceinline__ bool next(const StreamArgs& a, uint32_t pass)
    {
        row += static_cast<uint64_t>(a.shares) * pass;
        if (row < end) return true;
        item += gridDim.x;
        return find(a, pass);
    }
};
// sixteens of outputs of a layer that an item has: [first, last)
__device__ __forceinline__ void tiles_of(const StreamArgs& a, uint32_t layer, uint32_t chunk, uint32_t* first, uint32_t* last)
{
    const uint32_t all = (a.sizes[layer + 1u] + 15u) / 16u, per = (all + a.chunks - 1u) / a.chunks;
    *first = min(chunk * per, all);
    *last = min(*first + per, all);
}

// Sums of 16 outputs (weight rows w0 and, 8 further on, w1 of this lane) and 8 NT rows of x, of which those of the first `rows` are needed
template <uint32_t NT, bool VEC>
__device__ __forceinline__ void tile_sums(const float* w0, const float* w1, const float* x, uint32_t ld_x, uint32_t n_in, uint32_t rows, float (&sum)[NT][4])
{
    const uint32_t g = (threadIdx.x & 31u) >> 2, q = threadIdx.x & 3u;
    float large[NT][4] = {}, small[NT][4] = {}, less[NT][4] = {};          // hi hi', hi lo', lo hi'
#pragma unroll
    for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[c][i] = 0.f;
    const uint32_t steps = (n_in + 15u) / 16u;
#pragma unroll 4
    for (uint32_t s = 0; s < steps; ++s) {
        const uint32_t kk = 16u * s + 4u * q;
        float u[4], v[4];
        if constexpr (VEC) {
            const float4 m0 = kk < n_in ? *reinterpret_cast<const float4*>(w0 + kk) : make_float4(0.f, 0.f, 0.f, 0.f);
            const float4 m1 = kk < n_in ? *reinterpret_cast<const float4*>(w1 + kk) : make_float4(0.f, 0.f, 0.f, 0.f);
            u[0] = m0.x; u[1] = m0.y; u[2] = m0.z; u[3] = m0.w;
            v[0] = m1.x; v[1] = m1.y; v[2] = m1.z; v[3] = m1.w;
        } else {
#pragma unroll
            for (uint32_t e = 0; e < 4u; ++e) {
                u[e] = kk + e < n_in ? w0[kk + e] : 0.f;
                v[e] = kk + e < n_in ? w1[kk + e] : 0.f;
            }
        }
        uint32_t hi[2][4], lo[2][4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            gm::split(u[2 * h], hi[h][0], lo[h][0]);
            gm::split(v[2 * h], hi[h][1], lo[h][1]);
            gm::split(u[2 * h + 1], hi[h][2], lo[h][2]);
            gm::split(v[2 * h + 1], hi[h][3], lo[h][3]);
        }
#pragma unroll
        for (uint32_t c = 0; c < NT; ++c) {
            if (c && 8u * c >= rows) break;
            const float4 p = *reinterpret_cast<const float4*>(x + (8u * c + g) * ld_x + kk);
            uint32_t xh[4], xl[4];
            gm::split(p.x, xh[0], xl[0]); gm::split(p.y, xh[1], xl[1]); gm::split(p.z, xh[2], xl[2]); gm::split(p.w, xh[3], xl[3]);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                gm::mma_tf32(large[c], hi[h], xh[2 * h], xh[2 * h + 1]);
                gm::mma_tf32(small[c], hi[h], xl[2 * h], xl[2 * h + 1]);
                gm::mma_tf32(less[c], lo[h], xh[2 * h], xh[2 * h + 1]);
            }
        }
        if (s % 4u == 3u || s + 1u == steps)
#pragma unroll
            for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) { sum[c][i] += large[c][i]; large[c][i] = 0.f; }
    }
#pragma unroll
    for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[c][i] = gm::join(sum[c][i], small[c][i] + less[c][i]);
}

template <uint32_t NT>
__global__ void __launch_bounds__(kThreads, NT == 1u ? 2 : 1) k_member_stream(const __grid_constant__ StreamArgs a)
{
    extern __shared__ __align__(128) float smem[];
    __shared__ __align__(8) uint64_t full[kMostStages], empty[kMostStages];
    __shared__ uint32_t limit;
    __shared__ volatile int abort_flag;
    constexpr uint32_t kPass = 8u * NT;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    float* const ring = smem;
    float* const in = smem + a.stages * a.stage_floats;                    // two of [kPass][ld_in]
    float* const hidden = in + 2u * kPass * a.ld_in;                       // two of [kPass][ld_hidden]
    float* const biases = hidden + 2u * kPass * a.ld_hidden;               // two of all layers' biases
    if (tid == 0) {
        for (uint32_t s = 0; s < a.stages; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), kWarps); }
        mbar_init_fence();
        limit = 31u;
        abort_flag = 0;
    }
    __syncthreads();
    dep_wait();
    dep_trigger();
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(smem_u32(bar), parity) || abort_flag) return;
        if (!mbar_wait_bounded(smem_u32(bar), parity, &limit)) abort_flag = 1;
    };
    Walk at;
    at.item = blockIdx.x;
    uint32_t stage = 0, phase = 0;
    if (warp == kWarps) {
        uint32_t filled = 0;
        for (bool more = at.find(a, kPass); more; more = at.next(a, kPass)) {
            const float* const w = a.w + at.member * a.stride_w;
            for (uint32_t l = 0; l < a.n_layers && !abort_flag; ++l) {
                uint32_t t, last;
                tiles_of(a, l, at.chunk, &t, &last);
                for (; t < last; t += a.tiles_a_stage[l]) {
                    const uint32_t o0 = t * 16u, o1 = min(min(t + a.tiles_a_stage[l], last) * 16u, a.sizes[l + 1u]);
                    const uint64_t from = a.w_at[l] + static_cast<uint64_t>(o0) * a.sizes[l], to = a.w_at[l] + static_cast<uint64_t>(o1) * a.sizes[l];
                    wait(&empty[stage], phase ^ 1u);
                    if (__any_sync(0xffffffffu, abort_flag)) break;
                    // (16-byte ends: what lies before and behind is the member's too; the last few floats of a member come by themselves)
                    if (lane == 0) {
                        float* const there = ring + stage * a.stage_floats;
                        const uint64_t begin = from & ~3ull;
                        uint64_t end = (to + 3u) / 4u * 4u;
                        if (end > a.w_end) {
                            end = to / 4u * 4u;
                            for (uint64_t e = end; e < to; ++e) there[e - begin] = w[e];
                        }
                        if (end > begin) bulk_copy_g2s(smem_u32(there), w + begin, static_cast<uint32_t>(end - begin) * 4u, smem_u32(&full[stage]));
                        else mbar_arrive(smem_u32(&full[stage]));
                    }
                    __syncwarp();
                    ++filled;
                    if (++stage == a.stages) { stage = 0; phase ^= 1u; }
                }
            }
            if (__any_sync(0xffffffffu, abort_flag)) break;
        }
        if (__any_sync(0xffffffffu, abort_flag))                           // nothing may land after the block has gone
            for (uint32_t s = 0; s < min(filled, a.stages); ++s) {
                const uint32_t nth = filled - 1u - s;
                mbar_wait_bounded(smem_u32(&full[nth % a.stages]), nth / a.stages & 1u, &limit);
            }
        return;
    }
    const uint32_t g = lane >> 2, q = lane & 3u, in0 = a.sizes[0], pad0 = (in0 + 15u) / 16u * 16u;
    auto fetch = [&](const Walk& of, uint32_t buffer) {                     // rows of observations, zeros behind the last and up to 16
        const float* const x = static_cast<const float*>(a.g.x);
        for (uint32_t t = tid; t < kPass * pad0; t += kWorkers) {
            const uint32_t r = t / pad0, k = t % pad0;
            const bool there = of.row + r < of.end && k < in0;
            copy_async4(smem_u32(in + (buffer * kPass + r) * a.ld_in + k), x + (there ? (of.row + r) * a.g.ld_x + k : 0u), there);
        }
        float* to = biases + buffer * a.bias_floats;
        for (uint32_t l = 0; l < a.n_layers; ++l) {                         // biases of the item's outputs
            uint32_t t0, t1;
            tiles_of(a, l, of.chunk, &t0, &t1);
            const uint32_t count = min(t1 * 16u, a.sizes[l + 1u]) - min(t0 * 16u, a.sizes[l + 1u]);
            for (uint32_t t = tid; t < count; t += kWorkers)
                copy_async4(smem_u32(to + t), a.b ? a.b + of.member * a.stride_b + a.b_at[l] + t0 * 16u + t : a.w, a.b != nullptr);
            to += (t1 - t0) * 16u;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    bool more = at.find(a, kPass);
    if (more) fetch(at, 0u);
    for (uint32_t cur = 0; more; cur ^= 1u) {
        Walk then = at;
        const bool another = then.next(a, kPass);
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        asm volatile("bar.sync 1, %0;" :: "n"(kWorkers) : "memory");        // (and all have done with the buffers that are written next)
        if (another) fetch(then, cur ^ 1u);
        const uint32_t rows = static_cast<uint32_t>(min(static_cast<uint64_t>(kPass), at.end - at.row));
        const float* bias = biases + cur * a.bias_floats;
        for (uint32_t l = 0; l < a.n_layers; ++l) {
            const uint32_t n_in = a.sizes[l], n_out = a.sizes[l + 1u];
            const bool last_layer = l + 1u == a.n_layers, vec = a.aligned >> l & 1u;
            const float* const x = l ? hidden + (l - 1u & 1u) * kPass * a.ld_hidden : in + cur * kPass * a.ld_in;
            const uint32_t ld_x = l ? a.ld_hidden : a.ld_in;
            float* const y = hidden + (l & 1u) * kPass * a.ld_hidden;
            uint32_t first, last;
            tiles_of(a, l, at.chunk, &first, &last);
            for (uint32_t t0 = first; t0 < last; t0 += a.tiles_a_stage[l]) {
                wait(&full[stage], phase);
                const uint32_t t1 = min(t0 + a.tiles_a_stage[l], last);
                const uint32_t shift = static_cast<uint32_t>((a.w_at[l] + static_cast<uint64_t>(t0) * 16u * n_in) & 3u);
                const float* const rows_at = ring + stage * a.stage_floats + shift;
                for (uint32_t t = t0 + (warp + kWarps - (t0 - first) % kWarps) % kWarps; t < t1; t += kWarps) {
                    const uint32_t o = t * 16u + g;
                    const float b0 = o < n_out ? bias[o - first * 16u] : 0.f, b1 = o + 8u < n_out ? bias[o + 8u - first * 16u] : 0.f;
                    // what is beyond the last output is read as the last one, and not used
                    const float* const w0 = rows_at + (min(o, n_out - 1u) - t0 * 16u) * n_in;
                    const float* const w1 = rows_at + (min(o + 8u, n_out - 1u) - t0 * 16u) * n_in;
                    float sum[NT][4];
                    if (vec) tile_sums<NT, true>(w0, w1, x, ld_x, n_in, rows, sum);
                    else tile_sums<NT, false>(w0, w1, x, ld_x, n_in, rows, sum);
#pragma unroll
                    for (uint32_t c = 0; c < NT; ++c)
#pragma unroll
                        for (uint32_t i = 0; i < 4u; ++i) {
                            const uint32_t row = 8u * c + 2u * q + (i & 1u), out = o + 8u * (i >> 1);
                            if (c && 8u * c >= rows) continue;
                            float s = sum[c][i] + (i >> 1 ? b1 : b0);
                            if (!last_layer || a.g.activation == EVO_ACT_TANH) s = tanhf(s);
                            if (!last_layer) {
                                y[row * a.ld_hidden + out] = out < n_out ? s : 0.f;           // (zeros up to 16: the next layer's contracted index)
                            } else if (out < n_out && row < rows) {
                                if (a.g.activation == EVO_ACT_RELU) s = s < 0.f ? 0.f : s;
                                static_cast<float*>(a.g.y)[(at.row + row) * a.g.ld_y + out] = abort_flag ? __int_as_float(0x7FC00000) : a.g.scale * s;
                            }
                        }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                if (++stage == a.stages) { stage = 0; phase ^= 1u; }
            }
            bias += (last - first) * 16u;
            if (!last_layer) asm volatile("bar.sync 1, %0;" :: "n"(kWorkers) : "memory");
        }
        at = then;
        more = another;
    }
}

}  // namespace

bool stream_plan(StreamArgs* a, size_t* bytes)
{
    // passes of 8 rows, or of 32 where members have more than 8 on average (those that have fewer than 32 leave out what holds no row)
    a->row_tiles = a->g.rows > 8ull * a->g.groups ? 4u : 1u;
    const uint32_t pass = 8u * a->row_tiles;
    uint32_t widest_in = 0, hidden = 16;
    uint64_t total = 0;
    a->aligned = 0;
    for (uint32_t l = 0; l < a->n_layers; ++l) {
        widest_in = std::max(widest_in, a->sizes[l]);
        if (l) hidden = std::max(hidden, a->sizes[l]);
        total += static_cast<uint64_t>(a->sizes[l]) * a->sizes[l + 1];
        if (a->w_at[l] % 4u == 0u && a->sizes[l] % 4u == 0u) a->aligned |= 1u << l;
    }
    if (widest_in > 2048u || hidden > 1024u) return false;
    // parts of a wide layer's outputs where there are too few members to go round: eight tiles (one for each warp) at least, 64 at most
    const uint64_t used = std::max<uint64_t>(1u, std::min<uint64_t>(a->g.groups, a->g.rows));
    a->chunks = 1u;
    if (a->n_layers == 1u) {
        const uint64_t least = (a->sizes[1] + 1023u) / 1024u, most = (a->sizes[1] + 127u) / 128u;
        a->chunks = static_cast<uint32_t>(std::min(most, std::max<uint64_t>(least, (8u * kSms + used - 1u) / used)));
    }
    a->bias_floats = 0;
    for (uint32_t l = 0; l < a->n_layers; ++l) a->bias_floats += ((a->sizes[l + 1] + 15u) / 16u + a->chunks - 1u) / a->chunks * 16u;
    a->bias_floats = (a->bias_floats + 31u) / 32u * 32u;
    // 4 more than a multiple of 32 floats: the eight rows of an MMA operand, 16 bytes a lane, fall on different banks
    a->ld_in = (a->sizes[0] + 31u) / 32u * 32u + 4u;
    a->ld_hidden = a->n_layers > 1u ? (hidden + 31u) / 32u * 32u + 4u : 0u;
    const size_t act = 2u * (pass * static_cast<size_t>(a->ld_in + a->ld_hidden) + a->bias_floats) * sizeof(float);
    const size_t room = (a->row_tiles == 1u ? 112u : 220u) * 1024u, most = 220u * 1024u;
    a->stage_floats = (std::max(16u * widest_in, 2048u) + 3u + 31u) / 32u * 32u;
    for (uint32_t l = 0; l < a->n_layers; ++l) a->tiles_a_stage[l] = std::max(1u, (a->stage_floats - 3u) / (16u * a->sizes[l]));
    const size_t stage = a->stage_floats * sizeof(float);
    // two blocks an SM where four stages fit a half, else one
    size_t space = act + 4u * stage <= room ? room : most;
    if (act + 2u * stage > space) return false;
    a->stages = static_cast<uint32_t>(std::min<size_t>(kMostStages, (space - act) / stage));
    // no more of them than a few members have
    const uint64_t useful = std::max<uint64_t>(2u, 4u * ((total + a->stage_floats - 1u) / a->stage_floats + a->n_layers));
    a->stages = static_cast<uint32_t>(std::min<uint64_t>(a->stages, useful));
    *bytes = act + a->stages * stage;
    return true;
}

int launch_stream(cudaStream_t st, const StreamArgs& in, size_t bytes)
{
    StreamArgs a = in;
    const uint32_t pass = 8u * a.row_tiles;
    // shares of a member's rows where there are too few members to go round: a pass each on average
    const uint64_t places = 2u * kSms;
    const uint64_t passes = (a.g.rows + pass - 1u) / pass;
    const uint64_t most = (passes + a.g.groups - 1u) / a.g.groups;
    a.shares = static_cast<uint32_t>(std::max<uint64_t>(1u, std::min(most, (places + static_cast<uint64_t>(a.g.groups) * a.chunks - 1u) / (static_cast<uint64_t>(a.g.groups) * a.chunks))));
    const uint64_t items = static_cast<uint64_t>(a.g.groups) * a.chunks * a.shares;
    auto kernel = a.row_tiles == 1u ? k_member_stream<1> : k_member_stream<4>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess) return -1;
    const uint64_t resident = bytes <= 112u * 1024u && a.row_tiles == 1u ? 2u * kSms : kSms;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(std::min(items, resident))), dim3(kThreads), bytes, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace evo

// The MLP policy's get_actions over the rows of every member: all layers in one launch.
//
// A block takes a member (or a share of its rows where members are few): the member's parameter row comes into shared memory as
// one bulk copy per layer, so the first layer runs while the others are on their way, and is read from memory once however many
// rows there are.  Rows go through the layers 16 at a time, activations in shared memory; a warp makes 16 outputs.
#include "grouped.h"
#include "grouped_mma.cuh"
#include "async.cuh"
#include "mlp_actions.h"

namespace evo {
namespace {

constexpr uint32_t kThreads = 256;
constexpr uint32_t kRows = 16;           // rows that go through the layers together: two eights of MMA columns

__device__ __forceinline__ const float* clamp_row(const float* base, uint32_t row, uint32_t rows, uint32_t ld) { return base + min(row, rows - 1u) * ld; }

__global__ void __launch_bounds__(kThreads) k_mlp_actions(const __grid_constant__ ActionsArgs a)
{
    extern __shared__ __align__(128) float smem[];
    __shared__ __align__(8) uint64_t bar[EVO_MAX_LAYERS];
    __shared__ uint32_t limit;
    __shared__ volatile int abort_flag;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, g = lane >> 2, q = lane & 3u;
    const uint32_t member = blockIdx.x / a.shares, share = blockIdx.x % a.shares;
    float* const theta = smem;
    float* const act[2] = { smem + a.act_at, smem + a.act_at + kRows * a.ld_act };
    if (tid == 0) {
        for (uint32_t l = 0; l < a.n_layers; ++l) mbar_init(smem_u32(&bar[l]), 1);
        mbar_init_fence();
        limit = 31u;
        abort_flag = 0;
    }
    __syncthreads();
    dep_wait();
    dep_trigger();
    uint64_t first, end;
    group_rows(a.g, member, &first, &end);
    uint64_t r = first + static_cast<uint64_t>(share) * kRows;
    if (r >= end) return;
    // (pieces start and end on 16 bytes; what two layers share comes with the first of them, the last few floats by themselves)
    if (tid >= 32u && tid - 32u < a.dim - a.piece[a.n_layers]) theta[a.piece[a.n_layers] + tid - 32u] = a.theta[member * a.ld_theta + a.piece[a.n_layers] + tid - 32u];
    if (tid < a.n_layers) {
        const uint32_t from = a.piece[tid], to = a.piece[tid + 1u];
        if (from == to) mbar_arrive(smem_u32(&bar[tid]));
        else bulk_copy_g2s(smem_u32(theta + from), a.theta + member * a.ld_theta + from, (to - from) * 4u, smem_u32(&bar[tid]));
    }
    uint32_t arrived = 0;
    for (; r < end; r += static_cast<uint64_t>(a.shares) * kRows) {
        const uint32_t rows = static_cast<uint32_t>(min(static_cast<uint64_t>(kRows), end - r));
        // the rows of observations, padded with zeros to the pitch
        const uint32_t in0 = a.sizes[0], pad0 = (in0 + 15u) / 16u * 16u;
        for (uint32_t t = tid; t < kRows * pad0; t += kThreads) {
            const uint32_t row = t / pad0, k = t % pad0;
            act[0][row * a.ld_act + k] = row < rows && k < in0 ? static_cast<const float*>(a.g.x)[(r + row) * a.g.ld_x + k] : 0.f;
        }
        __syncthreads();
        for (uint32_t l = 0; l < a.n_layers; ++l) {
            if (l >= arrived) {
                // layer l reads only what the copies 0 .. l brought
                if (!abort_flag && !mbar_wait_bounded(smem_u32(&bar[l]), 0u, &limit)) abort_flag = 1;
                arrived = l + 1u;
            }
            const uint32_t n_in = a.sizes[l], n_out = a.sizes[l + 1u], pad_out = (n_out + 15u) / 16u * 16u;
            const float* const w = theta + a.layer_at[l];
            const float* const bias = w + n_out * n_in;
            const float* const x = act[l & 1u];
            float* const y = act[(l + 1u) & 1u];
            const bool last = l + 1u == a.n_layers, two = rows > 8u;
            for (uint32_t o0 = warp * 16u; o0 < pad_out; o0 += kThreads / 2u) {
                const float* const w0 = clamp_row(w, o0 + g, n_out, n_in);
                const float* const w1 = clamp_row(w, o0 + g + 8u, n_out, n_in);
                float large[2][4] = {}, small[2][4] = {}, sum[2][4] = {};
                for (uint32_t k = 0; k < n_in; k += 16u) {
                    // a lane's k: 4 consecutive ones where the rows are aligned for it, else as they come
                    float u[4], v[4];
                    const uint32_t at = k + 4u * q;
                    if (a.aligned >> l & 1u) {
                        const bool in = at < n_in;
                        const float4 p = in ? *reinterpret_cast<const float4*>(w0 + at) : make_float4(0.f, 0.f, 0.f, 0.f);
                        const float4 s = in ? *reinterpret_cast<const float4*>(w1 + at) : make_float4(0.f, 0.f, 0.f, 0.f);
                        u[0] = p.x; u[1] = p.y; u[2] = p.z; u[3] = p.w;
                        v[0] = s.x; v[1] = s.y; v[2] = s.z; v[3] = s.w;
                    } else {
#pragma unroll
                        for (uint32_t e = 0; e < 4u; ++e) {
                            u[e] = at + e < n_in ? w0[at + e] : 0.f;
                            v[e] = at + e < n_in ? w1[at + e] : 0.f;
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
                    for (uint32_t t = 0; t < 2u; ++t) {
                        if (t && !two) break;
                        const float4 p = *reinterpret_cast<const float4*>(x + (8u * t + g) * a.ld_act + at);
                        const float xs[4] = { p.x, p.y, p.z, p.w };
                        uint32_t xh[4], xl[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) gm::split(xs[e], xh[e], xl[e]);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            gm::mma_tf32(large[t], hi[h], xh[2 * h], xh[2 * h + 1]);
                            gm::mma_tf32(small[t], hi[h], xl[2 * h], xl[2 * h + 1]);
                            gm::mma_tf32(small[t], lo[h], xh[2 * h], xh[2 * h + 1]);
                        }
                    }
                    if ((k + 16u) % 64u == 0u || k + 16u >= n_in)
#pragma unroll
                        for (int t = 0; t < 2; ++t)
#pragma unroll
                            for (int i = 0; i < 4; ++i) { sum[t][i] += large[t][i]; large[t][i] = 0.f; }
                }
#pragma unroll
                for (uint32_t h = 0; h < 2u; ++h) {
                    const uint32_t o = o0 + g + 8u * h;
                    const float b = o < n_out ? bias[o] : 0.f;
#pragma unroll
                    for (uint32_t t = 0; t < 2u; ++t)
#pragma unroll
                        for (uint32_t i = 0; i < 2u; ++i) {
                            const uint32_t row = 8u * t + 2u * q + i;
                            const float s = gm::join(sum[t][2u * h + i], small[t][2u * h + i]);
                            if (last) {
                                if (o < n_out && row < rows)
                                    static_cast<float*>(a.g.y)[(r + row) * a.g.ld_y + o] = abort_flag ? __int_as_float(0x7FC00000) : a.g.scale * tanhf(s + b);
                            } else if (t == 0u || two) {
                                y[row * a.ld_act + o] = o < n_out ? tanhf(s + b) : 0.f;
                            }
                        }
                }
            }
            __syncthreads();
        }
    }
    // nothing may land after the block has gone (a time-out only: otherwise all layers were waited for)
    if (abort_flag)
        for (uint32_t l = 0; l < a.n_layers; ++l) mbar_wait_bounded(smem_u32(&bar[l]), 0u, &limit);
}

}  // namespace

bool actions_plan(const uint32_t* sizes, uint32_t n_layers, ActionsArgs* a, size_t* bytes)
{
    uint64_t at = 0;
    uint32_t widest = 16u;
    a->n_layers = n_layers;
    a->aligned = 0;
    a->piece[0] = 0;
    for (uint32_t l = 0; l <= n_layers; ++l) {
        a->sizes[l] = sizes[l];
        widest = sizes[l] > widest ? sizes[l] : widest;
    }
    for (uint32_t l = 0; l < n_layers; ++l) {
        if (at % 4u == 0u && sizes[l] % 4u == 0u) a->aligned |= 1u << l;
        a->layer_at[l] = static_cast<uint32_t>(at);
        at += static_cast<uint64_t>(sizes[l + 1]) * sizes[l] + sizes[l + 1];
        if (at > 65536u) return false;
        a->piece[l + 1u] = static_cast<uint32_t>((at + 3u) / 4u * 4u);
    }
    a->dim = static_cast<uint32_t>(at);
    for (uint32_t l = 1; l <= n_layers; ++l)
        if (a->piece[l] > a->dim / 4u * 4u) a->piece[l] = a->dim / 4u * 4u;
    // 4 more than a multiple of 32 floats: the eight rows of an MMA operand, 16 bytes a lane, fall on different banks
    a->ld_act = (widest + 31u) / 32u * 32u + 4u;
    a->act_at = (a->dim + 3u) / 4u * 4u;
    *bytes = (a->act_at + 2u * kRows * static_cast<size_t>(a->ld_act)) * sizeof(float);
    return *bytes <= 220u * 1024u;
}

int launch_actions(cudaStream_t st, const ActionsArgs& in, size_t bytes)
{
    ActionsArgs a = in;
    // shares of a member's rows: enough blocks for two per SM where members are few, none with less than a tile of rows on average
    const uint64_t tiles = (a.g.rows + kRows - 1u) / kRows;
    uint64_t shares = (2u * kSms + a.g.groups - 1u) / a.g.groups;
    const uint64_t most = (tiles + a.g.groups - 1u) / a.g.groups;
    if (shares > most) shares = most;
    if (shares < 1u) shares = 1u;
    a.shares = static_cast<uint32_t>(shares);
    if (shares * a.g.groups > 0x7FFFFFFFull) return -2;
    if (cudaFuncSetAttribute(k_mlp_actions, cudaFuncAttributeMaxDynamicSharedMemorySize, 220 * 1024) != cudaSuccess) return -1;
    return launch_dependent(k_mlp_actions, dim3(static_cast<uint32_t>(shares * a.g.groups)), dim3(kThreads), bytes, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace evo

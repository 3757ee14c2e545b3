// Newton-Schulz iteration of matrices of any size: one launch per product, over all matrices of the list.
//
// k_ns_norm sums the squares of pieces of 128 x 64 elements, k_ns_split writes X in panels (zero in the padding, and so is all
// that is made of it), k_ns_gemm<kGram / kPoly / kApply> is one of the three products of a step.  A block of k_ns_gemm walks over
// 128 x 128 tiles: a thread copies operands into a ring of three stages (64 of the contracted index: two pairs of 128 x 64
// matrices, 64 KB in four TMA boxes of 8 runs of 2 KB or 16 of 1 KB), another issues the MMAs, and eight warps take the sums out of tensor memory and
// turn them into fp16 pairs while the next ones are under way (two sets of accumulators).  A and B are symmetric: tiles on
// and under the diagonal only, written twice.
#include "newton_schulz.cuh"
#include "tma.h"

namespace evo {
namespace ns {

enum Product : uint32_t { kGram = 0, kPoly = 1, kApply = 2 };

constexpr uint32_t kStages = 3;
constexpr uint32_t kOperand = kTile * 64u * 2u;              // bytes of 128 x 64 halves
constexpr uint32_t kStage = 4u * kOperand;
constexpr uint32_t kTurn = 8u * 32u * 33u * 4u;              // where the eight warps turn 32 x 32 pairs
constexpr uint32_t kGemmSmem = kStages * kStage + kTurn;
constexpr uint32_t kGemmThreads = 320;

__device__ __forceinline__ const Group& group_of(const Args& a, uint32_t at, uint32_t Group::*first)
{
    uint32_t gi = 0;
    while (gi + 1u < a.groups && at >= a.g[gi + 1u].*first) ++gi;
    return a.g[gi];
}

// buffer 0, 1: X and the next X; 2: A; 3: B
__device__ __forceinline__ char* buffer(const Args& a, const Group& g, uint32_t which, uint32_t buf)
{
    const size_t x = static_cast<size_t>(g.mp) * g.np * 4u, q = static_cast<size_t>(g.mp) * g.mp * 4u;
    char* const base = a.work + g.work + which * (2u * x + 2u * q);
    return buf < 2u ? base + buf * x : base + 2u * x + (buf - 2u) * q;
}

// the eight elements (i, 8 jc ...) of a thread's turn in a piece: 128 rows x 8 panels over 256 threads
__device__ __forceinline__ void piece_place(const Group& g, uint32_t t, uint32_t& i, uint32_t& jc)
{
    if (g.tall) { i = t % kTile; jc = t / kTile; }
    else { jc = t / 8u % 8u; i = t / 64u * 8u + t % 8u; }
}

template <uint32_t SRC>
__global__ void __launch_bounds__(256) k_ns_norm(const __grid_constant__ Args a)
{
    __shared__ double red[8];
    dep_wait();
    dep_trigger();
    if (SRC == kMuon && a.skip && *a.skip == 0.0) return;
    const Group& g = group_of(a, blockIdx.x, &Group::first_block);
    const uint32_t pieces = g.mp / kTile * (g.np / kPieceCols), at = blockIdx.x - g.first_block, which = at / pieces, p = at % pieces;
    const uint32_t i0 = p % (g.mp / kTile) * kTile, j0 = p / (g.mp / kTile) * kPieceCols;
    double sum = 0.0;
    for (uint32_t t = threadIdx.x; t < kTile * 8u; t += 256u) {
        uint32_t i, jc;
        piece_place(g, t, i, jc);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            float unused;
            const double x = i0 + i < g.m && j0 + jc * 8u + e < g.n ? load<SRC>(a, in_index(g, which, i0 + i, j0 + jc * 8u + e), &unused) : 0.f;
            sum += x * x;
        }
    }
    sum = block_sum<256>(sum, red);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = sum;
}

template <uint32_t SRC>
__global__ void __launch_bounds__(256) k_ns_split(const __grid_constant__ Args a)
{
    __shared__ double red[8];
    dep_wait();
    dep_trigger();
    if (SRC == kMuon && a.skip && *a.skip == 0.0) return;
    const Group& g = group_of(a, blockIdx.x, &Group::first_block);
    const uint32_t pieces = g.mp / kTile * (g.np / kPieceCols), at = blockIdx.x - g.first_block, which = at / pieces, p = at % pieces;
    const uint32_t i0 = p % (g.mp / kTile) * kTile, j0 = p / (g.mp / kTile) * kPieceCols;
    double sum = 0.0;
    for (uint32_t k = threadIdx.x; k < pieces; k += 256u) sum += __ldcg(a.partial + blockIdx.x - p + k);
    uint32_t lift;
    const double scale = first_scale(a.s, block_sum<256>(sum, red), &lift);
    if (p == 0u && threadIdx.x == 0u) a.lift[g.first_matrix + which] = lift;
    char* const x_hi = buffer(a, g, which, 0u);
    char* const x_lo = x_hi + static_cast<size_t>(g.mp) * g.np * 2u;
    for (uint32_t t = threadIdx.x; t < kTile * 8u; t += 256u) {
        uint32_t i, jc;
        piece_place(g, t, i, jc);
        float x[8];
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            x[e] = 0.f;
            if (i0 + i < g.m && j0 + jc * 8u + e < g.n) {
                const uint64_t from = in_index(g, which, i0 + i, j0 + jc * 8u + e);
                float momentum;
                x[e] = static_cast<float>(scale * load<SRC>(a, from, &momentum));
                if constexpr (SRC == kMuon) store_moments(a, from, momentum);
            }
        }
        uint4 hi, lo;
        split8(x, hi, lo);
        const size_t to = (static_cast<size_t>(j0 / 8u + jc) * g.mp + i0 + i) * 16u;
        *reinterpret_cast<uint4*>(x_hi + to) = hi;
        *reinterpret_cast<uint4*>(x_lo + to) = lo;
    }
}

// A tile: which matrix, its place, how far the sum goes.  (Pairs of row blocks, I >= J, are numbered along the rows of the triangle.)
struct Tile {
    const Group* g;
    uint32_t which, i0, j0, k;
};
template <uint32_t MODE>
__device__ __forceinline__ Tile tile_at(const Args& a, uint32_t at)
{
    Tile t;
    t.g = &group_of(a, at, MODE == kApply ? &Group::first_tile : &Group::first_pair);
    const uint32_t rows = t.g->mp / kTile;
    if constexpr (MODE == kApply) {
        const uint32_t cols = (t.g->np + kTile - 1u) / kTile, local = at - t.g->first_tile, p = local % (rows * cols);
        t.which = local / (rows * cols);
        t.i0 = p % rows * kTile;
        t.j0 = p / rows * kTile;
        t.k = t.g->mp;
    } else {
        const uint32_t pairs = rows * (rows + 1u) / 2u, local = at - t.g->first_pair, p = local % pairs;
        t.which = local / pairs;
        uint32_t i = static_cast<uint32_t>((sqrtf(8.0f * static_cast<float>(p) + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1u) / 2u > p) --i;
        while ((i + 1u) * (i + 2u) / 2u <= p) ++i;
        t.i0 = i * kTile;
        t.j0 = (p - i * (i + 1u) / 2u) * kTile;
        t.k = MODE == kGram ? t.g->np : t.g->mp;
    }
    return t;
}

// A box of a buffer's panels to shared memory: runs of a panel (8-byte elements), panels, matrix of the group
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, uint32_t row, uint32_t panel, uint32_t which, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(2u * row), "r"(panel), "r"(which) : "memory");
}

// The operands of a product: kGram: X, kPoly: A (the same for both); kApply: B and X
struct Maps { CUtensorMap first[kMaxLarge], second[kMaxLarge]; };

template <uint32_t MODE, uint32_t SRC>
__global__ void __launch_bounds__(kGemmThreads, 1) k_ns_gemm(const __grid_constant__ Args a, const __grid_constant__ Maps maps, uint32_t step)
{
    const uint32_t cur = step & 1u;                              // which of the two X buffers holds X
    const bool last = step + 1u == a.s.steps;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) uint64_t full[kStages], empty[kStages], done[2], taken[2], drain;
    __shared__ uint32_t slot, limit;
    __shared__ volatile int abort_flag;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    if (tid == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
        for (uint32_t b = 0; b < 2u; ++b) { mbar_init(smem_u32(&done[b]), 1); mbar_init(smem_u32(&taken[b]), 8); }
        mbar_init(smem_u32(&drain), 1);
        mbar_init_fence();
        limit = a.wait_log2;
        abort_flag = 0;
    }
    dep_wait();
    dep_trigger();
    if (a.skip && *a.skip == 0.0) return;
    if (warp == 1) tmem_alloc(smem_u32(&slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = slot;
    const Waits waits{ &abort_flag, &limit, a.sticky };
    const uint32_t total = MODE == kApply ? a.tiles : a.pairs;

    if (warp == 0) {
        uint32_t stage = 0, phase = 0, filled = 0;
        for (uint32_t at = blockIdx.x; at < total; at += gridDim.x) {
            const Tile t = tile_at<MODE>(a, at);
            const uint32_t gi = static_cast<uint32_t>(t.g - a.g), lo = (MODE == kGram ? t.g->np : t.g->mp) / 8u, x_lo = t.g->np / 8u;
            const bool twice = MODE == kApply || t.i0 != t.j0;
            for (uint32_t k = 0; k < t.k; k += 64u) {
                waits.wait(smem_u32(&empty[stage]), phase ^ 1u);
                if (__any_sync(0xffffffffu, abort_flag)) break;
                if (lane == 0) {
                    const uint32_t bar = smem_u32(&full[stage]), to = smem_u32(smem) + stage * kStage;
                    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(twice ? kStage : kStage / 2u) : "memory");
                    copy_box(to, &maps.first[gi], t.i0, k / 8u, t.which, bar);
                    copy_box(to + kOperand, &maps.first[gi], t.i0, k / 8u + lo, t.which, bar);
                    if constexpr (MODE == kApply) {             // 64 rows of X by 16 panels (those beyond the last are not looked at)
                        copy_box(to + 2u * kOperand, &maps.second[gi], k, t.j0 / 8u, t.which, bar);
                        copy_box(to + 3u * kOperand, &maps.second[gi], k, t.j0 / 8u + x_lo, t.which, bar);
                    } else if (twice) {
                        copy_box(to + 2u * kOperand, &maps.first[gi], t.j0, k / 8u, t.which, bar);
                        copy_box(to + 3u * kOperand, &maps.first[gi], t.j0, k / 8u + lo, t.which, bar);
                    }
                }
                __syncwarp();
                ++filled;
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
            }
            if (__any_sync(0xffffffffu, abort_flag)) break;
        }
        if (__any_sync(0xffffffffu, abort_flag)) {               // nothing may land after the block has gone
            for (uint32_t s = 0; s < min(filled, kStages); ++s) {
                const uint32_t nth = filled - 1u - s;
                mbar_wait_bounded(smem_u32(&full[nth % kStages]), nth / kStages & 1u, &limit);
            }
        }
    } else if (warp == 1) {
        uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0;
        for (uint32_t at = blockIdx.x; at < total; at += gridDim.x) {
            const Tile t = tile_at<MODE>(a, at);
            const uint32_t panels = MODE == kApply ? min(16u, t.g->np / 8u - t.j0 / 8u) : 16u;
            const uint32_t idesc = idesc_f16(128, panels * 8u, MODE == kApply);
            for (uint32_t k = 0; k < t.k; k += 64u) {
                const uint32_t d = tmem + acc * 2u * kTile, low = d + kTile, fresh = k % kChunk == 0u;
                const bool ends = (k + 64u) % kChunk == 0u || k + 64u >= t.k;
                if (fresh) waits.wait(smem_u32(&taken[acc]), acc_phase ^ 1u);
                waits.wait(smem_u32(&full[stage]), phase);
                tc_fence_after();
                if (__any_sync(0xffffffffu, abort_flag)) break;
                if (lane == 0) {
                    const uint32_t p = smem_u32(smem) + stage * kStage;
                    const uint32_t q = MODE == kApply || t.i0 != t.j0 ? p + 2u * kOperand : p;
                    for (uint32_t s = 0; s < 4u; ++s) {
                        // K-major: 16 of the contracted index are two panels (2 KB apart); MN-major: two groups of 8 rows (128 bytes apart)
                        const uint32_t po = s * 4096u, qo = MODE == kApply ? s * 256u : s * 4096u;
                        const uint32_t ks = MODE == kApply ? 128u : 2048u, ms = MODE == kApply ? 1024u : 128u;
                        const uint64_t ph = umma_smem_desc(p + po, 2048u, 128u), pl = umma_smem_desc(p + kOperand + po, 2048u, 128u);
                        const uint64_t qh = umma_smem_desc(q + qo, ks, ms), ql = umma_smem_desc(q + kOperand + qo, ks, ms);
                        const uint32_t more = fresh && s == 0u ? 0u : 1u;
                        umma_bf16(d, ph, qh, idesc, more);
                        umma_bf16(low, ph, ql, idesc, more);
                        umma_bf16(low, pl, qh, idesc, 1u);
                    }
                    umma_commit(smem_u32(&empty[stage]));
                    if (ends) umma_commit(smem_u32(&done[acc]));
                }
                __syncwarp();
                if (++stage == kStages) { stage = 0; phase ^= 1u; }
                if (ends) {
                    acc ^= 1u;
                    if (acc == 0u) acc_phase ^= 1u;
                }
            }
            if (__any_sync(0xffffffffu, abort_flag)) break;
        }
        if (__any_sync(0xffffffffu, abort_flag)) {               // nor may an MMA write after its tensor memory is freed
            if (lane == 0) umma_commit(smem_u32(&drain));
            __syncwarp();
            mbar_wait_bounded(smem_u32(&drain), 0u, &limit);
        }
    } else {
        const uint32_t quarter = warp & 3u, part = (warp - 2u) >> 2, row = quarter * 32u + lane;      // 64 columns of 32 rows
        uint32_t* const turn = reinterpret_cast<uint32_t*>(smem + kStages * kStage) + (warp - 2u) * 32u * 33u;
        const float poly_b = a.s.b * a.s.s_b / a.s.s_a, poly_c = a.s.c * a.s.s_b / (a.s.s_a * a.s.s_a), from_bx = 1.0f / a.s.s_b;
        uint32_t acc = 0, acc_phase = 0;
        for (uint32_t at = blockIdx.x; at < total; at += gridDim.x) {
            const Tile t = tile_at<MODE>(a, at);
            const Group& g = *t.g;
            const uint32_t first_lift = __ldcg(a.lift + g.first_matrix + t.which), lift = lift_at(a.s, first_lift, step);
            const uint32_t next_lift = lift_at(a.s, first_lift, step + 1u);
            const float to_a = power_of_two(-2 * static_cast<int>(lift)) * (a.s.s_a / (a.s.s_x * a.s.s_x));
            const float drop = power_of_two(static_cast<int>(next_lift) - static_cast<int>(lift));
            const size_t q_half = static_cast<size_t>(g.mp) * g.mp * 2u, x_half = static_cast<size_t>(g.mp) * g.np * 2u;
            const char* const old = buffer(a, g, t.which, MODE == kApply ? cur : 2u);
            char* const out = buffer(a, g, t.which, MODE == kGram ? 2u : MODE == kPoly ? 3u : cur ^ 1u);
            const size_t half = MODE == kApply ? x_half : q_half;
            const uint32_t width = MODE == kApply ? min(kTile, g.np - t.j0) : kTile;
            float sum[2][4][8];
            for (uint32_t k = 0; k < t.k; k += kChunk) {
                const float cut = MODE == kGram ? kCut * static_cast<float>(min(kChunk, t.k - k) / 16u) : 0.f;
                waits.wait(smem_u32(&done[acc]), acc_phase);
                tc_fence_after();
#pragma unroll
                for (uint32_t h = 0; h < 2u; ++h) {
                    uint32_t u[4][8], v[4][8];
                    const uint32_t from = tmem + acc * 2u * kTile + (quarter << 21) + part * 64u + h * 32u;
                    tmem_ld32_issue(from, u);
                    tmem_ld32_issue(from + kTile, v);
                    tmem_ld8x4_fence(u[0], u[1], u[2], u[3]);
                    tmem_ld8x4_fence(v[0], v[1], v[2], v[3]);
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float x = __uint_as_float(u[c][e]) + fmaf(cut, __uint_as_float(u[c][e]), __uint_as_float(v[c][e]));
                            sum[h][c][e] = k == 0u ? x : sum[h][c][e] + x;
                        }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&taken[acc]));
                acc ^= 1u;
                if (acc == 0u) acc_phase ^= 1u;
            }
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h) {
                const uint32_t c0 = part * 64u + h * 32u;
                if (c0 >= width) break;
                uint4 hi[4], lo[4];
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c) {
                    const size_t place = (static_cast<size_t>(t.j0 / 8u + c0 / 8u + c) * g.mp + t.i0 + row) * 16u;
                    float x[8];
                    if constexpr (MODE == kGram) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = to_a * sum[h][c][e];
                    } else {
                        join8(__ldcg(reinterpret_cast<const uint4*>(old + place)), __ldcg(reinterpret_cast<const uint4*>(old + half + place)), x);
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            x[e] = MODE == kPoly ? fmaf(poly_b, x[e], poly_c * sum[h][c][e]) : drop * fmaf(a.s.a, x[e], from_bx * sum[h][c][e]);
                    }
                    if (MODE == kApply && last) {
                        const float back = abort_flag ? __int_as_float(0x7FC00000) : power_of_two(-static_cast<int>(next_lift)) / a.s.s_x;
                        if (t.i0 + row < g.m) {
#pragma unroll
                            for (uint32_t e = 0; e < 8u; ++e) {
                                const uint32_t j = t.j0 + c0 + c * 8u + e;
                                if (j < g.n) store<SRC>(a, out_index(g, t.which, t.i0 + row, j), x[e] * back, g.gain);
                            }
                        }
                    } else {
                        split8(x, hi[c], lo[c]);
                        *reinterpret_cast<uint4*>(out + place) = hi[c];
                        *reinterpret_cast<uint4*>(out + half + place) = lo[c];
                    }
                }
                if (MODE != kApply && t.i0 != t.j0) {             // the same above the diagonal: thread `lane` takes column c0 + lane as its row
                    __syncwarp();
#pragma unroll
                    for (uint32_t c = 0; c < 4u; ++c) {
                        const uint32_t p[4] = { hi[c].x, hi[c].y, hi[c].z, hi[c].w }, q[4] = { lo[c].x, lo[c].y, lo[c].z, lo[c].w };
#pragma unroll
                        for (uint32_t e = 0; e < 4u; ++e) {
                            turn[(c * 8u + 2u * e) * 33u + lane] = __byte_perm(p[e], q[e], 0x5410);
                            turn[(c * 8u + 2u * e + 1u) * 33u + lane] = __byte_perm(p[e], q[e], 0x7632);
                        }
                    }
                    __syncwarp();
#pragma unroll
                    for (uint32_t c = 0; c < 4u; ++c) {
                        uint32_t p[4], q[4];
#pragma unroll
                        for (uint32_t e = 0; e < 4u; ++e) {
                            const uint32_t x = turn[lane * 33u + c * 8u + 2u * e], y = turn[lane * 33u + c * 8u + 2u * e + 1u];
                            p[e] = __byte_perm(x, y, 0x5410);
                            q[e] = __byte_perm(x, y, 0x7632);
                        }
                        const size_t place = (static_cast<size_t>((t.i0 + quarter * 32u) / 8u + c) * g.mp + t.j0 + c0 + lane) * 16u;
                        *reinterpret_cast<uint4*>(out + place) = make_uint4(p[0], p[1], p[2], p[3]);
                        *reinterpret_cast<uint4*>(out + half + place) = make_uint4(q[0], q[1], q[2], q[3]);
                    }
                    __syncwarp();
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// boxes of `rows` x `panels` of a buffer (high and low parts: twice cols / 8 panels) of all matrices of a group
static bool encode(EncodeTiled f, CUtensorMap* map, char* base, const Group& g, uint32_t cols, uint32_t rows, uint32_t panels)
{
    const cuuint64_t dims[3] = { 2ull * g.mp, cols / 4u, g.count }, strides[2] = { 16ull * g.mp, large_bytes(g.mp, g.np) };
    const cuuint32_t box[3] = { 2u * rows, panels, 1u }, steps[3] = { 1u, 1u, 1u };
    return f(map, CU_TENSOR_MAP_DATA_TYPE_INT64, 3, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <uint32_t SRC>
static int launch_list(cudaStream_t st, const Args& a)
{
    static_assert(kGemmSmem <= 227u * 1024u - 512u, "the ring and the turning space fit a block");
    const void* kernels[3] = { reinterpret_cast<const void*>(k_ns_gemm<kGram, kF32>), reinterpret_cast<const void*>(k_ns_gemm<kPoly, kF32>),
                               reinterpret_cast<const void*>(k_ns_gemm<kApply, SRC>) };
    for (const void* k : kernels)
        if (cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kGemmSmem) != cudaSuccess) return -1;
    const EncodeTiled f = tensor_map_encoder();
    if (!f) return -1;
    Maps gram[2], poly, apply[2];
    for (uint32_t i = 0; i < a.groups; ++i) {
        const Group& g = a.g[i];
        const size_t x = x_bytes(g.mp, g.np), q = a_bytes(g.mp);
        char* const base = a.work + g.work;
        bool ok = encode(f, &poly.first[i], base + 2u * x, g, g.mp, kTile, 8u) && encode(f, &apply[0].first[i], base + 2u * x + q, g, g.mp, kTile, 8u);
        for (uint32_t b = 0; ok && b < 2u; ++b)
            ok = encode(f, &gram[b].first[i], base + b * x, g, g.np, kTile, 8u) && encode(f, &apply[b].second[i], base + b * x, g, g.np, 64u, 16u);
        if (!ok) return -1;
        apply[1].first[i] = apply[0].first[i];
    }
    if (launch_dependent(k_ns_norm<SRC>, dim3(a.blocks), dim3(256), 0, st, a) != cudaSuccess) return -1;
    if (launch_dependent(k_ns_split<SRC>, dim3(a.blocks), dim3(256), 0, st, a) != cudaSuccess) return -1;
    const dim3 pairs(a.pairs < kSms ? a.pairs : kSms), tiles(a.tiles < kSms ? a.tiles : kSms);
    for (uint32_t step = 0; step < a.s.steps; ++step)
        if (launch_dependent(k_ns_gemm<kGram, kF32>, pairs, dim3(kGemmThreads), kGemmSmem, st, a, gram[step & 1u], step) != cudaSuccess ||
            launch_dependent(k_ns_gemm<kPoly, kF32>, pairs, dim3(kGemmThreads), kGemmSmem, st, a, poly, step) != cudaSuccess ||
            launch_dependent(k_ns_gemm<kApply, SRC>, tiles, dim3(kGemmThreads), kGemmSmem, st, a, apply[step & 1u], step) != cudaSuccess)
            return -1;
    return 2 + 3 * static_cast<int>(a.s.steps);
}

int launch_large(cudaStream_t st, uint32_t source, const Args& a)
{
    switch (source) {
        case kF32: return launch_list<kF32>(st, a);
        case kBf16: return launch_list<kBf16>(st, a);
        case kF16: return launch_list<kF16>(st, a);
        default: return launch_list<kMuon>(st, a);
    }
}

}  // namespace ns
}  // namespace evo

// Newton-Schulz iteration of matrices of any size: one launch per product, over all matrices of the list.
//
// k_ns_norm sums the squares of pieces of 128 x 64 elements, k_ns_split writes X in panels (zero in the padding, and so is all
// that is made of it), k_ns_gemm<kGram / kPoly / kApply> is one of the three products of a step.  A block of k_ns_gemm walks over
// 128 x 128 tiles: a thread copies operands into a ring of three stages (64 of the contracted index: two pairs of 128 x 64
// matrices, 64 KB in two TMA boxes), another issues the MMAs, and eight warps take the sums out of tensor memory and
// turn them into fp16 pairs while the next ones are under way (two sets of accumulators).  What the sums are added to (A, X) comes
// through the ring as well.  An MMA of 128 x 128 is bound by its operands' way out of shared memory (104 clocks instead of 64), so the high
// parts of the first operand meet the high and low parts of the second, which lie side by side, in one MMA of 128 x 256.
// A and B are symmetric: tiles on and under the diagonal only, written twice.
// 2048 x 2048, five steps: 0.64 ms, of which 9 us a launch are its start, its first loads and its last tile; the three passes of fp16
// would take 0.31 ms at the rate of a large library product.  256 x 256 and 32 of 512 x 1,408 are mostly starts and ends: 150 us, 1 ms.
#include <algorithm>

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

__device__ __forceinline__ const Group& group_of(const Args& a, uint32_t block)
{
    uint32_t gi = 0;
    while (gi + 1u < a.groups && block >= a.g[gi + 1u].first_block) ++gi;
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
    const Group& g = group_of(a, blockIdx.x);
    const uint32_t pieces = g.mp / kTile * (g.np / kPieceCols), at = blockIdx.x - g.first_block, which = at / pieces, p = at % pieces;
    const uint32_t i0 = p % (g.mp / kTile) * kTile, j0 = p / (g.mp / kTile) * kPieceCols;
    double sum = 0.0;
    for (uint32_t t = threadIdx.x; t < kTile * 8u; t += 256u) {
        uint32_t i, jc;
        piece_place(g, t, i, jc);
        const uint32_t j = j0 + jc * 8u, count = i0 + i < g.m && j < g.n ? min(8u, g.n - j) : 0u;
        float x[8];
        load8<SRC, false, false>(a, in_index(g, which, i0 + i, j), g.tall ? g.in_ld : 1u, count, x);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) sum += static_cast<double>(x[e]) * x[e];
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
    const Group& g = group_of(a, blockIdx.x);
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
        const uint32_t j = j0 + jc * 8u, count = i0 + i < g.m && j < g.n ? min(8u, g.n - j) : 0u;
        load8<SRC, false, true>(a, in_index(g, which, i0 + i, j), g.tall ? g.in_ld : 1u, count, x);
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) x[e] = static_cast<float>(scale * x[e]);
        uint4 hi, lo;
        split8(x, hi, lo);
        const size_t to = (static_cast<size_t>(j0 / 8u + jc) * g.mp + i0 + i) * 16u;
        *reinterpret_cast<uint4*>(x_hi + to) = hi;
        *reinterpret_cast<uint4*>(x_lo + to) = lo;
    }
}

// A tile: which matrix, its place, how far the sum goes.  (Pairs of row blocks, I >= J, are numbered along the rows of the triangle.)
struct Tile { uint32_t gi, which, i0, j0, k; };
template <uint32_t MODE>
__device__ __forceinline__ Tile tile_at(const Args& a, uint32_t at)
{
    Tile t;
    t.gi = 0;
    while (t.gi + 1u < a.groups && at >= (MODE == kApply ? a.g[t.gi + 1u].first_tile : a.g[t.gi + 1u].first_pair)) ++t.gi;
    const Group& g = a.g[t.gi];
    const uint32_t rows = g.mp / kTile, local = at - (MODE == kApply ? g.first_tile : g.first_pair);
    const uint32_t each = MODE == kApply ? rows * ((g.np + kTile - 1u) / kTile) : rows * (rows + 1u) / 2u;
    t.which = g.count == 1u ? 0u : local / each;
    const uint32_t p = local - t.which * each;
    if constexpr (MODE == kApply) {
        t.j0 = p / rows * kTile;
        t.i0 = p % rows * kTile;
        t.k = g.mp;
    } else {
        uint32_t i = static_cast<uint32_t>((sqrtf(8.0f * static_cast<float>(p) + 1.0f) - 1.0f) * 0.5f);
        while (i * (i + 1u) / 2u > p) --i;
        while ((i + 1u) * (i + 2u) / 2u <= p) ++i;
        t.i0 = i * kTile;
        t.j0 = (p - i * (i + 1u) / 2u) * kTile;
        t.k = MODE == kGram ? g.np : g.mp;
    }
    return t;
}

__device__ __forceinline__ uint4 load_shared(uint32_t addr)
{
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// A box of a buffer to shared memory
__device__ __forceinline__ void copy_box(uint32_t dst, const CUtensorMap* map, uint32_t run, uint32_t c1, uint32_t c2, uint32_t which, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.4d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 :: "r"(dst), "l"(map), "r"(bar), "r"(run), "r"(c1), "r"(c2), "r"(which) : "memory");
}

// The operands: X (either of its buffers), A and B as 128 rows by 64 columns, a panel's high parts followed by its low ones; X as the second
// operand of B X, 64 rows by 128 columns, all high parts followed by the low ones
struct Maps { CUtensorMap x[2][kMaxLarge], x_second[2][kMaxLarge], a[kMaxLarge], b[kMaxLarge]; };

struct Shared {
    uint64_t full[kStages], empty[kStages], done[2], taken[2], drain;
    uint32_t slot, limit;
    volatile int abort_flag;
};
// Where a role of a block stands in the ring of stages and among the accumulators
struct Place {
    uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0, filled = 0;
    __device__ __forceinline__ void next_stage() { if (++stage == kStages) { stage = 0; phase ^= 1u; } }
    __device__ __forceinline__ void next_acc() { acc ^= 1u; if (acc == 0u) acc_phase ^= 1u; }
};
__device__ __forceinline__ bool aborted(const Shared& sh) { return __any_sync(0xffffffffu, sh.abort_flag) != 0; }

template <uint32_t MODE>
__device__ __forceinline__ void copy_operands(const Args& a, const Maps& maps, Shared& sh, const Waits& waits, uint32_t ring, Place& at, uint32_t step)
{
    const uint32_t lane = threadIdx.x & 31u, total = MODE == kApply ? a.tiles : a.pairs, cur = step & 1u;
    for (uint32_t tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const Tile t = tile_at<MODE>(a, tile);
        const uint32_t gi = t.gi;
        const bool twice = MODE == kApply || t.i0 != t.j0;
        const CUtensorMap* const first = MODE == kGram ? &maps.x[cur][gi] : MODE == kPoly ? &maps.a[gi] : &maps.b[gi];
        for (uint32_t k = 0; k < t.k + (MODE == kGram ? 0u : 64u); k += 64u) {
            waits.wait(smem_u32(&sh.empty[at.stage]), at.phase ^ 1u);
            if (aborted(sh)) return;
            if (lane == 0) {
                const uint32_t bar = smem_u32(&sh.full[at.stage]), to = ring + at.stage * kStage;
                asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(twice || k >= t.k ? kStage : kStage / 2u) : "memory");
                if (MODE != kGram && k >= t.k) {                // what the sums are added to: the tile of A or X
                    const CUtensorMap* const old = MODE == kPoly ? first : &maps.x[cur][gi];
                    copy_box(to, old, 2u * t.i0, 0u, t.j0 / 8u, t.which, bar);
                    copy_box(to + kStage / 2u, old, 2u * t.i0, 0u, t.j0 / 8u + 8u, t.which, bar);
                } else {
                    copy_box(to, first, 2u * t.i0, 0u, k / 8u, t.which, bar);
                    if (MODE == kApply) copy_box(to + kStage / 2u, &maps.x_second[cur][gi], 2u * k, t.j0 / 8u, 0u, t.which, bar);
                    else if (twice) copy_box(to + kStage / 2u, first, 2u * t.j0, 0u, k / 8u, t.which, bar);
                }
            }
            __syncwarp();
            ++at.filled;
            at.next_stage();
        }
    }
}

template <uint32_t MODE>
__device__ __forceinline__ void issue_products(const Args& a, Shared& sh, const Waits& waits, uint32_t ring, uint32_t tmem, Place& at, uint32_t step)
{
    const uint32_t lane = threadIdx.x & 31u, total = MODE == kApply ? a.tiles : a.pairs;
    const bool drop = MODE == kGram && a.drop && blockIdx.x == 0u && step == 0u;
    for (uint32_t tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const Tile t = tile_at<MODE>(a, tile);
        constexpr uint32_t wide = idesc_f16(128, 256, MODE == kApply), narrow = idesc_f16(128, 128, MODE == kApply);
        for (uint32_t k = 0; k < t.k; k += 64u) {
            const uint32_t d = tmem + at.acc * 2u * kTile, fresh = k % kChunk == 0u;
            const bool ends = (k + 64u) % kChunk == 0u || k + 64u >= t.k;
            if (fresh) waits.wait(smem_u32(&sh.taken[at.acc]), at.acc_phase ^ 1u);
            waits.wait(smem_u32(&sh.full[at.stage]), at.phase);
            tc_fence_after();
            if (aborted(sh)) return;
            if (lane == 0) {
                const uint32_t p = ring + at.stage * kStage, q = MODE == kApply || t.i0 != t.j0 ? p + kStage / 2u : p;
                // K-major: a panel is 128 high and 128 low rows, 4 KB; MN-major: 8 rows are 128 bytes, panels 1 KB apart, the low ones behind the high ones
                constexpr uint32_t ks = MODE == kApply ? 128u : 4096u, ms = MODE == kApply ? 1024u : 128u, hop = 2u * ks / 16u;
                uint64_t ph = umma_smem_desc(p, 4096u, 128u), pl = umma_smem_desc(p + 2048u, 4096u, 128u), qq = umma_smem_desc(q, ks, ms);
#pragma unroll
                for (uint32_t s = 0; s < 4u; ++s) {
                    umma_bf16(d, ph, qq, wide, fresh && s == 0u ? 0u : 1u);      // hi hi' and, in the next 128 columns, hi lo'
                    umma_bf16(d + kTile, pl, qq, narrow, 1u);                    // lo hi'
                    ph += 512u; pl += 512u; qq += hop;
                }
                umma_commit(smem_u32(&sh.empty[at.stage]));
                if (ends && !drop) umma_commit(smem_u32(&sh.done[at.acc]));
            }
            __syncwarp();
            at.next_stage();
            if (ends) at.next_acc();
        }
        if (MODE != kGram) at.next_stage();                       // (that one is for the warps below)
    }
}

template <uint32_t MODE, uint32_t SRC>
__device__ __forceinline__ void turn_sums(const Args& a, Shared& sh, const Waits& waits, uint32_t ring, uint32_t* turn, uint32_t tmem, Place& at, uint32_t step)
{
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u, total = MODE == kApply ? a.tiles : a.pairs, cur = step & 1u;
    const uint32_t quarter = warp & 3u, part = (warp - 2u) >> 2, row = quarter * 32u + lane;      // 64 columns of 32 rows
    const bool last = step + 1u == a.s.steps;
    const float poly_b = a.s.b * a.s.s_b / a.s.s_a, poly_c = a.s.c * a.s.s_b / (a.s.s_a * a.s.s_a), from_bx = 1.0f / a.s.s_b;
    for (uint32_t tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const Tile t = tile_at<MODE>(a, tile);
        const Group& g = a.g[t.gi];
        const uint32_t first_lift = __ldcg(a.lift + g.first_matrix + t.which), lift = lift_at(a.s, first_lift, step);
        const uint32_t next_lift = lift_at(a.s, first_lift, step + 1u);
        const float to_a = power_of_two(-2 * static_cast<int>(lift)) * (a.s.s_a / (a.s.s_x * a.s.s_x));
        const float drop = power_of_two(static_cast<int>(next_lift) - static_cast<int>(lift)), next_a = drop * a.s.a, next_bx = drop * from_bx;
        char* const out = buffer(a, g, t.which, MODE == kGram ? 2u : MODE == kPoly ? 3u : cur ^ 1u);
        const size_t half = static_cast<size_t>(g.mp) * (MODE == kApply ? g.np : g.mp) * 2u;
        const uint32_t width = MODE == kApply ? min(kTile, g.np - t.j0) : kTile;
        float sum[64];                                            // of this thread's row and its warp's 64 columns
        for (uint32_t k = 0; k < t.k; k += kChunk) {
            const float cut = MODE == kGram ? kCut * static_cast<float>(min(kChunk, t.k - k) / 16u) : 0.f;
            waits.wait(smem_u32(&sh.done[at.acc]), at.acc_phase);
            tc_fence_after();
#pragma unroll
            for (int h = 0; h < 4; ++h) {
                uint32_t u[16], v[16];
                const uint32_t from = tmem + at.acc * 2u * kTile + (quarter << 21) + part * 64u + h * 16u;
                tmem_ld16_issue(from, u);
                tmem_ld16_issue(from + kTile, v);
                tmem_ld16_fence(u);
                tmem_ld16_fence(v);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float x = __uint_as_float(u[e]) + fmaf(cut, __uint_as_float(u[e]), __uint_as_float(v[e]));
                    sum[h * 16 + e] = k == 0u ? x : sum[h * 16 + e] + x;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&sh.taken[at.acc]));
            at.next_acc();
            for (uint32_t s = k; s < min(k + kChunk, t.k); s += 64u) at.next_stage();
        }
        const uint32_t old = ring + at.stage * kStage + row * 16u;
        if (MODE != kGram) waits.wait(smem_u32(&sh.full[at.stage]), at.phase);
        // what a wait that ran out leaves is not a number, here and in all that is made of it
        const float sound = sh.abort_flag ? __int_as_float(0x7FC00000) : 1.0f;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t c0 = part * 64u + h * 32u;
            if (c0 < width) {
            uint4 hi[4], lo[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const size_t place = (static_cast<size_t>(t.j0 / 8u + c0 / 8u + c) * g.mp + t.i0 + row) * 16u;
                float x[8];
                if constexpr (MODE == kGram) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = sound * to_a * sum[h * 32 + c * 8 + e];
                } else {
                    join8(load_shared(old + (c0 / 8u + c) * 4096u), load_shared(old + (c0 / 8u + c) * 4096u + 2048u), x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = MODE == kPoly ? fmaf(poly_b, x[e], sound * poly_c * sum[h * 32 + c * 8 + e]) : fmaf(next_a, x[e], sound * next_bx * sum[h * 32 + c * 8 + e]);
                }
                if (MODE == kApply && last) {
                    const float back = power_of_two(-static_cast<int>(next_lift)) / a.s.s_x;
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e) turn[(c * 8u + e) * 33u + lane] = __float_as_uint(x[e] * back);
                } else {
                    split8(x, hi[c], lo[c]);
                    *reinterpret_cast<uint4*>(out + place) = hi[c];
                    *reinterpret_cast<uint4*>(out + half + place) = lo[c];
                }
            }
            if (MODE == kApply && last) {
                // neighbouring lanes are neighbours in memory: rows of the source where the matrix lies as it is, columns where it is transposed
                __syncwarp();
                const uint32_t i0 = t.i0 + quarter * 32u, j0 = t.j0 + c0;
                const uint32_t left = g.tall ? (g.n > j0 ? g.n - j0 : 0u) : (g.m > i0 ? g.m - i0 : 0u);
                const uint32_t count = (g.tall ? i0 + lane < g.m : j0 + lane < g.n) ? min(32u, left) : 0u;
                const uint64_t to = g.tall ? out_index(g, t.which, i0 + lane, j0) : out_index(g, t.which, i0, j0 + lane);
                const uint32_t from = g.tall ? lane : lane * 33u, hop = g.tall ? 33u : 1u;
                for (uint32_t e0 = 0; e0 < count; e0 += 8u) {
                    float centre[8];                             // all asked for before the first store (Muon, 784-1536-1536-1000: 144 us a launch without, 82 with)
                    if constexpr (SRC == kMuon)
#pragma unroll
                        for (uint32_t e = 0; e < 8u; ++e) centre[e] = e0 + e < count ? a.c_in[to + static_cast<uint64_t>(e0 + e) * g.out_ld] : 0.f;
#pragma unroll
                    for (uint32_t e = 0; e < 8u; ++e)
                        if (e0 + e < count) {
                            const uint64_t at_e = to + static_cast<uint64_t>(e0 + e) * g.out_ld;
                            const float x = __uint_as_float(turn[from + (e0 + e) * hop]);
                            if constexpr (SRC == kMuon) static_cast<float*>(a.out)[at_e] = fmaf(g.gain, x, a.s.keep * centre[e]);
                            else store<SRC, false>(a, at_e, x, g.gain);
                        }
                }
                __syncwarp();
            }
            if (MODE != kApply && t.i0 != t.j0) {             // the same above the diagonal: thread `lane` takes column c0 + lane as its row
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint32_t p[4] = { hi[c].x, hi[c].y, hi[c].z, hi[c].w }, q[4] = { lo[c].x, lo[c].y, lo[c].z, lo[c].w };
#pragma unroll
                    for (uint32_t e = 0; e < 4u; ++e) {
                        turn[(c * 8u + 2u * e) * 33u + lane] = __byte_perm(p[e], q[e], 0x5410);
                        turn[(c * 8u + 2u * e + 1u) * 33u + lane] = __byte_perm(p[e], q[e], 0x7632);
                    }
                }
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) {
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
        if (MODE != kGram) {                                      // the ring may have the stage again
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (warp == 2u && lane == 0u) mbar_arrive(smem_u32(&sh.empty[at.stage]));
            at.next_stage();
        }
    }
}

template <uint32_t MODE, uint32_t SRC>
__global__ void __launch_bounds__(kGemmThreads, 1) k_ns_gemm(const __grid_constant__ Args a, const __grid_constant__ Maps maps, uint32_t step)
{
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ __align__(8) Shared sh;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    if (tid == 0) {
        for (uint32_t s = 0; s < kStages; ++s) { mbar_init(smem_u32(&sh.full[s]), 1); mbar_init(smem_u32(&sh.empty[s]), 1); }
        for (uint32_t b = 0; b < 2u; ++b) { mbar_init(smem_u32(&sh.done[b]), 1); mbar_init(smem_u32(&sh.taken[b]), 8); }
        mbar_init(smem_u32(&sh.drain), 1);
        mbar_init_fence();
        sh.limit = a.wait_log2;
        sh.abort_flag = 0;
    }
    dep_wait();
    dep_trigger();
    if (a.skip && *a.skip == 0.0) return;
    if (warp == 1) tmem_alloc(smem_u32(&sh.slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.slot, ring = smem_u32(smem);
    const Waits waits{ &sh.abort_flag, &sh.limit, a.sticky };
    uint32_t* const turn = reinterpret_cast<uint32_t*>(smem + kStages * kStage) + (warp - 2u) * 32u * 33u;
    Place at;
    if (warp == 0) copy_operands<MODE>(a, maps, sh, waits, ring, at, step);
    else if (warp == 1) issue_products<MODE>(a, sh, waits, ring, tmem, at, step);
    else turn_sums<MODE, SRC>(a, sh, waits, ring, turn, tmem, at, step);
    if (warp == 0 && aborted(sh))                                // nothing may land after the block has gone
        for (uint32_t s = 0; s < min(at.filled, kStages); ++s) {
            const uint32_t nth = at.filled - 1u - s;
            mbar_wait_bounded(smem_u32(&sh.full[nth % kStages]), nth / kStages & 1u, &sh.limit);
        }
    if (warp == 1 && aborted(sh)) {                              // nor may an MMA write after its tensor memory is freed
        if (lane == 0) umma_commit(smem_u32(&sh.drain));
        __syncwarp();
        mbar_wait_bounded(smem_u32(&sh.drain), 0u, &sh.limit);
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// A buffer of `cols` columns of all matrices of a group.  As a first operand: runs of 128 rows (8-byte elements), high and low parts, 8 panels; as
// the second operand of B X: runs of 64 rows, 16 panels, high and low parts.
static bool encode(EncodeTiled f, CUtensorMap* map, char* base, const Group& g, uint32_t cols, bool second)
{
    const cuuint64_t run = 2ull * g.mp, panel = 16ull * g.mp, half = panel * (cols / 8u), all = large_bytes(g.mp, g.np), panels = cols / 8u;
    const cuuint64_t dims[4] = { run, second ? panels : 2u, second ? 2u : panels, g.count };
    const cuuint64_t strides[3] = { second ? panel : half, second ? half : panel, all };
    const cuuint32_t box[4] = { second ? 128u : 256u, second ? 16u : 2u, second ? 2u : 8u, 1u }, steps[4] = { 1u, 1u, 1u, 1u };
    return f(map, CU_TENSOR_MAP_DATA_TYPE_INT64, 4, base, dims, strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_NONE,
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
    Maps maps;
    for (uint32_t i = 0; i < a.groups; ++i) {
        const Group& g = a.g[i];
        const size_t x = x_bytes(g.mp, g.np), q = a_bytes(g.mp);
        char* const base = a.work + g.work;
        bool ok = encode(f, &maps.a[i], base + 2u * x, g, g.mp, false) && encode(f, &maps.b[i], base + 2u * x + q, g, g.mp, false);
        for (uint32_t b = 0; ok && b < 2u; ++b)
            ok = encode(f, &maps.x[b][i], base + b * x, g, g.np, false) && encode(f, &maps.x_second[b][i], base + b * x, g, g.np, true);
        if (!ok) return -1;
    }
    if (launch_dependent(k_ns_norm<SRC>, dim3(a.blocks), dim3(256), 0, st, a) != cudaSuccess) return -1;
    if (launch_dependent(k_ns_split<SRC>, dim3(a.blocks), dim3(256), 0, st, a) != cudaSuccess) return -1;
    const dim3 pairs(std::min(a.pairs, kSms)), tiles(std::min(a.tiles, kSms));
    for (uint32_t step = 0; step < a.s.steps; ++step)
        if (launch_dependent(k_ns_gemm<kGram, kF32>, pairs, dim3(kGemmThreads), kGemmSmem, st, a, maps, step) != cudaSuccess ||
            launch_dependent(k_ns_gemm<kPoly, kF32>, pairs, dim3(kGemmThreads), kGemmSmem, st, a, maps, step) != cudaSuccess ||
            launch_dependent(k_ns_gemm<kApply, SRC>, tiles, dim3(kGemmThreads), kGemmSmem, st, a, maps, step) != cudaSuccess)
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

// Gradients of the products grouped by member on tcgen05.
//
// dW_g = scale sum_r dz[r] x[r]' over the group's rows: both operands lie with the contracted index, the rows, outermost, so TMA brings boxes of 64 columns x 64 (or 16)
// rows as they are and the MMA takes both as MN-major; nothing is transposed.  A tile is 128 outputs x up to 256 inputs; blocks stay and walk over (set, split, 128 outputs,
// inputs), the inputs of 128 outputs side by side, so that dz is read from L2.  One thread copies, one issues the MMAs, eight warps take the sums of one
// tile out of tensor memory, through shared memory so that rows of a tile are written whole, while the next tile's are under way.  The last rows of a group end inside a box: the
// rows behind them, another group's, are overwritten with zeros in shared memory (both operands: theirs may be infinities).
// dx goes through the forward's kernel with the weights' rows as the contracted index.
// 8,192 rows of bf16 of 4 groups, 4,096 -> 4,096: dW 232 us, 1,185 TFLOP/s, dx 209, 1,315; the MMAs alone, without copies and stores, take 210 either way.  Of 32 ragged groups,
// 1,024 -> 4,096: dW 104 us, dx 92 (3.7 us a tile of four times 64 rows, of which the MMAs need 1.2 and the result's way out 1.7).  Pairs of blocks on 256 x 256 tiles took 4 % less and
// are not kept.
//
// dz = dy act'(z) is laid out first where it is not dy itself, scale left to the end: fp32 as three bf16 parts like the rows (and weights), of 16-bit types with
// tanh as two parts of the type (rounded once it would be off by as much as the result's own rounding), of fp16 the second 2^11 times as large (kSecondUp); relu's is dy or 0.
#include <cmath>

#include "grouped_gradient.h"
#include "grouped_tc.cuh"

namespace evo {
namespace {

constexpr uint32_t kMostStages = 8, kThreads = 352, kMostColumns = 256;
constexpr uint32_t kRing = 192u * 1024u, kStaging = 8u * 4096u, kSmem = kRing + kStaging + 1024u;

// The tensor core cuts its sums off (2.7e-5 of 4,096 numbers of one sign).  fp32: the last pass, of the large products, is taken out every 8 chunks of 64 rows and added up in
// fp32; 16-bit types: every 128.
constexpr uint32_t kSegment = 8, kLongSegment = 128;

// What a stage waits for before it is filled anew: its MMAs, and the warp that clears rows, which looks at every stage.  (With the MMAs alone that warp could be overtaken by a
// turn of the ring, whose phase a barrier's parity does not tell from the one it waits for.)
constexpr uint32_t kEmptyArrivals = 2;

struct DwArgs {
    GradientArgs a;
    CUtensorMap dz[2], x[2], dw;                             // boxes of 16 and of 64 rows; of 32 outputs x 128 bytes
    uint32_t all, sets, splits, out_tiles, in_tiles, columns, stages;
    uint32_t passes, pitch_dz, pitch_x;
    Waits waits;
    float* part;                                             // splits > 1: [splits][sets][n_out][n_in]
    float* sums;                                             // 16-bit types: room for the sums of long sets, [first row / long_rows][n_out][n_in]
    uint32_t long_rows, pieces, boxes;                       // pieces: 16-byte stores are possible; boxes: TMA can store the result
};

// A tile's set, and what it is of the set: the offsets are asked for a tile ahead and looked at when it is its turn.
struct Item { uint32_t o0, i0, columns, set, split; uint64_t row, end; };
struct Asked { uint32_t o0, i0, set, split; int64_t from, to; };
__device__ __forceinline__ Asked ask_for(const DwArgs& p, uint32_t at)
{
    Asked t;
    t.i0 = at % p.in_tiles * p.columns; at /= p.in_tiles;
    t.o0 = at % p.out_tiles * 128u; at /= p.out_tiles;
    t.split = at % p.splits; t.set = at / p.splits;
    const GroupedArgs& f = p.a.f;
    const uint32_t behind = p.all ? f.groups : t.set + 1u;
    if (f.wide_offsets) {
        t.from = __ldg(static_cast<const long long*>(f.offsets) + t.set);
        t.to = __ldg(static_cast<const long long*>(f.offsets) + behind);
    } else {
        t.from = __ldg(static_cast<const int*>(f.offsets) + t.set);
        t.to = __ldg(static_cast<const int*>(f.offsets) + behind);
    }
    return t;
}
__device__ __forceinline__ Item item_of(const DwArgs& p, const Asked& a)
{
    Item t;
    t.o0 = a.o0; t.i0 = a.i0; t.set = a.set; t.split = a.split;
    t.columns = min(p.columns, (p.a.f.n_in - t.i0 + 15u) / 16u * 16u);
    split_rows(p.a, a.from, a.to, a.split, p.splits, &t.row, &t.end);
    if (t.end < t.row) t.end = t.row;
    return t;
}

template <typename T, typename O>
__global__ void __launch_bounds__(kThreads, 1) k_weights_tc(const __grid_constant__ DwArgs p)
{
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t full[kMostStages], empty[kMostStages], cleared[kMostStages], done[2], taken[2], drain;
    __shared__ uint32_t slot, limit, longest;
    __shared__ volatile int abort_flag;
    constexpr bool kFloat = std::is_same<O, float>::value;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    const uint32_t smem = (smem_u32(raw) + 1023u) / 1024u * 1024u;
    if (tid == 0) {
        for (uint32_t s = 0; s < kMostStages; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), kEmptyArrivals); mbar_init(smem_u32(&cleared[s]), 1); }
        for (uint32_t b = 0; b < 2u; ++b) { mbar_init(smem_u32(&done[b]), 1); mbar_init(smem_u32(&taken[b]), 8); }
        mbar_init(smem_u32(&drain), 1);
        mbar_init_fence();
        limit = p.waits.cycles_log2;
        longest = kLongestWait;
        abort_flag = 0;
    }
    dep_begin(p.a);
    if (warp == 1) tmem_alloc(smem_u32(&slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = slot, stages = p.stages, boxes = (p.columns + 63u) / 64u, stage_bytes = (2u + boxes) * 8192u;
    const uint32_t items = p.sets * p.splits * p.out_tiles * p.in_tiles;
    // false: it, or another wait of the block, ran out
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(smem_u32(bar), parity)) return true;
        if (abort_flag) return false;
        if (mbar_wait_bounded(smem_u32(bar), parity, &limit)) return true;
        abort_flag = 1;
        return false;
    };
    auto all_of = [](bool fine) { return __all_sync(0xffffffffu, fine) != 0; };
    // fp16 in two parts: the step at which the sums of second parts end (0: there are none), the first of whose MMAs takes the sum so far down
    auto turn_of = [&](uint32_t chunks) { return std::is_same<T, __half>::value && p.passes == 2u ? chunks : 0u; };
    auto chunks_of = [&](const Item& t) { return static_cast<uint32_t>((t.end - t.row + 63u) / 64u); };
    // the step behind the part of a sum that begins at step k
    auto part_end = [&](uint32_t k, uint32_t chunks) {
        const uint32_t steps = chunks * p.passes;
        return kFloat ? min(steps, max(k, steps - chunks) + kSegment) : min(steps, k + kLongSegment);
    };
    uint32_t stage = 0, phase = 0, acc = 0, acc_phase = 0, filled = 0;

    if (warp == 0) {
        bool fine = true;
        Asked next = blockIdx.x < items ? ask_for(p, blockIdx.x) : Asked{};
        for (uint32_t at = blockIdx.x; at < items; at += gridDim.x) {
            const Item t = item_of(p, next);
            if (at + gridDim.x < items) next = ask_for(p, at + gridDim.x);
            const uint32_t chunks = chunks_of(t), steps = chunks * p.passes, across = (t.columns + 63u) / 64u, high = t.o0 + 64u < p.a.f.n_out ? 2u : 1u;
            uint32_t pass = 0, chunk = 0;
            for (uint32_t k = 0; k < steps; ++k) {
                fine = all_of(wait(&empty[stage], phase ^ 1u));
                if (!fine) break;
                const uint32_t bar = smem_u32(&full[stage]), to = smem + stage * stage_bytes;
                const uint64_t row = t.row + chunk * 64ull;
                const uint32_t box = t.end - row > 16u ? 1u : 0u, bytes = box ? 8192u : 2048u;
                if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"((high + across) * bytes) : "memory");
                __syncwarp();
                // a box a lane: those of dz first
                if (lane < 2u + across && (lane >= 2u || lane < high)) {
                    const bool is_x = lane >= 2u;
                    uint32_t c = is_x ? t.i0 + 64u * (lane - 2u) : t.o0 + 64u * lane;
                    if (p.passes == 2u) c += is_x ? 0u : kPartTwo[pass] * p.pitch_dz;
                    else if (p.passes > 1u) c += is_x ? kPartX[pass] * p.pitch_x : kPartW[pass] * p.pitch_dz;
                    copy2(to + lane * bytes, (is_x ? p.x : p.dz) + box, c, static_cast<uint32_t>(row), bar);
                }
                if (++chunk == chunks) { chunk = 0; ++pass; }
                __syncwarp();
                ++filled;
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
            if (!fine) break;
        }
        if (!fine)                                           // nothing may land after the block has gone
            for (uint32_t s = 0; s < min(filled, stages); ++s) {
                const uint32_t nth = filled - 1u - s;
                mbar_wait_bounded(smem_u32(&full[nth % stages]), nth / stages & 1u, &longest);
            }
    } else if (warp == 1) {
        if (lane == 0) {                                     // (one thread: what it does between two MMAs is time that the tensor core has nothing to do)
            bool fine = true;
            uint32_t was_cleared = 0;                        // a bit a stage: the phase of its barrier
            Asked next = blockIdx.x < items ? ask_for(p, blockIdx.x) : Asked{};
            for (uint32_t at = blockIdx.x; at < items && fine; at += gridDim.x) {
                const Item t = item_of(p, next);
                if (at + gridDim.x < items) next = ask_for(p, at + gridDim.x);
                const uint32_t chunks = chunks_of(t), steps = chunks * p.passes, turn = turn_of(chunks), id = idesc<T, true, true>(t.columns);
                const uint32_t rest = static_cast<uint32_t>(t.end - t.row) - (chunks - 1u) * 64u;      // rows of the last chunk
                uint32_t chunk = 0;
                for (uint32_t k = 0; k < steps && fine;) {
                    const uint32_t d = tmem + acc * kMostColumns, first = k, end = part_end(k, chunks);
                    fine = wait(&taken[acc], acc_phase ^ 1u);
                    tc_fence_after();
                    for (; k < end && fine; ++k) {
                        const bool down = k == turn && k != first;
                        auto multiply = [&](uint64_t a, uint64_t b, uint32_t s) {
                            if (std::is_same<T, __half>::value && s == 0u && down) umma_scaling_down<kSecondUp>(d, a, b, id);
                            else umma_bf16(d, a + s * 128u, b + s * 128u, id, k - first + s != 0u);
                        };
                        const uint32_t at_stage = smem + stage * stage_bytes;
                        if (chunk + 1u < chunks || rest == 64u) {
                            fine = wait(&full[stage], phase);
                            const uint64_t a = desc_sw128_mn(at_stage, 8192u), b = desc_sw128_mn(at_stage + 16384u, 8192u);
#pragma unroll
                            for (uint32_t s = 0; s < 4u; ++s) multiply(a, b, s);
                        } else {
                            if (rest & 15u) {
                                fine = wait(&cleared[stage], was_cleared >> stage & 1u);
                                was_cleared ^= 1u << stage;
                            } else {
                                fine = wait(&full[stage], phase);
                            }
                            const uint32_t bytes = rest > 16u ? 8192u : 2048u;
                            const uint64_t a = desc_sw128_mn(at_stage, bytes), b = desc_sw128_mn(at_stage + 2u * bytes, bytes);
                            for (uint32_t s = 0; s * 16u < rest; ++s) multiply(a, b, s);
                        }
#ifdef EVO_DEBUG
                        if (!p.waits.drop || at != 0u || k != 0u)
#endif
                        umma_commit(smem_u32(&empty[stage]));
                        if (++chunk == chunks) chunk = 0;
                        if (++stage == stages) { stage = 0; phase ^= 1u; }
                    }
                    umma_commit(smem_u32(&done[acc]));
                    acc ^= 1u;
                    if (acc == 0u) acc_phase ^= 1u;
                }
            }
            if (!fine) {                                     // no MMA may write after its tensor memory is freed
                umma_commit(smem_u32(&drain));
                mbar_wait_bounded(smem_u32(&drain), 0u, &longest);
            }
        }
        __syncwarp();
    } else if (warp == 10) {
        // Rows of the last chunk's boxes that are not the set's, as far as the MMAs reach, become zeros (rows of a box are 128 bytes, whatever the swizzle).
        bool fine = true;
        Asked next = blockIdx.x < items ? ask_for(p, blockIdx.x) : Asked{};
        for (uint32_t at = blockIdx.x; at < items && fine; at += gridDim.x) {
            const Item t = item_of(p, next);
            if (at + gridDim.x < items) next = ask_for(p, at + gridDim.x);
            const uint32_t chunks = chunks_of(t), across = (t.columns + 63u) / 64u, rest = static_cast<uint32_t>(t.end - t.row) - (chunks - 1u) * 64u;
            const uint32_t bytes = rest > 16u ? 8192u : 2048u, upto = (rest + 15u) / 16u * 16u;
            uint32_t chunk = 0;
            for (uint32_t k = 0; k < chunks * p.passes && fine; ++k) {
                fine = all_of(wait(&full[stage], phase));
                if (!fine) break;
                const bool last = ++chunk == chunks;
                if (last) chunk = 0;
                if (last && (rest & 15u)) {
                    for (uint32_t b = 0; b < 2u + across; ++b)
                        for (uint32_t row = rest + (lane >> 3); row < upto; row += 4u)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" :: "r"(smem + stage * stage_bytes + b * bytes + row * 128u + (lane & 7u) * 16u), "r"(0u) : "memory");
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&cleared[stage]));
                }
                if (lane == 0) mbar_arrive(smem_u32(&empty[stage]));
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
        }
    } else {
        const uint32_t quarter = warp & 3u, half = (warp - 2u) >> 2, n_in = p.a.f.n_in, n_out = p.a.f.n_out;
        const uint32_t staging = smem + kRing + (warp - 2u) * 4096u;
        Asked next = blockIdx.x < items ? ask_for(p, blockIdx.x) : Asked{};
        for (uint32_t at = blockIdx.x; at < items; at += gridDim.x) {
            const Item t = item_of(p, next);
            if (at + gridDim.x < items) next = ask_for(p, at + gridDim.x);
            const uint32_t chunks = chunks_of(t), steps = chunks * p.passes, o0 = t.o0 + quarter * 32u;
            // where the result goes, and where sums of several parts are kept meanwhile
            O* const to = static_cast<O*>(p.a.dw) + static_cast<uint64_t>(t.set) * p.a.stride_dw;
            float* sums = nullptr;
            uint64_t ld_sums = n_in;
            if (p.splits > 1u) sums = p.part + (static_cast<uint64_t>(t.split) * p.sets + t.set) * n_out * n_in;
            else if constexpr (kFloat) { sums = reinterpret_cast<float*>(to); ld_sums = p.a.ld_dw; }
            else if (steps > kLongSegment) sums = p.sums + t.row / p.long_rows * n_out * n_in;
            for (uint32_t first = 0, end = 0; first == 0u || end < steps; first = end) {
                if (steps) {
                    end = part_end(first, chunks);
                    wait(&done[acc], acc_phase);
                    __syncwarp();
                    tc_fence_after();
                }
                const float scale = abort_flag ? __int_as_float(0x7FC00000) : p.a.f.scale;
                const bool last = end >= steps;
                if (p.boxes && first == 0u && last) {        // a sum in one part goes out as TMA has it: 128 bytes of 32 outputs
                    constexpr uint32_t kWide = 128u / sizeof(O);
                    for (uint32_t c = half * kWide; c < t.columns; c += 2u * kWide) {
                        uint32_t u[kWide / 32u][4][8];
                        if (steps) {
#pragma unroll
                            for (uint32_t i = 0; i < kWide / 32u; ++i) tmem_ld32_issue(tmem + acc * kMostColumns + (quarter << 21) + c + 32u * i, u[i]);
#pragma unroll
                            for (uint32_t i = 0; i < kWide / 32u; ++i) tmem_ld8x4_fence(u[i][0], u[i][1], u[i][2], u[i][3]);
                        } else {
#pragma unroll
                            for (uint32_t i = 0; i < kWide; ++i) u[i / 32u][i / 8u % 4u][i % 8u] = 0u;
                        }
                        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");      // (the box before has left)
                        __syncwarp();
#pragma unroll
                        for (uint32_t i = 0; i < 8u; ++i) {
                            uint32_t w[4];
#pragma unroll
                            for (uint32_t e = 0; e < 4u; ++e) {
                                if constexpr (kFloat) {
                                    w[e] = __float_as_uint(scale * __uint_as_float(u[0][i / 2u][i % 2u * 4u + e]));
                                } else {
                                    const uint32_t k = i * 8u + 2u * e;
                                    const float x = scale * __uint_as_float(u[k / 32u][k / 8u % 4u][k % 8u]), y = scale * __uint_as_float(u[k / 32u][k / 8u % 4u][k % 8u + 1u]);
                                    if constexpr (std::is_same<O, __half>::value) { const __half2 h = __floats2half2_rn(x, y); w[e] = *reinterpret_cast<const uint32_t*>(&h); }
                                    else w[e] = pack_bf16(x, y);
                                }
                            }
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(staging + lane * 128u + ((i ^ lane) & 7u) * 16u), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3])
                                         : "memory");
                        }
                        fence_async_smem();
                        __syncwarp();
                        if (lane == 0 && o0 < n_out) {
                            asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                                         :: "l"(&p.dw), "r"(staging), "r"(t.i0 + c), "r"(o0), "r"(t.set) : "memory");
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    }
                } else for (uint32_t c = half * 32u; c < t.columns; c += 64u) {
                    uint32_t u[4][8];
                    if (steps) {
                        tmem_ld32_issue(tmem + acc * kMostColumns + (quarter << 21) + c, u);
                        tmem_ld8x4_fence(u[0], u[1], u[2], u[3]);
                    } else {
#pragma unroll
                        for (uint32_t i = 0; i < 32u; ++i) u[i / 8u][i % 8u] = 0u;
                    }
                    if (std::is_same<T, __half>::value && end <= turn_of(chunks))          // (a part of second numbers alone)
#pragma unroll
                        for (uint32_t i = 0; i < 32u; ++i) u[i / 8u][i % 8u] = __float_as_uint(kDown<T> * __uint_as_float(u[i / 8u][i % 8u]));
                    // a row of 32 numbers a lane, its eight pieces of 16 bytes in an order that the lane's number turns: no bank is hit twice
                    if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    __syncwarp();
#pragma unroll
                    for (uint32_t i = 0; i < 8u; ++i)
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(staging + lane * 128u + ((i ^ lane) & 7u) * 16u), "r"(u[i / 2u][i % 2u * 4u]),
                                     "r"(u[i / 2u][i % 2u * 4u + 1u]), "r"(u[i / 2u][i % 2u * 4u + 2u]), "r"(u[i / 2u][i % 2u * 4u + 3u]) : "memory");
                    __syncwarp();
                    const uint32_t column = t.i0 + c;
                    if (p.pieces) {                          // eight lanes a row, four rows at a time
                        const uint32_t k = column + (lane & 7u) * 4u, row = o0 + (lane >> 3), outputs = row < n_out && k < n_in ? n_out - row : 0u;
                        float4 v[8];
#pragma unroll
                        for (uint32_t i = 0; i < 8u; ++i)
                            asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v[i].x), "=f"(v[i].y), "=f"(v[i].z), "=f"(v[i].w)
                                         : "r"(staging + (i * 4u + (lane >> 3)) * 128u + ((lane ^ (i * 4u + (lane >> 3))) & 7u) * 16u));
                        if (sums) {
                            float* const sum_at = sums + row * ld_sums + k;
                            if (first) {
                                float4 w[8];
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i)
                                    if (4u * i < outputs) w[i] = *reinterpret_cast<const float4*>(sum_at + 4u * i * ld_sums);
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i)
                                    if (4u * i < outputs) { v[i].x += w[i].x; v[i].y += w[i].y; v[i].z += w[i].z; v[i].w += w[i].w; }
                            }
                            if (!last || p.splits > 1u) {
                                const float factor = last ? scale : 1.f;
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i)
                                    if (4u * i < outputs)
                                        *reinterpret_cast<float4*>(sum_at + 4u * i * ld_sums) = make_float4(factor * v[i].x, factor * v[i].y, factor * v[i].z, factor * v[i].w);
                                continue;
                            }
                        }
                        O* at = to + row * p.a.ld_dw + k;
#pragma unroll
                        for (uint32_t i = 0; i < 8u; ++i) {
                            if (4u * i < outputs) {
                                const float4 x = make_float4(scale * v[i].x, scale * v[i].y, scale * v[i].z, scale * v[i].w);
                                if constexpr (kFloat) {
                                    *reinterpret_cast<float4*>(at) = x;
                                } else if constexpr (std::is_same<O, __half>::value) {
                                    const __half2 a = __floats2half2_rn(x.x, x.y), b = __floats2half2_rn(x.z, x.w);
                                    *reinterpret_cast<uint2*>(at) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
                                } else {
                                    *reinterpret_cast<uint2*>(at) = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
                                }
                            }
                            at += 4u * p.a.ld_dw;
                        }
                    } else {                                 // a number a lane, row by row, eight rows on their way together
                        const uint32_t k = column + lane;
                        const bool live = k < n_in;
                        const uint32_t outputs = o0 < n_out && live ? min(32u, n_out - o0) : 0u;
                        auto number = [&](uint32_t r) {
                            float v;
                            asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(staging + r * 128u + ((lane >> 2 ^ r) & 7u) * 16u + (lane & 3u) * 4u));
                            return v;
                        };
                        if (!sums || (kFloat && p.splits == 1u && first == 0u && last)) {
                            const float factor = scale;
                            O* at = to + o0 * p.a.ld_dw + k;
                            for (uint32_t r0 = 0; r0 < 32u; r0 += 8u) {
                                float v[8];
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i) v[i] = factor * number(r0 + i);
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i) {
                                    if (r0 + i < outputs) {
                                        if constexpr (kFloat) *at = v[i];
                                        else if constexpr (std::is_same<O, __half>::value) *at = __float2half_rn(v[i]);
                                        else *at = __float2bfloat16_rn(v[i]);
                                    }
                                    at += p.a.ld_dw;
                                }
                            }
                        } else {
                            float* sum_at = sums + o0 * ld_sums + k;
                            for (uint32_t r0 = 0; r0 < 32u; r0 += 8u) {
                                float v[8];
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i) {
                                    v[i] = number(r0 + i);
                                    if (first && r0 + i < outputs) v[i] += sum_at[(r0 + i) * ld_sums];
                                }
#pragma unroll
                                for (uint32_t i = 0; i < 8u; ++i) {
                                    if (r0 + i >= outputs) continue;
                                    if (!last) sum_at[(r0 + i) * ld_sums] = v[i];
                                    else if (p.splits > 1u) sum_at[(r0 + i) * ld_sums] = scale * v[i];
                                    else if constexpr (kFloat) to[(o0 + r0 + i) * p.a.ld_dw + k] = scale * v[i];
                                    else if constexpr (std::is_same<O, __half>::value) to[(o0 + r0 + i) * p.a.ld_dw + k] = __float2half_rn(scale * v[i]);
                                    else to[(o0 + r0 + i) * p.a.ld_dw + k] = __float2bfloat16_rn(scale * v[i]);
                                }
                            }
                        }
                    }
                }
                if (!steps) break;
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&taken[acc]));
                acc ^= 1u;
                if (acc == 0u) acc_phase ^= 1u;
            }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
    dep_end(p.a);
}

// dz / scale of every row, in parts `pitch` apart that are filled up with zeros; 256 columns of a row a warp.
template <typename T, uint32_t PARTS>
__global__ void __launch_bounds__(256) k_lay_dz(const __grid_constant__ GradientArgs a, uint16_t* __restrict__ to, uint32_t pitch)
{
    dep_wait();
    dep_trigger();
    const uint32_t across = (pitch + 255u) / 256u, at = blockIdx.x * 8u + (threadIdx.x >> 5), first = at % across * 256u + (threadIdx.x & 31u);
    const uint64_t row = at / across;
    if (row >= a.f.rows) return;
    const T* const dy = static_cast<const T*>(a.dy) + row * a.ld_dy;
    const T* const y = static_cast<const T*>(a.f.y) + row * a.f.ld_y;
    const bool act = a.f.activation != EVO_ACT_NONE;
    uint16_t* const dst = to + row * PARTS * pitch;
    T d[8], z[8];
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i)
        if (first + 32u * i < a.f.n_out) {
            d[i] = dy[first + 32u * i];
            if (act) z[i] = y[first + 32u * i];
        }
#pragma unroll
    for (uint32_t i = 0; i < 8u; ++i) {
        const uint32_t k = first + 32u * i;
        if (k >= pitch) break;
        const bool live = k < a.f.n_out;
        if constexpr (std::is_same<T, float>::value) {
            three_parts(live ? dz_unit(a, d[i], act ? z[i] : 0.f) : 0.f, dst + k, dst + pitch + k, dst + 2u * pitch + k);
        } else {
            auto number = [](T x) { if constexpr (std::is_same<T, __half>::value) return __half2float(x); else return __bfloat162float(x); };
            auto rounded = [](float x) { if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x); else return __float2bfloat16_rn(x); };
            const float x = live ? dz_unit(a, number(d[i]), act ? number(z[i]) : 0.f) : 0.f;
            const T whole = rounded(x);
            reinterpret_cast<T*>(dst)[k] = whole;
            if constexpr (PARTS == 2u) reinterpret_cast<T*>(dst)[pitch + k] = rounded(isfinite(number(whole)) ? kUp<T> * (x - number(whole)) : 0.f);      // (an infinity has no second part)
        }
    }
}

bool addressable(const void* p, uint64_t ld, uint64_t rows) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0u && (ld & 7u) == 0u && ld < (1ull << 38) && rows < (1ull << 31); }
uint64_t padded(uint64_t bytes) { return (bytes + 255u) / 256u * 256u; }

}  // namespace

TcPlan grouped_gradient_tc_plan(uint32_t type, const GradientArgs& a, bool dx, bool dw, uint32_t splits, bool any_address)
{
    TcPlan p;
    const GroupedArgs& f = a.f;
    const bool fp32 = type == EVO_F32, tanh = f.activation == EVO_ACT_TANH;
    p.dx = dx; p.dw = dw;
    p.dz_parts = fp32 ? 3u : tanh ? 2u : 1u;
    p.lay_dz = (dx || dw) && (fp32 || f.activation != EVO_ACT_NONE || any_address || !addressable(a.dy, a.ld_dy, f.rows));
    p.lay_x = dw && (fp32 || any_address || !addressable(f.x, f.ld_x, f.rows));
    p.lay_w = dx && (fp32 || any_address || !addressable(f.w, f.ld_w | f.stride_w, 1u));
    p.pitch_dz = (f.n_out + 63u) / 64u * 64u;
    p.pitch = grouped_tc_pitch(type, f.n_in);
    const uint64_t parts = fp32 ? 3u : 1u, sets = f.groups > 1u && f.stride_w == 0u ? 1u : f.groups, steps = dw && !fp32 && splits == 1u ? p.dz_parts : 0u;
    p.long_rows = 64u * kLongSegment / p.dz_parts;
    p.dz_bytes = p.lay_dz ? padded(2ull * f.rows * p.dz_parts * p.pitch_dz) : 0u;
    p.x_bytes = p.lay_x ? padded(2ull * f.rows * parts * p.pitch) : 0u;
    p.w_bytes = p.lay_w ? padded(2ull * sets * f.n_out * parts * p.pitch) : 0u;
    p.sum_bytes = steps && f.rows > p.long_rows ? padded(4ull * (f.rows / p.long_rows + 1u) * f.n_out * f.n_in) : 0u;
    return p;
}

int launch_grouped_gradient_tc(cudaStream_t st, uint32_t type, const GradientArgs& a, const TcPlan& plan, uint32_t splits, float* part, void* work)
{
    const GroupedArgs& f = a.f;
    uint8_t* at = static_cast<uint8_t*>(work);
    const bool fp32 = type == EVO_F32;
    const uint32_t passes = fp32 ? 6u : plan.dz_parts;
    int launches = 0;
    const void* dz = a.dy; const void* x = f.x; const void* w = f.w;
    uint64_t ld_dz = a.ld_dy, span_dz = f.n_out, ld_x = f.ld_x, span_x = f.n_in, ld_w = f.ld_w, span_w = f.n_in, stride_w = f.stride_w;
    if (plan.lay_dz) {
        const uint64_t blocks = (f.rows * ((plan.pitch_dz + 255u) / 256u) + 7u) / 8u;
        if (blocks > 0x0FFFFFFFull) return -2;               // (warps are numbered with 32 bits)
        uint16_t* const to = reinterpret_cast<uint16_t*>(at);
        at += plan.dz_bytes;
        auto kernel = fp32 ? k_lay_dz<float, 3> : type == EVO_F16 ? (plan.dz_parts == 2u ? k_lay_dz<__half, 2> : k_lay_dz<__half, 1>)
                                                                  : (plan.dz_parts == 2u ? k_lay_dz<__nv_bfloat16, 2> : k_lay_dz<__nv_bfloat16, 1>);
        if (launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st, a, to, plan.pitch_dz) != cudaSuccess) return -1;
        ++launches;
        dz = to;
        ld_dz = span_dz = static_cast<uint64_t>(plan.dz_parts) * plan.pitch_dz;
    }
    const uint64_t parts = fp32 ? 3u : 1u;
    if (plan.lay_x) {
        uint16_t* const to = reinterpret_cast<uint16_t*>(at);
        at += plan.x_bytes;
        const int n = lay_out(st, type, f, true, plan.pitch, to);
        if (n < 0) return n;
        launches += n;
        x = to; ld_x = parts * plan.pitch; span_x = fp32 ? ld_x : f.n_in;
    }
    if (plan.lay_w) {
        uint16_t* const to = reinterpret_cast<uint16_t*>(at);
        at += plan.w_bytes;
        const int n = lay_out(st, type, f, false, plan.pitch, to);
        if (n < 0) return n;
        launches += n;
        w = to; ld_w = parts * plan.pitch; span_w = fp32 ? ld_w : f.n_in;
        stride_w = f.groups > 1u && f.stride_w == 0u ? 0u : ld_w * f.n_out;
    }
    if (plan.dx) {
        GroupedArgs t = f;
        t.w = w; t.ld_w = ld_w; t.stride_w = stride_w; t.x = dz; t.ld_x = ld_dz; t.b = nullptr; t.y = a.dx; t.ld_y = a.ld_dx;
        t.n_in = f.n_out; t.n_out = f.n_in; t.activation = EVO_ACT_NONE;
        const int n = launch_grouped_tc_transposed(st, type, t, passes, plan.pitch, plan.pitch_dz, span_w, span_dz);
        if (n < 0) return n;
        launches += n;
    }
    if (!plan.dw) return launches;
    const EncodeTiled encode = tensor_map_encoder();
    if (!encode) return -1;
    DwArgs p;
    p.a = a;
    p.waits = grouped_waits();
    p.a.late = plan.dx;                                      // (what is laid out is behind dx's kernel)
    p.all = a.sum_w; p.sets = a.sum_w ? 1u : f.groups; p.splits = splits;
    p.out_tiles = (f.n_out + 127u) / 128u;
    p.in_tiles = (f.n_in + kMostColumns - 1u) / kMostColumns;
    // (several tiles are whole boxes wide: sums leave tensor memory 32 columns at a time)
    p.columns = p.in_tiles > 1u ? ((f.n_in + p.in_tiles - 1u) / p.in_tiles + 63u) / 64u * 64u : (f.n_in + 15u) / 16u * 16u;
    p.in_tiles = (f.n_in + p.columns - 1u) / p.columns;
    const uint32_t stage_bytes = (2u + (p.columns + 63u) / 64u) * 8192u;
    p.stages = kRing / stage_bytes < kMostStages ? kRing / stage_bytes : kMostStages;
    p.passes = passes; p.pitch_dz = plan.pitch_dz; p.pitch_x = plan.pitch;
    p.part = part;
    p.sums = reinterpret_cast<float*>(at);
    p.long_rows = plan.long_rows;
    const uint32_t size = fp32 ? 4u : 2u;
    p.pieces = f.n_in % 4u == 0u && (splits > 1u || (reinterpret_cast<uintptr_t>(a.dw) % (4u * size) == 0u && (a.ld_dw | a.stride_dw) % 4u == 0u));
    const CUtensorMapDataType t = type == EVO_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    for (uint32_t box = 0; box < 2u; ++box) {
        const cuuint64_t dd[2] = { span_dz, f.rows }, ds[1] = { 2u * ld_dz }, xd[2] = { span_x, f.rows }, xs[1] = { 2u * ld_x };
        const cuuint32_t size_of[2] = { 64u, box ? 64u : 16u }, one[2] = { 1u, 1u };
        if (encode(&p.dz[box], t, 2, const_cast<void*>(dz), dd, ds, size_of, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS ||
            encode(&p.x[box], t, 2, const_cast<void*>(x), xd, xs, size_of, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return -1;
    }
    p.boxes = splits == 1u && reinterpret_cast<uintptr_t>(a.dw) % 16u == 0u && (a.ld_dw | a.stride_dw) * size % 16u == 0u && a.ld_dw < (1ull << 36) && a.stride_dw < (1ull << 36);
    if (p.boxes) {
        const uint64_t own = (f.n_in * size + 15ull) / 16ull * 16ull;
        const cuuint64_t wd[3] = { f.n_in, f.n_out, p.sets }, ws[2] = { a.ld_dw * size, a.stride_dw ? a.stride_dw * size : own };
        const cuuint32_t box[3] = { 128u / size, 32u, 1u }, one[3] = { 1u, 1u, 1u };
        if (encode(&p.dw, fp32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : t, 3, a.dw, wd, ws, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
                   CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return -1;
    }
    const uint64_t items = static_cast<uint64_t>(p.sets) * splits * p.out_tiles * p.in_tiles;
    if (items > 0x7FFFFFFFull) return -2;
    auto kernel = fp32 ? k_weights_tc<__nv_bfloat16, float> : type == EVO_F16 ? k_weights_tc<__half, __half> : k_weights_tc<__nv_bfloat16, __nv_bfloat16>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return -1;
    return launch_dependent(kernel, dim3(items < kSms ? static_cast<uint32_t>(items) : kSms), dim3(kThreads), kSmem, st, p) == cudaSuccess ? launches + 1 : -1;
}

}  // namespace evo

// Products grouped by member on tcgen05: y[r] = scale act(W_g x[r] + b_g).
//
// 16-bit operands are taken as they lie where TMA can address their rows; where it cannot (a contracted index that is no multiple of 8, an odd start), and
// fp32 ones, they are first laid out in the workspace, fp32 numbers as three bf16 numbers each (24 bits, no exponent is lost): of their nine
// products the six down to 2^-16 of the largest are made, the small ones first, by running through the contracted index six times.
//
// The weights are the MMA's first operand, 128 outputs, and a group's rows the second, as many as it has (16 .. 256 a tile): a group
// of one row costs one pass over its weights and hardly any tensor time, a long one runs at the tensor core's pace, and no row
// count is padded beyond 16.  Blocks stay and walk over (group, row tile, 128 outputs), the outputs of a row tile side by side, so
// that its rows are read from L2.  A thread copies 64 of the contracted index a stage by TMA (weights 128 x 64, rows in boxes of 128, 64 and 32), another
// issues the MMAs, eight warps take the sums of one tile out of tensor memory while the next tile's are under way.
// One thread waits for operands and issues (a warp that voted on a time-out between two steps left the tensor core idle: 4 groups 225 us).
// 8,192 even rows of 4 groups, 4,096 -> 4,096: 209 us, 1,315 TFLOP/s; of 32 groups, 1,024 -> 4,096: 76 us (the weights alone are 41 from
// memory).  What is left is the first loads, the last wave and, in ragged groups, tiles of few rows.
//
// TR: the weights' rows are the contracted index (the gradient of the rows, dx[r] = W_g' dz[r]): they come as boxes of 64 x 64, MN-major, and nothing is transposed.
#include <cmath>
#include <type_traits>

#include "grouped_gradient.h"
#include "grouped_mma.cuh"
#include "grouped_tc.cuh"

namespace evo {
namespace {

constexpr uint32_t kMostStages = 8;
constexpr uint32_t kMostRows = 256;                          // of a tile, at most
constexpr uint32_t kWBytes = 128u * 128u;                    // of a stage; and as many for every 128 rows of a tile
constexpr uint32_t kRing = 216u * 1024u, kSmem = kRing + 1024u;
constexpr uint32_t kThreads = 320;

// The tensor core cuts its sums off: fp32 rows 1e-6 off per 1,000 of the contracted index.  So the last pass (the large products; the others lie in
// front of its first chunks) is added up in parts of 8 chunks of 64, in fp32 in y (2,060
// numbers 2.1e-6 off in one part).  Of 16-bit operands 6.6e-9 of a sum of numbers of one sign is lost per number (262,144: 1.6e-3, 1,048,576: 7e-3), which
// one part may have of 8,192 numbers; longer sums are added up in parts of 64 chunks (2.7e-5) in the registers of the threads that take them out, which hold
// those of 128 rows.
constexpr uint32_t kSegment = 8, kLongSegment = 64, kLong = 8192, kLongRows = 128;

struct TcArgs {
    GroupedArgs g;
    CUtensorMap w, x[3];                                     // the rows in boxes of 32, 64 and 128
    uint32_t out_tiles, shared_w;                            // shared_w: one set of weights for all groups
    uint32_t most_rows, stages;                              // of a tile (a multiple of 32); as many as the ring has room for
    Waits waits;
    uint32_t passes, pitch_w, pitch_x;                       // passes through the contracted index (1, 6, or TR 2); from one part of an operand to the next
};
// Walks a warp over the tiles of all groups.  Row tiles of a group: as few as can be, equal up to 16 rows.
struct Walk {
    uint32_t base = 0;                                       // groups [base, base + 32): a lane each
    uint64_t before = 0, first = 0, end = 0;                 // row tiles of earlier groups; the lane's rows
    uint32_t tiles = 0, upto = 0;                            // the lane's row tiles, and the running sum

    __device__ __forceinline__ void fill(const TcArgs& p)
    {
        const GroupedArgs& a = p.g;
        const uint32_t lane = threadIdx.x & 31u;
        first = end = 0;
        if (base + lane < a.groups) group_rows(a, base + lane, &first, &end);
        tiles = static_cast<uint32_t>((end - first + p.most_rows - 1u) / p.most_rows);
        upto = tiles;
#pragma unroll
        for (uint32_t d = 1; d < 32u; d <<= 1) {
            const uint32_t v = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += v;
        }
    }
    // row tile `at`: its group, first row and rows; false behind the last
    __device__ __forceinline__ bool find(const TcArgs& p, uint64_t at, uint32_t* group, uint64_t* row, uint32_t* rows)
    {
        for (;;) {
            const uint32_t here = __shfl_sync(0xffffffffu, upto, 31);
            if (at - before < here) break;
            before += here;
            base += 32u;
            if (base >= p.g.groups) return false;
            fill(p);
        }
        const uint32_t local = static_cast<uint32_t>(at - before);
        const uint32_t lane = __ffs(__ballot_sync(0xffffffffu, upto > local)) - 1;
        const uint32_t n = __shfl_sync(0xffffffffu, tiles, lane), nth = local - (__shfl_sync(0xffffffffu, upto, lane) - n);
        const uint64_t f = __shfl_sync(0xffffffffu, first, lane), e = __shfl_sync(0xffffffffu, end, lane);
        const uint64_t per = ((e - f + n - 1u) / n + 15u) / 16u * 16u;        // (n tiles of `per` may be one too many: then the last has no rows)
        *group = base + lane;
        *row = f + nth * per;
        *rows = *row >= e ? 0u : static_cast<uint32_t>(min(per, e - *row));
        return true;
    }
};

// T: type of the operands, O: of bias and result; LONG: a sum of 16-bit operands in several parts
template <typename T, typename O, bool LONG, bool TR>
__global__ void __launch_bounds__(kThreads, 1) k_grouped_tc(const __grid_constant__ TcArgs p)
{
    extern __shared__ uint8_t raw[];
    __shared__ __align__(8) uint64_t full[kMostStages], empty[kMostStages], done[2], taken[2], drain;
    __shared__ uint32_t slot, limit, longest;
    __shared__ volatile int abort_flag;
    const GroupedArgs& a = p.g;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    const uint32_t smem = (smem_u32(raw) + 1023u) / 1024u * 1024u;
    if (tid == 0) {
        for (uint32_t s = 0; s < kMostStages; ++s) { mbar_init(smem_u32(&full[s]), 1); mbar_init(smem_u32(&empty[s]), 1); }
        for (uint32_t b = 0; b < 2u; ++b) { mbar_init(smem_u32(&done[b]), 1); mbar_init(smem_u32(&taken[b]), 8); }
        mbar_init(smem_u32(&drain), 1);
        mbar_init_fence();
        limit = p.waits.cycles_log2;
        longest = kLongestWait;
        abort_flag = 0;
    }
    dep_wait();
    dep_trigger();
    if (warp == 1) tmem_alloc(smem_u32(&slot), 512);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = slot, chunks = (a.n_in + 63u) / 64u, steps = chunks * p.passes, stages = p.stages;
    const uint32_t stage_bytes = kWBytes + p.most_rows * 128u;
    // false: it, or another wait of the block, ran out
    auto wait = [&](uint64_t* bar, uint32_t parity) {
        if (mbar_try_wait(smem_u32(bar), parity)) return true;
        if (abort_flag) return false;
        if (mbar_wait_bounded(smem_u32(bar), parity, &limit)) return true;
        abort_flag = 1;
        return false;
    };
    auto all_of = [](bool fine) { return __all_sync(0xffffffffu, fine) != 0; };
    // the step behind the part of a sum that begins at step k
    const uint32_t small_steps = steps - chunks;
    auto part_end = [&](uint32_t k) { return LONG ? min(steps, k + kLongSegment) : std::is_same<O, float>::value && p.passes > 1u ? min(steps, max(k, small_steps) + kSegment) : steps; };
    // rows of fp16 in two parts: the step at which the sums of second parts end (0: there are none), the first of whose MMAs takes the sum so far down
    constexpr bool kHalfRows = TR && std::is_same<T, __half>::value;
    const uint32_t turn = kHalfRows && p.passes == 2u ? chunks : 0u;
    Walk walk;
    walk.fill(p);
    uint32_t group, rows, stage = 0, phase = 0, acc = 0, acc_phase = 0, filled = 0;
    uint64_t row;

    bool fine = true;
    if (warp == 0) {
        for (uint64_t at = blockIdx.x; fine && walk.find(p, at / p.out_tiles, &group, &row, &rows); at += gridDim.x) {
            if (rows == 0u) continue;
            const uint32_t o0 = static_cast<uint32_t>(at % p.out_tiles) * 128u, read = (rows + 31u) / 32u * 32u, set = p.shared_w ? 0u : group;
            // a copy a lane: the weights' (TR: two boxes of 64 columns), then as few boxes of rows as make them up (8,192 of 4 groups, 4,096 -> 4,096, 323 us with 32 rows
            // each, 242 with 128): whole 128s, a 64, a 32
            constexpr uint32_t kBoxes = TR ? 2u : 1u;
            const uint32_t nth = lane - kBoxes, whole = read / 128u, rest = read % 128u, copies = whole + (rest >= 64u) + (rest % 64u != 0u);
            const uint32_t box = nth < whole ? 2u : nth == whole && rest >= 64u ? 1u : 0u;
            const uint32_t before = nth <= whole ? nth * 128u : whole * 128u + 64u;
            uint32_t pass = 0, chunk = 0;
            for (uint32_t k = 0; k < steps; ++k) {
                fine = all_of(wait(&empty[stage], phase ^ 1u));
                if (!fine) break;
                const uint32_t bar = smem_u32(&full[stage]), to = smem + stage * stage_bytes;
                if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(kWBytes + read * 128u) : "memory");
                __syncwarp();
                uint32_t at_w = 0, at_x = 0;                 // (where the operands' parts begin)
                if (TR && p.passes == 2u) at_x = kPartTwo[pass] * p.pitch_x;
                else if (p.passes > 1u) { at_w = kPartW[pass] * p.pitch_w; at_x = kPartX[pass] * p.pitch_x; }
                if (lane < kBoxes) {
                    if constexpr (TR) copy3(to + 8192u * lane, &p.w, at_w + o0 + 64u * lane, chunk * 64u, set, bar);
                    else copy3(to, &p.w, at_w + chunk * 64u, o0, set, bar);
                } else if (nth < copies) {
                    copy2(to + kWBytes + before * 128u, &p.x[box], at_x + chunk * 64u, static_cast<uint32_t>(row) + before, bar);
                }
                if (++chunk == chunks) { chunk = 0; ++pass; }
                __syncwarp();
                ++filled;
                if (++stage == stages) { stage = 0; phase ^= 1u; }
            }
        }
        if (!fine)                                           // nothing may land after the block has gone
            for (uint32_t s = 0; s < min(filled, stages); ++s) {
                const uint32_t nth = filled - 1u - s;
                mbar_wait_bounded(smem_u32(&full[nth % stages]), nth / stages & 1u, &longest);
            }
    } else if (warp == 1) {
        for (uint64_t at = blockIdx.x; fine && walk.find(p, at / p.out_tiles, &group, &row, &rows); at += gridDim.x) {
            if (rows == 0u) continue;
            if (lane == 0) {                                 // (one thread: what it does between two MMAs is time that the tensor core has nothing to do)
                const uint32_t id = idesc<T, TR>((rows + 15u) / 16u * 16u);
                for (uint32_t k = 0; k < steps && fine;) {
                    const uint32_t d = tmem + acc * kMostRows, first = k, end = part_end(k);
                    fine = wait(&taken[acc], acc_phase ^ 1u);
                    tc_fence_after();
                    for (; k < end && fine; ++k) {
                        fine = wait(&full[stage], phase);
                        const uint32_t w = smem + stage * stage_bytes;
                        const uint64_t a = TR ? desc_sw128_mn(w, 8192u) : desc_sw128(w), b = desc_sw128(w + kWBytes);
#pragma unroll
                        for (uint32_t s = 0; s < 4u; ++s) {
                            if (kHalfRows && s == 0u && k == turn && k != first) umma_scaling_down<kSecondUp>(d, a, b, id);
                            else umma_bf16(d, a + s * (TR ? 128u : 2u), b + s * 2u, id, k - first + s != 0u);
                        }
#ifdef EVO_DEBUG
                        if (!p.waits.drop || blockIdx.x != 0u || at != 0u || k != 0u)
#endif
                        umma_commit(smem_u32(&empty[stage]));
                        if (++stage == stages) { stage = 0; phase ^= 1u; }
                    }
                    umma_commit(smem_u32(&done[acc]));
                    acc ^= 1u;
                    if (acc == 0u) acc_phase ^= 1u;
                }
            }
            fine = __shfl_sync(0xffffffffu, fine, 0);
        }
        if (!fine && lane == 0) {                            // no MMA may write after its tensor memory is freed
            umma_commit(smem_u32(&drain));
            mbar_wait_bounded(smem_u32(&drain), 0u, &longest);
        }
        __syncwarp();
    } else {
        const uint32_t quarter = warp & 3u, half = (warp - 2u) >> 2;
        for (uint64_t at = blockIdx.x; walk.find(p, at / p.out_tiles, &group, &row, &rows); at += gridDim.x) {
            if (rows == 0u) continue;
            const uint32_t o = static_cast<uint32_t>(at % p.out_tiles) * 128u + quarter * 32u + lane;
            const bool live = o < a.n_out;
            float bias = 0.f;
            if (a.b && live) {
                const O b = static_cast<const O*>(a.b)[group * a.stride_b + o];
                if constexpr (std::is_same<O, __half>::value) bias = __half2float(b);
                else if constexpr (std::is_same<O, float>::value) bias = b;
                else bias = __bfloat162float(b);
            }
            O* const y = static_cast<O*>(a.y) + row * a.ld_y + o;
            float held[LONG ? kLongRows / 64u : 1u][32];          // the sum of the parts before this one
            for (uint32_t first = 0, end = 0; end < steps; first = end) {
                end = part_end(first);
                wait(&done[acc], acc_phase);
                __syncwarp();
                tc_fence_after();
                const float scale = abort_flag ? __int_as_float(0x7FC00000) : a.scale;
                auto take = [&](uint32_t c, float (&so_far)[32]) {
                    uint32_t u[4][8];
                    tmem_ld32_issue(tmem + acc * kMostRows + (quarter << 21) + c, u);
                    tmem_ld8x4_fence(u[0], u[1], u[2], u[3]);
                    O* to = y + c * a.ld_y;
                    const uint32_t count = live ? min(32u, rows - c) : 0u;
                    float v[32];
#pragma unroll
                    for (uint32_t i = 0; i < 32u; ++i) v[i] = __uint_as_float(u[i / 8u][i % 8u]);
                    if constexpr (LONG) {
                        if (kHalfRows && end <= turn)        // (a part of second numbers alone)
#pragma unroll
                            for (uint32_t i = 0; i < 32u; ++i) v[i] *= kDown<__half>;
#pragma unroll
                        for (uint32_t i = 0; i < 32u; ++i) so_far[i] = v[i] = first ? so_far[i] + v[i] : v[i];
                        if (end != steps) return;
                    }
                    if constexpr (std::is_same<O, float>::value) {
                        if (first != 0u) {
#pragma unroll
                            for (uint32_t i = 0; i < 32u; ++i) v[i] += i < count ? to[i * a.ld_y] : 0.f;
                        }
                        if (end != steps) {
#pragma unroll
                            for (uint32_t i = 0; i < 32u; ++i)
                                if (i < count) to[i * a.ld_y] = v[i];
                            __syncwarp();
                            return;
                        }
                    }
#pragma unroll
                    for (uint32_t i = 0; i < 32u; ++i) v[i] += bias;
                    if (a.activation == EVO_ACT_TANH) {
#pragma unroll
                        for (uint32_t i = 0; i < 32u; ++i) v[i] = gm::tanh32(v[i]);
                    } else if (a.activation == EVO_ACT_RELU) {
#pragma unroll
                        for (uint32_t i = 0; i < 32u; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
                    }
#pragma unroll
                    for (uint32_t i = 0; i < 32u; ++i) {
                        if (i < count) {
                            if constexpr (std::is_same<O, __half>::value) *to = __float2half_rn(scale * v[i]);
                            else if constexpr (std::is_same<O, float>::value) *to = scale * v[i];
                            else *to = __float2bfloat16_rn(scale * v[i]);
                        }
                        to += a.ld_y;
                    }
                    __syncwarp();
                };
                // the halves take every other 32 rows
                if constexpr (LONG) {
#pragma unroll
                    for (uint32_t i = 0; i < kLongRows / 64u; ++i)
                        if (half * 32u + i * 64u < rows) take(half * 32u + i * 64u, held[i]);
                } else {
                    for (uint32_t c = half * 32u; c < rows; c += 64u) take(c, held[0]);
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&taken[acc]));
                acc ^= 1u;
                if (acc == 0u) acc_phase ^= 1u;
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

// Lays rows out for TMA: 16-bit ones as they are, fp32 ones as three bf16 parts, `pitch` apart and filled up with zeros.  Weight rows of groups that have
// rows; or, where n_out is 0, the rows themselves.
template <typename T>
__global__ void __launch_bounds__(256) k_lay_out(const __grid_constant__ GroupedArgs a, const T* __restrict__ from, uint64_t stride, uint64_t ld, uint32_t n_out, uint16_t* __restrict__ to, uint32_t pitch)
{
    constexpr uint32_t kParts = std::is_same<T, float>::value ? 3u : 1u;
    dep_wait();
    dep_trigger();
    const uint32_t warp = threadIdx.x >> 5, lane = threadIdx.x & 31u;
    uint64_t row = static_cast<uint64_t>(blockIdx.x) * 8u + warp, count = a.rows;      // a row a warp
    const T* src = from;
    if (n_out) {
        const uint32_t per = (n_out + 7u) / 8u, group = blockIdx.x / per, o = blockIdx.x % per * 8u + warp;
        uint64_t first = 0, end = 1;
        if (stride || a.groups == 1u) group_rows(a, group, &first, &end);
        if (first == end || o >= n_out) return;
        src += group * stride + o * ld;
        row = static_cast<uint64_t>(group) * n_out + o;
        count = row + 1u;
    } else {
        src += row * ld;
    }
    if (row >= count) return;
    uint16_t* const dst = to + row * kParts * pitch;
    if constexpr (kParts == 1u) {                            // (the pitch is even; a number behind the last is written and never read)
        const uint16_t* const s = reinterpret_cast<const uint16_t*>(src);
        for (uint32_t k = 2u * lane; k < a.n_in; k += 64u)
            *reinterpret_cast<uint32_t*>(dst + k) = s[k] | (k + 1u < a.n_in ? static_cast<uint32_t>(s[k + 1u]) << 16 : 0u);
    } else {
        // (Without branches: 61 groups of 159 rows, 2,428 -> 5, 169 us, with them 197.)
#pragma unroll 4
        for (uint32_t k = lane; k < pitch; k += 32u) {
            const float x = k < a.n_in ? src[k] : 0.f;
            three_parts(x, dst + k, dst + pitch + k, dst + 2u * pitch + k);
        }
    }
}

}  // namespace

bool grouped_tc_addressable(uint32_t type, const GroupedArgs& a)
{
    if (type == EVO_F32 || ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15u)) return false;
    if ((a.ld_x | a.ld_w | a.stride_w) & 7u) return false;
    return a.rows < (1ull << 31) && a.ld_x < (1ull << 38) && a.ld_w < (1ull << 38) && a.stride_w < (1ull << 38);
}

// The SMs that a tile for each 128 outputs of every group with rows leaves without one
static double idle_share(const GroupedArgs& a)
{
    const double tiles = std::fmin(static_cast<double>(a.rows), a.groups) * ((a.n_out + 127u) / 128u);
    return std::fmax(0.0, 1.0 - tiles / kSms);
}

// Whether they pay against mma.sync with 16-byte loads: not with few rows a group where weight rows are short, where every warp's walk over many groups takes longer
// than the products (26 ns a group), where a tile for each 128 outputs leaves SMs without one, and where most of a tile's outputs do not exist.  us, without / with, rows
// a group in brackets:
//   4,096 of 128 -> 128 (4) 40 / 114, (32) 79 / 118; 200 of 512 -> 512 (4) 30.1 / 31.8, (8) 35.9 / 32.0, (32) 64 / 33; 64 of 2,048 -> 2,048 (1) 96 / 87, (8) 133 / 100;
//   1 of 4,096 -> 4,096 (8) 18.4 / 29.8, (32) 33.6 / 29.8; 8 of them (1) 55 / 59, (4) 67 / 59; 500 of 2,048 -> 16 (7) 24.7 / 62.5.
// Over 809 shapes (740 of them drawn, up to 4,096 -> 4,096, 4,096 groups, 300 rows a group) 1.013 times the faster side's time in the geometric mean, 1.85 at worst;
// with the tensor cores always, 1.45 and 7.7.
bool grouped_tc_takes(uint32_t type, const GroupedArgs& a)
{
    if (!grouped_tc_addressable(type, a)) return false;
    const double rows = static_cast<double>(a.rows), groups = a.groups, out_tiles = (a.n_out + 127u) / 128u, idle = idle_share(a);
    return rows >= groups * (1000.0 / a.n_in + groups / 133.0 + 0.5 * (out_tiles * 128.0 / a.n_out - 1.0) + 24.0 * idle * idle * idle);
}

uint32_t grouped_tc_pitch(uint32_t type, uint32_t n_in) { return type == EVO_F32 ? (n_in + 63u) / 64u * 64u : (n_in + 7u) / 8u * 8u; }

// Bytes for rows laid out anew where that pays (0: it does not): the weights are read, written and read again whatever the rows, so a group has to have some, and
// more where its rows are short, where there are many groups to walk over, and where a tile for each 128 outputs leaves SMs without one.  16-bit operands, against loads of
// single numbers; fp32, three bf16 parts of each number and six products, against pairs in tf32 with mma.sync.  Without / with, us, rows a group in brackets:
//   16 bits  1,000 groups of 61 -> 49 (8) 8.6 / 39.3, (32) 19.2 / 43.6; 300 of 207 -> 379 (8) 38.7 / 64.7, (16) 53.5 / 65.6, (32) 84.1 / 68.5; 50 of
//            1,001 -> 1,000 (4) 69.8 / 77.8, (8) 87.1 / 78.0, (32) 204.8 / 78.9; 8 of 2,047 -> 2,048 (4) 57.5 / 51.2
//   fp32     1,000 of 128 -> 128 (28) 51.8 / 102, (48) 83.3 / 109; 50 of 1,000 -> 1,000 (28) 163.8 / 231, (48) 316 / 237; 100 of 512 -> 512 (32) 96 / 122, (64) 163 / 127;
//            38 of 1,684 -> 27 (45) 359 / 96
// Over 1,100 drawn shapes (up to 4,096 -> 4,096, 4,096 groups, 300 rows a group) the choice takes 1.02 times the faster side's time in the geometric mean.
size_t grouped_tc_bytes(uint32_t type, const GroupedArgs& a)
{
    const uint64_t pitch = grouped_tc_pitch(type, a.n_in), parts = type == EVO_F32 ? 3u : 1u;
    const bool shared = a.groups > 1u && a.stride_w == 0u, fp32 = type == EVO_F32;
    const double least = (fp32 ? 24.0 : 4.0) + 1500.0 / a.n_in + std::fmin(a.groups, 400.0) / 50.0 + (fp32 ? 8.0 : 4.0) * idle_share(a);
    if (a.rows >= (1ull << 31) || static_cast<double>(a.rows) < least * a.groups || (shared ? 1ull : a.groups) * a.n_out >= (1ull << 31)) return 0;
    const uint64_t rows = (shared ? 1ull : a.groups) * a.n_out + a.rows;
    return static_cast<size_t>(rows * parts * pitch * 2u + 256u);
}

// Rows of a tile, at most.  The groups' sizes are on the device, so their tiles are guessed at (a tile for every so many rows and half a one
// more a group); a tile takes as long as its operands, 128 rows of weights and its own rows, and the blocks take tiles in waves.  64 / 128 / 192 /
// 256 rows: 8,192 even rows of 32 groups, 1,024 -> 4,096, 209 / 119 / 118 / 82 us; 3,774 of 6, 1,207 -> 2,379, 103 / 81 / 69 / 73;
// 3,000 of 100, 1,024 -> 1,024, 55 / 59 / 59 / 64 (fewer rows a stage are more stages in flight).
static uint32_t rows_of_a_tile(const GroupedArgs& a, uint32_t out_tiles, uint32_t limit)
{
    uint32_t best = limit;
    double least = 1e300;
    for (uint32_t most = 64u; most <= limit; most += 64u) {
        const double used = static_cast<double>(a.rows < a.groups ? a.rows : a.groups), guess = static_cast<double>(a.rows) / most + 0.5 * used;
        const double tiles = guess > used ? guess : used, time = std::ceil(tiles * out_tiles / kSms) * (128.0 + a.rows / tiles);
        if (time < least * 0.999) { least = time; best = most; }
    }
    return best;
}

// Weights of groups that have rows, or (rows) the rows of x, as TMA can address them.
int lay_out(cudaStream_t st, uint32_t type, const GroupedArgs& a, bool rows, uint32_t pitch, uint16_t* to)
{
    const uint64_t sets = a.groups > 1u && a.stride_w == 0u ? 1u : a.groups;
    const uint64_t blocks = rows ? (a.rows + 7u) / 8u : sets * ((a.n_out + 7u) / 8u), stride = rows ? 0u : a.stride_w, ld = rows ? a.ld_x : a.ld_w;
    if (blocks > 0x7FFFFFFFull) return -2;
    const void* const from = rows ? a.x : a.w;
    const uint32_t n_out = rows ? 0u : a.n_out;
    const dim3 grid(static_cast<uint32_t>(blocks));
    const cudaError_t e = type == EVO_F32 ? launch_dependent(k_lay_out<float>, grid, dim3(256), 0, st, a, static_cast<const float*>(from), stride, ld, n_out, to, pitch)
                                          : launch_dependent(k_lay_out<__half>, grid, dim3(256), 0, st, a, static_cast<const __half*>(from), stride, ld, n_out, to, pitch);
    return e == cudaSuccess ? 1 : -1;
}

// The product with operands as they lie (or have been laid out): span_w and span_x numbers of a row of each can be addressed.
static int launch_tiles(cudaStream_t st, uint32_t type, TcArgs& p, bool transposed, uint64_t span_w, uint64_t span_x)
{
    const EncodeTiled f = tensor_map_encoder();
    if (!f) return -1;
    const GroupedArgs& a = p.g;
    p.waits = grouped_waits();
    p.out_tiles = (a.n_out + 127u) / 128u;
    p.shared_w = a.groups > 1u && a.stride_w == 0u;
    const CUtensorMapDataType t = type == EVO_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    // (a pitch of 0 is one that is never taken: any valid one stands in for it)
    const uint64_t own_w = (span_w + 7ull) / 8ull * 8ull, own_x = (span_x + 7ull) / 8ull * 8ull;
    const cuuint64_t wd[3] = { span_w, transposed ? a.n_in : a.n_out, p.shared_w ? 1u : a.groups }, ws[2] = { 2u * (a.ld_w ? a.ld_w : own_w), 2u * (a.stride_w ? a.stride_w : own_w) };
    const cuuint64_t xd[2] = { span_x, a.rows }, xs[1] = { 2u * (a.ld_x ? a.ld_x : own_x) };
    const cuuint32_t wb[3] = { 64u, transposed ? 64u : 128u, 1u }, xb[3][2] = { { 64u, 32u }, { 64u, 64u }, { 64u, 128u } }, one[3] = { 1u, 1u, 1u };
    if (f(&p.w, t, 3, const_cast<void*>(a.w), wd, ws, wb, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
          CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return -1;
    for (int box = 0; box < 3; ++box)
        if (f(&p.x[box], t, 2, const_cast<void*>(a.x), xd, xs, xb[box], one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return -1;
    const bool parts_held = type != EVO_F32 && static_cast<uint64_t>(a.n_in) * p.passes > kLong;
    p.most_rows = rows_of_a_tile(a, p.out_tiles, parts_held ? kLongRows : kMostRows);
    p.stages = kRing / (kWBytes + p.most_rows * 128u);
    if (p.stages > kMostStages) p.stages = kMostStages;
    const uint64_t used = a.rows < a.groups ? a.rows : a.groups, most = (a.rows / p.most_rows + used) * p.out_tiles;
    using B = __nv_bfloat16;
    auto kernel = transposed ? (type == EVO_F32 ? k_grouped_tc<B, float, false, true>
                              : type == EVO_F16 ? (parts_held ? k_grouped_tc<__half, __half, true, true> : k_grouped_tc<__half, __half, false, true>)
                                                : (parts_held ? k_grouped_tc<B, B, true, true> : k_grouped_tc<B, B, false, true>))
                             : (type == EVO_F32 ? k_grouped_tc<B, float, false, false>
                              : type == EVO_F16 ? (parts_held ? k_grouped_tc<__half, __half, true, false> : k_grouped_tc<__half, __half, false, false>)
                                                : (parts_held ? k_grouped_tc<B, B, true, false> : k_grouped_tc<B, B, false, false>));
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return -1;
    return launch_dependent(kernel, dim3(most < kSms ? static_cast<uint32_t>(most) : kSms), dim3(kThreads), kSmem, st, p) == cudaSuccess ? 1 : -1;
}

int launch_grouped_tc(cudaStream_t st, uint32_t type, const GroupedArgs& in, void* work)
{
    TcArgs p;
    p.g = in;
    GroupedArgs& a = p.g;
    p.passes = type == EVO_F32 ? 6u : 1u;
    p.pitch_w = p.pitch_x = grouped_tc_pitch(type, a.n_in);
    int launches = 0;
    uint64_t span = a.n_in;                                  // of the contracted index, all parts
    if (work) {
        const bool shared = a.groups > 1u && a.stride_w == 0u;
        const uint32_t parts = type == EVO_F32 ? 3u : 1u, pitch = p.pitch_x;
        uint16_t* const w = static_cast<uint16_t*>(work);
        uint16_t* const x = w + (static_cast<uint64_t>(shared ? 1u : a.groups) * a.n_out * parts * pitch + 127u) / 128u * 128u;
        for (int rows = 0; rows < 2; ++rows) {
            const int n = lay_out(st, type, a, rows != 0, pitch, rows ? x : w);
            if (n < 0) return n;
            launches += n;
        }
        a.w = w; a.x = x;
        a.ld_w = a.ld_x = static_cast<uint64_t>(parts) * pitch;
        a.stride_w = shared ? 0u : a.ld_w * a.n_out;
        if (type == EVO_F32) span = a.ld_w;
    }
    const int n = launch_tiles(st, type, p, false, span, span);
    return n < 0 ? n : launches + n;
}

int launch_grouped_tc_transposed(cudaStream_t st, uint32_t type, const GroupedArgs& a, uint32_t passes, uint32_t pitch_w, uint32_t pitch_x, uint64_t span_w, uint64_t span_x)
{
    TcArgs p;
    p.g = a;
    p.passes = passes; p.pitch_w = pitch_w; p.pitch_x = pitch_x;
    return launch_tiles(st, type, p, true, span_w, span_x);
}

}  // namespace evo

// The stable order of pairs by member: a counting sort.
//
// A warp walks over consecutive pairs, 32 at a time.  Lanes that chose the same member find each other by ballots, so that a pair's rank among
// the earlier ones of its member is what the warp has counted plus the lanes before it; a block's warps have counters of their own
// in shared memory, which a scan over the warps turns into positions.  No atomics: the order is the pairs' own.
// Up to 32,768 pairs are in the registers of one block or of a cluster of eight, whose totals meet through distributed shared memory: one launch.  More are counted,
// scanned and placed in three; the table in between holds a count for every member and block.  Of more than 2,047 members, whose counters would take longer than
// the pairs, a pass sorts by the lower half of the bits and another by the upper (524,288 pairs of 4,096: 57 us at once, 45 so).
// It is bound by latency: 131,072 pairs are 1.6 MB.  In a graph 64 pairs take 1.8 us, 4,096 of 64 members 7.0, 16,384 8.6 (one launch each), 131,072 11.4, 524,288 18.5.
#include "async.cuh"
#include "routing.h"

namespace evo {
namespace {

constexpr uint32_t kMostBins = 2048, kMostBlocks = 592;
constexpr uint32_t kSmem = 200u * 1024u, kOwn = 32u * 4u;      // of counters at most; beside them (warp_sums)

struct Pass {
    RouteArgs a;
    uint32_t shift, mask, bins, bits;    // bin = (member >> shift) & mask; pairs without a member have member `groups`
    uint32_t counting, per_warp;         // warps that count, and the pairs of each (a multiple of 32)
    const uint32_t* order_in;            // pairs in the order of the pass before, or NULL
    uint32_t* order_out;                 // the order that this pass makes, or NULL: it is the last
    uint32_t* sorted;                    // the last of two: members in their new order, or NULL
    uint32_t* table; uint32_t* totals;   // [bins][blocks], [bins]
    uint32_t blocks;
};

__device__ __forceinline__ uint32_t member_of(const RouteArgs& a, uint32_t p)
{
    const uint64_t at = a.ld == a.choices ? p : static_cast<uint64_t>(p / a.choices) * a.ld + p % a.choices;
    const int64_t m = a.wide ? static_cast<const int64_t*>(a.members)[at] : static_cast<const int32_t*>(a.members)[at];
    return m < 0 || m >= static_cast<int64_t>(a.groups) ? a.groups : static_cast<uint32_t>(m);
}

// Lanes of the same bin, of those that have one: a ballot for every bit of the bins' numbers (match.any takes several times as long: 131,072 pairs of 64
// members 32 us with it).
__device__ __forceinline__ uint32_t same_bin(uint32_t bin, bool live, uint32_t bits)
{
    uint32_t same = __ballot_sync(0xffffffffu, live);
    for (uint32_t b = 0; b < bits; ++b) {
        const bool one = bin >> b & 1u;
        const uint32_t ones = __ballot_sync(0xffffffffu, one);
        same &= one ? ones : ~ones;
    }
    return same;
}

// the place of a pair
__device__ __forceinline__ void put(const Pass& p, uint32_t pair, uint32_t member, uint32_t at)
{
    if (p.order_out) {
        p.order_out[at] = pair;
        return;
    }
    const bool live = member < p.a.groups;
    p.a.place[pair] = live ? static_cast<int32_t>(at) : -1;
    if (p.sorted) p.sorted[at] = member;
    if (p.a.source) p.a.source[at] = live ? static_cast<int32_t>(pair) : -1;
}

// Exclusive prefix sums of v[0 .. n) in place, by a block; `warp_sums` has room for 32.
__device__ void block_scan(uint32_t* v, uint32_t n, uint32_t* warp_sums)
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, per = (n + blockDim.x - 1u) / blockDim.x;
    const uint32_t first = min(threadIdx.x * per, n), end = min(first + per, n);
    uint32_t sum = 0;
    for (uint32_t i = first; i < end; ++i) sum += v[i];
    uint32_t upto = sum;
#pragma unroll
    for (uint32_t d = 1; d < 32u; d <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += x;
    }
    if (lane == 31u) warp_sums[warp] = upto;
    __syncthreads();
    if (warp == 0) {
        const uint32_t mine = lane < blockDim.x / 32u ? warp_sums[lane] : 0u;
        uint32_t s = mine;
#pragma unroll
        for (uint32_t d = 1; d < 32u; d <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += x;
        }
        warp_sums[lane] = s - mine;
    }
    __syncthreads();
    uint32_t before = warp_sums[warp] + upto - sum;
    for (uint32_t i = first; i < end; ++i) {
        const uint32_t x = v[i];
        v[i] = before;
        before += x;
    }
    __syncthreads();
}

// ---- one launch ----
// The pairs in registers, IT of a lane; CTAS blocks, of which each has the same part.
template <uint32_t CTAS, uint32_t IT>
__global__ void __launch_bounds__(1024) k_route_once(const __grid_constant__ Pass p)
{
    extern __shared__ uint32_t counts[];                     // [counting][bins], total[bins], base[bins]
    __shared__ uint32_t warp_sums[32];
    uint32_t* const total = counts + p.counting * p.bins;
    uint32_t* const base = total + p.bins;
    const RouteArgs& a = p.a;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    const bool counts_here = warp < p.counting;
    uint32_t* const mine = counts + (counts_here ? warp * p.bins : 0u);
    for (uint32_t i = threadIdx.x; i < p.counting * p.bins; i += blockDim.x) counts[i] = 0u;
    dep_wait();
    dep_trigger();
    const uint32_t first = (blockIdx.x * p.counting + warp) * 32u * IT + lane, end = counts_here ? a.pairs : 0u;
    uint32_t pair[IT], member[IT], rank[IT];
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) {
        pair[i] = first + 32u * i;
        if (p.order_in && pair[i] < end) pair[i] = p.order_in[pair[i]];
    }
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) member[i] = first + 32u * i < end ? member_of(a, pair[i]) : 0u;
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) {
        const bool live = first + 32u * i < end;
        const uint32_t bin = member[i] >> p.shift & p.mask, same = same_bin(bin, live, p.bits);
        rank[i] = 0u;
        if (live) rank[i] = mine[bin] + __popc(same & ((1u << lane) - 1u));
        __syncwarp();
        if (live && lane == __ffs(same) - 1u) mine[bin] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) {
        uint32_t sum = 0;
#pragma unroll 4
        for (uint32_t w = 0; w < p.counting; ++w) {
            const uint32_t c = counts[w * p.bins + b];
            counts[w * p.bins + b] = sum;
            sum += c;
        }
        total[b] = sum;
        if (CTAS == 1u) base[b] = sum;
    }
    if constexpr (CTAS > 1u) {
        __syncwarp();                                        // (.aligned: a warp comes to it as one, from loops that its lanes leave at different turns)
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        // the sum over the blocks, and what the blocks before this one have (added to the first warp's counts and so on below)
        for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) {
            uint32_t sum = 0, before = 0;
#pragma unroll
            for (uint32_t r = 0; r < CTAS; ++r) {
                uint32_t there, c;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(smem_u32(total + b)), "r"(r));
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(c) : "r"(there) : "memory");
                if (r < blockIdx.x) before += c;
                sum += c;
            }
            base[b] = sum;
            for (uint32_t w = 0; w < p.counting; ++w) counts[w * p.bins + b] += before;
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");       // (waited for at the end: the others may still be reading)
    }
    __syncthreads();
    block_scan(base, p.bins, warp_sums);
    if (!p.order_out && !p.sorted && blockIdx.x == 0u)
        for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) a.offsets[b] = static_cast<int32_t>(base[b]);
#pragma unroll
    for (uint32_t i = 0; i < IT; ++i) {
        if (first + 32u * i >= end) break;
        const uint32_t bin = member[i] >> p.shift & p.mask;
        put(p, pair[i], member[i], base[bin] + mine[bin] + rank[i]);
    }
    if constexpr (CTAS > 1u) {
        __syncwarp();
        asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    }
}

// ---- three launches ----
enum { kCount = 1, kPlace = 2 };

template <int MODE>
__global__ void __launch_bounds__(1024) k_route(const __grid_constant__ Pass p)
{
    extern __shared__ uint32_t counts[];                     // [counting][bins], base[bins]
    __shared__ uint32_t warp_sums[32];
    uint32_t* const base = counts + p.counting * p.bins;
    const RouteArgs& a = p.a;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
    for (uint32_t i = threadIdx.x; i < p.counting * p.bins; i += blockDim.x) counts[i] = 0u;
    dep_wait();
    dep_trigger();
    __syncthreads();
    const uint64_t first = (static_cast<uint64_t>(blockIdx.x) * p.counting + warp) * p.per_warp;
    const uint64_t end = warp < p.counting ? min(first + p.per_warp, static_cast<uint64_t>(a.pairs)) : first;
    uint32_t* const mine = counts + (warp < p.counting ? warp * p.bins : 0u);
    // calls f(pair, its member, its bin, whether there is one, lanes of the same bin) for the warp's pairs in their order
    auto walk = [&](auto f) {
        for (uint64_t i = first; i < end; i += 32u) {
            uint32_t pair = 0, member = 0, bin = 0;
            const bool live = i + lane < end;
            if (live) {
                pair = p.order_in ? p.order_in[i + lane] : static_cast<uint32_t>(i) + lane;
                member = member_of(a, pair);
                bin = member >> p.shift & p.mask;
            }
            f(pair, member, bin, live, same_bin(bin, live, p.bits));
            __syncwarp();
        }
    };
    walk([&](uint32_t, uint32_t, uint32_t bin, bool live, uint32_t same) {
        if (live && lane == __ffs(same) - 1u) mine[bin] += __popc(same);
    });
    __syncthreads();
    // counts of the warps before, and of all of them
    for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) {
        uint32_t sum = 0;
        for (uint32_t w = 0; w < p.counting; ++w) {
            const uint32_t c = counts[w * p.bins + b];
            if (MODE != kCount) counts[w * p.bins + b] = sum;
            sum += c;
        }
        if (MODE == kCount) p.table[static_cast<uint64_t>(b) * p.blocks + blockIdx.x] = sum;
        else base[b] = p.totals[b];
    }
    if (MODE == kCount) return;
    __syncthreads();
    block_scan(base, p.bins, warp_sums);
    if (!p.order_out && !p.sorted && blockIdx.x == 0u)
        for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) a.offsets[b] = static_cast<int32_t>(base[b]);
    __syncthreads();
    for (uint32_t b = threadIdx.x; b < p.bins; b += blockDim.x) base[b] += p.table[static_cast<uint64_t>(b) * p.blocks + blockIdx.x];
    __syncthreads();
    walk([&](uint32_t pair, uint32_t member, uint32_t bin, bool live, uint32_t same) {
        if (live) {
            put(p, pair, member, base[bin] + mine[bin] + __popc(same & ((1u << lane) - 1u)));
        }
        __syncwarp();
        if (live && lane == __ffs(same) - 1u) mine[bin] += __popc(same);
    });
}

// the table's counts to those of the blocks before, a warp a bin
__global__ void __launch_bounds__(256) k_route_scan(uint32_t* __restrict__ table, uint32_t* __restrict__ totals, uint32_t bins, uint32_t blocks)
{
    dep_wait();
    dep_trigger();
    const uint32_t bin = blockIdx.x * 8u + (threadIdx.x >> 5), lane = threadIdx.x & 31u;
    if (bin >= bins) return;
    uint32_t* const t = table + static_cast<uint64_t>(bin) * blocks;
    uint32_t before = 0;
    for (uint32_t i = 0; i < blocks; i += 32u) {
        const uint32_t c = i + lane < blocks ? t[i + lane] : 0u;
        uint32_t upto = c;
#pragma unroll
        for (uint32_t d = 1; d < 32u; d <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += x;
        }
        if (i + lane < blocks) t[i + lane] = before + upto - c;
        before += __shfl_sync(0xffffffffu, upto, 31);
    }
    if (lane == 0u) totals[bin] = before;
}

// After two passes: offsets[g] = pairs whose member is below g, by bisection of the members in their new order.
__global__ void __launch_bounds__(256) k_route_offsets(const __grid_constant__ RouteArgs a, const uint32_t* __restrict__ sorted)
{
    dep_wait();
    dep_trigger();
    const uint32_t g = blockIdx.x * 256u + threadIdx.x;
    if (g > a.groups) return;
    uint32_t low = 0, high = a.pairs;
    while (low < high) {
        const uint32_t middle = low + (high - low) / 2u;
        if (sorted[middle] < g) low = middle + 1u;
        else high = middle;
    }
    a.offsets[g] = static_cast<int32_t>(low);
}

// A cluster has no more SMs than eight for the scattered stores: 16,384 / 32,768 / 131,072 pairs of 64 members 8.6 / 8.7 / 25 us with it.
constexpr uint32_t kCluster = 8, kClusterPairs = 32768, kClusterBins = 1024, kWarps = 8;

struct Plan {
    uint32_t passes, low_bits, bins[2], counting[2], per_warp[2], blocks[2], it[2];      // it 0: three launches
};

uint32_t warps_for(uint32_t bins)
{
    uint32_t w = 32;
    while (w > 1u && (w + 2u) * bins * 4u > kSmem) w /= 2u;
    return w;
}

Plan plan_for(const RouteArgs& a)
{
    Plan p;
    p.passes = a.groups + 1u <= kMostBins ? 1u : 2u;
    p.low_bits = (33u - __builtin_clz(a.groups)) / 2u;       // half of a member's bits, the odd one among them
    p.bins[0] = p.passes == 1u ? a.groups + 1u : 1u << p.low_bits;
    p.bins[1] = (a.groups >> p.low_bits) + 1u;
    for (uint32_t i = 0; i < p.passes; ++i) {
        const uint32_t most = warps_for(p.bins[i]);
        if (a.pairs <= 128u * most || (a.pairs <= kClusterPairs && p.bins[i] <= kClusterBins)) {
            // one block with up to four pairs a lane, then a cluster
            p.blocks[i] = a.pairs <= 128u * most ? 1u : kCluster;
            const uint32_t mine = (a.pairs + p.blocks[i] - 1u) / p.blocks[i];
            uint32_t w = 1;
            while (w < most && w * 32u < mine) w *= 2u;
            p.counting[i] = w; p.it[i] = w * 32u < mine ? 4u : 1u; p.per_warp[i] = 32u * p.it[i];
            continue;
        }
        const uint32_t w = most < kWarps ? most : kWarps;
        uint64_t tile = 128ull * w;                          // pairs of a block
        if ((a.pairs + tile - 1u) / tile > kMostBlocks) tile = (a.pairs + kMostBlocks - 1ull) / kMostBlocks;
        p.it[i] = 0; p.counting[i] = w;
        p.per_warp[i] = static_cast<uint32_t>((tile + w * 32ull - 1u) / (w * 32ull) * 32u);
        const uint64_t per = static_cast<uint64_t>(p.per_warp[i]) * w;
        p.blocks[i] = static_cast<uint32_t>((a.pairs + per - 1u) / per);
    }
    return p;
}

// (48 KB without asking, what a kernel has beside its counters included)
bool has_room(void (*kernel)(Pass), size_t smem)
{
    return smem + kOwn <= 48u * 1024u || cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmem)) == cudaSuccess;
}

template <uint32_t CTAS>
cudaError_t launch_once(cudaStream_t st, uint32_t it, uint32_t threads, size_t smem, const Pass& p)
{
    auto kernel = it == 1u ? k_route_once<CTAS, 1> : k_route_once<CTAS, 4>;
    if (!has_room(kernel, smem)) return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(CTAS); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = CTAS; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = CTAS > 1u ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

size_t round_up(size_t n) { return (n + 255u) / 256u * 256u; }

}  // namespace

size_t route_bytes(const RouteArgs& a)
{
    const Plan p = plan_for(a);
    size_t table = 0;
    for (uint32_t i = 0; i < p.passes; ++i)
        if (p.it[i] == 0u) {
            const size_t need = round_up(4u * static_cast<size_t>(p.bins[i]) * p.blocks[i]) + round_up(4u * static_cast<size_t>(p.bins[i]));
            table = need > table ? need : table;
        }
    return table + (p.passes > 1u ? 2u * round_up(4u * static_cast<size_t>(a.pairs)) : 0u);
}

int launch_route(cudaStream_t st, const RouteArgs& a, void* work)
{
    const Plan plan = plan_for(a);
    int launches = 0;
    uint8_t* at = static_cast<uint8_t*>(work);
    uint32_t* order = nullptr; uint32_t* sorted = nullptr;
    if (plan.passes > 1u) {
        order = reinterpret_cast<uint32_t*>(at); at += round_up(4u * static_cast<size_t>(a.pairs));
        sorted = reinterpret_cast<uint32_t*>(at); at += round_up(4u * static_cast<size_t>(a.pairs));
    }
    for (uint32_t i = 0; i < plan.passes; ++i) {
        Pass p;
        p.a = a;
        p.shift = i * plan.low_bits; p.bins = plan.bins[i]; p.mask = plan.passes > 1u && i == 0u ? (1u << plan.low_bits) - 1u : 0xffffffffu;
        p.bits = 32u - __builtin_clz(p.bins);                // (bins - 1 may be the number of pairs without a member)
        p.counting = plan.counting[i]; p.per_warp = plan.per_warp[i]; p.blocks = plan.blocks[i];
        p.order_in = i ? order : nullptr;
        p.order_out = i + 1u < plan.passes ? order : nullptr;
        p.sorted = i ? sorted : nullptr;
        p.table = reinterpret_cast<uint32_t*>(at);
        p.totals = reinterpret_cast<uint32_t*>(at + round_up(4u * static_cast<size_t>(p.bins) * p.blocks));
        // warps that only help with the scans
        const uint32_t helping = p.bins > 2048u ? 32u : p.bins > 256u ? 8u : 1u, warps = p.counting > helping ? p.counting : helping;
        const size_t smem = 4u * static_cast<size_t>(p.counting + 2u) * p.bins;
        auto launch = [&](void (*kernel)(Pass), uint32_t blocks) {
            if (!has_room(kernel, smem)) return false;
            ++launches;
            return launch_dependent(kernel, dim3(blocks), dim3(warps * 32u), smem, st, p) == cudaSuccess;
        };
        if (plan.it[i]) {
            const cudaError_t e = p.blocks == 1u ? launch_once<1>(st, plan.it[i], warps * 32u, smem, p) : launch_once<kCluster>(st, plan.it[i], warps * 32u, smem, p);
            if (e != cudaSuccess) return -1;
            ++launches;
        } else {
            if (!launch(k_route<kCount>, p.blocks)) return -1;
            if (launch_dependent(k_route_scan, dim3((p.bins + 7u) / 8u), dim3(256), 0, st, p.table, p.totals, p.bins, p.blocks) != cudaSuccess) return -1;
            ++launches;
            if (!launch(k_route<kPlace>, p.blocks)) return -1;
        }
    }
    if (plan.passes > 1u) {
        if (launch_dependent(k_route_offsets, dim3(a.groups / 256u + 1u), dim3(256), 0, st, a, sorted) != cudaSuccess) return -1;
        ++launches;
    }
    return launches;
}

}  // namespace evo

// Newton-Schulz iteration of matrices of 33 to 128 rows and up to 1,024 columns (the shorter side counts as rows): all steps in one
// launch, a block or a cluster of up to eight for a matrix.
//
// A block holds up to 128 columns of X, as a pair of fp16 matrices in shared memory for the tensor core and in fp32 in the registers
// of the threads that update them.  A step is three products, each followed by what turns its sums into operands, and nothing of it
// overlaps: it is bound by that chain (128 x 128: 38 us, 5.75 a step; 64 x 64: 21 us).
// Blocks of a cluster each make the part of A that their columns give.  The parts go to their owners (block r adds up the r-th
// share of A's columns, all parts in the order of the blocks) and the sums, as fp16 pairs, to everybody, both as bulk copies between
// the blocks' shared memories; A^2 is then made by every block, B X for its own columns.  (Loads of the other blocks' parts by the
// threads took 8 us a step and block.)
#include "newton_schulz.cuh"

namespace evo {
namespace ns {

constexpr uint32_t kThreads = 512;
constexpr uint32_t kHalfCols = 128;                                        // tensor memory of an accumulator (512 threads of 119 to 128 registers: a block an SM)
constexpr uint32_t kItems = kSmallCols * kSmallRows / 8u / kThreads;       // eights of elements of a thread

__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();                                            // (.aligned: a warp comes to it as one)
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ void copy_to_block(uint32_t dst, uint32_t src, uint32_t bytes, uint32_t dst_bar)
{
    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 :: "r"(dst), "r"(src), "r"(bytes), "r"(dst_bar) : "memory");
}
__device__ __forceinline__ void expect(uint32_t bar, uint32_t bytes)
{
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" :: "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void touch8(uint32_t* u)
{
    asm volatile("" : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]));
}

// X in panels of mp rows, hi then lo; A, then B over it, the same way (before, this block's part of A in fp32); cluster: the other
// blocks' parts of this block's share; 2 KB that the products may read beyond (their first operand is always 128 rows; the rows from mp
// on are other data and give sums that nothing looks at).
template <uint32_t SRC, bool CLUSTER>
__global__ void __launch_bounds__(kThreads, 1) k_ns_small(const __grid_constant__ Args a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bar, drain, parts_bar, sums_bar;
    __shared__ uint32_t slot, limit;
    __shared__ volatile int abort_flag;
    __shared__ double red[kThreads / 32], total;
    const bool late = SRC == kMuon && a.late;
    if (!late) dep_wait();
    dep_trigger();
    if (SRC == kMuon && a.skip && __ldcg(a.skip) == 0.0) {
        if (late) dep_wait();
        return;
    }
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    const uint32_t blocks = CLUSTER ? a.cluster : 1u, rank = CLUSTER ? blockIdx.x % blocks : 0u, at_block = blockIdx.x / blocks;
    uint32_t gi = 0;
    while (gi + 1u < a.groups && at_block >= a.g[gi + 1u].first_block) ++gi;
    const Group& g = a.g[gi];
    const uint32_t which = at_block - g.first_block;
    // this block's columns: j_first and the n that follow
    const uint32_t m = g.m, mp = g.mp, np = g.np, j_first = rank * np, panel = mp * 16u, eights = mp / 8u;
    const uint32_t n = CLUSTER ? (j_first < g.n ? min(np, g.n - j_first) : 0u) : g.n;
    const uint32_t x_half = mp * np * 2u, q_half = mp * mp * 2u;
    uint8_t* const x_hi = smem;
    uint8_t* const x_lo = smem + x_half;
    uint8_t* const q_hi = smem + 2u * x_half;
    uint8_t* const q_lo = q_hi + q_half;
    uint8_t* const parts = q_lo + q_half;
    // the eights of A's columns that block r adds up: r each_owner ...
    const uint32_t each_owner = (eights + blocks - 1u) / blocks, share = each_owner * panel * 2u;
    auto owned = [&](uint32_t r) { return min(each_owner, eights - min(eights, r * each_owner)); };

    if (tid == 0) {
        mbar_init(smem_u32(&bar), 1);
        mbar_init(smem_u32(&drain), 1);
        mbar_init(smem_u32(&parts_bar), 1);
        mbar_init(smem_u32(&sums_bar), 1);
        mbar_init_fence();
        limit = a.wait_log2;
        abort_flag = 0;
    }
    // two accumulators of a product's columns, the large products' and the small ones'
    if (warp == 0) tmem_alloc(smem_u32(&slot), 2u * kHalfCols);

    // an item is eight j of one i; neighbouring lanes read neighbouring elements of the source
    const uint32_t jcs = np / 8u, items = jcs * mp;
    auto place = [&](uint32_t t, uint32_t& i, uint32_t& jc) {
        if (g.tall) { i = t % mp; jc = t / mp; }
        else { const uint32_t q = t / 8u; jc = q % jcs; i = q / jcs * 8u + t % 8u; }      // (mp is a multiple of 8)
    };
    float kept[kItems][8];
    double sum = 0.0;
#pragma unroll
    for (uint32_t c = 0; c < kItems; ++c) {
        const uint32_t t = tid + c * kThreads;
        uint32_t i, jc;
        place(t, i, jc);
        const uint32_t j = jc * 8u, count = t < items && i < m && j < n ? min(8u, n - j) : 0u;
        load8<SRC, true, true>(a, in_index(g, which, i, j_first + j), g.tall ? g.in_ld : 1u, count, kept[c]);
    }
#pragma unroll
    for (uint32_t c = 0; c < kItems; ++c)
#pragma unroll
        for (int e = 0; e < 8; ++e) sum += static_cast<double>(kept[c][e]) * kept[c][e];
    sum = block_sum<kThreads>(sum, red);
    if constexpr (CLUSTER) {
        if (tid == 0) total = sum;
        cluster_sync();
        sum = 0.0;
        for (uint32_t r = 0; r < blocks; ++r) {
            double part;
            asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(part) : "r"(in_block(smem_u32(&total), r)) : "memory");
            sum += part;
        }
    }
    uint32_t first_lift;
    const double scale = first_scale(a.s, sum, &first_lift);
#pragma unroll
    for (uint32_t c = 0; c < kItems; ++c) {
        const uint32_t t = tid + c * kThreads;
        uint32_t i, jc;
        place(t, i, jc);
        if (t < items) {
#pragma unroll
            for (int e = 0; e < 8; ++e) kept[c][e] = static_cast<float>(scale * kept[c][e]);
            uint4 hi, lo;
            split8(kept[c], hi, lo);
            *reinterpret_cast<uint4*>(x_hi + jc * panel + i * 16u) = hi;
            *reinterpret_cast<uint4*>(x_lo + jc * panel + i * 16u) = lo;
        }
    }
    const Waits waits{ &abort_flag, &limit, a.sticky };
    uint32_t phase = 0;
    auto finish = [&] {
        waits.wait(smem_u32(&bar), phase);
        phase ^= 1u;
        tc_fence_after();
    };
    // what the threads have written to shared memory is for the tensor core, what they have read of tensor memory may be overwritten
    auto hand_over = [&] {
        fence_async_smem();
        tc_fence_before();
        __syncthreads();
        tc_fence_after();
    };
    hand_over();
    const uint32_t tmem = slot;
    // descriptors of the first K-step of each operand, and what a step adds to them (in 16 bytes)
    const uint64_t x_k_hi = umma_smem_desc(smem_u32(x_hi), panel, 128u), x_k_lo = umma_smem_desc(smem_u32(x_lo), panel, 128u);
    const uint64_t x_m_hi = umma_smem_desc(smem_u32(x_hi), 128u, panel), x_m_lo = umma_smem_desc(smem_u32(x_lo), 128u, panel);
    const uint64_t q_k_hi = umma_smem_desc(smem_u32(q_hi), panel, 128u), q_k_lo = umma_smem_desc(smem_u32(q_lo), panel, 128u);
    const uint32_t k_step = panel / 8u, m_step = 16u;
    // (128 x N) = sum over K of the products of two pairs
    auto product = [&](uint32_t idesc, uint64_t ph, uint64_t pl, uint32_t p_step, uint64_t rh, uint64_t rl, uint32_t r_step, uint32_t K, bool drop = false) {
        if (abort_flag) return;
#pragma unroll 4
        for (uint32_t k = 0; k < K / 16u; ++k) {
            umma_bf16(tmem, ph, rh, idesc, k != 0u);
            umma_bf16(tmem + kHalfCols, ph, rl, idesc, k != 0u);
            umma_bf16(tmem + kHalfCols, pl, rh, idesc, 1u);
            ph += p_step; pl += p_step; rh += r_step; rl += r_step;
        }
        if (!drop) umma_commit(smem_u32(&bar));
    };
    // After a wait that ran out nothing is multiplied any more: what a block has in hand then, and what it sends to the others, is not a number.
    // (What the others have by the last exchange, and make of it, does not depend on this block any further.)
    auto sound = [&] { return abort_flag ? __int_as_float(0x7FC00000) : 1.0f; };
    const uint32_t row = (warp & 3u) * 32u + lane, lanes = (warp & 3u) << 21, part = warp >> 2;      // four warps share a quarter of the lanes
    const bool rows_live = (warp & 3u) * 32u < mp, row_live = row < mp;
    // this thread's eights of columns: 2 part + 8 t and the next, t = 0, 1, of A as of X
    auto mine = [&](uint32_t c) { return 2u * part + 8u * (c >> 1) + (c & 1u); };
    // sums of the eights mine(c) and mine(c + 1) (of the first alone where `two` is not set)
    auto sums = [&](uint32_t c, bool two, float (&x)[2][8], float cut) {
        uint32_t u[2][8], v[2][8];
        const uint32_t from = tmem + lanes + mine(c) * 8u;
        tmem_ld8_issue(from, u[0]);
        tmem_ld8_issue(from + kHalfCols, v[0]);
        if (two) {
            tmem_ld8_issue(from + 8u, u[1]);
            tmem_ld8_issue(from + kHalfCols + 8u, v[1]);
        }
        wait_loads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            touch8(u[h]);
            touch8(v[h]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[h][e] = __uint_as_float(u[h][e]) + fmaf(cut, __uint_as_float(u[h][e]), __uint_as_float(v[h][e]));
        }
    };
    auto put = [&](uint8_t* hi_at, uint8_t* lo_at, uint32_t c, const float (&x)[8]) {
        uint4 hi, lo;
        split8(x, hi, lo);
        if (row_live) {
            *reinterpret_cast<uint4*>(hi_at + mine(c) * panel + row * 16u) = hi;
            *reinterpret_cast<uint4*>(lo_at + mine(c) * panel + row * 16u) = lo;
        }
    };
    float x[kItems][8];
    if (rows_live)
#pragma unroll
        for (uint32_t c = 0; c < kItems; ++c)
            if (mine(c) < jcs && row_live)
                join8(*reinterpret_cast<const uint4*>(x_hi + mine(c) * panel + row * 16u), *reinterpret_cast<const uint4*>(x_lo + mine(c) * panel + row * 16u), x[c]);
    const float poly_c = a.s.c * a.s.s_b / (a.s.s_a * a.s.s_a), cut = kCut * static_cast<float>(np / 16u);

    for (uint32_t step = 0; step < a.s.steps; ++step) {
        const uint32_t lift = lift_at(a.s, first_lift, step), next_lift = lift_at(a.s, first_lift, step + 1u);
        const float unlift = power_of_two(-2 * static_cast<int>(lift)), to_a = unlift * (a.s.s_a / (a.s.s_x * a.s.s_x));
        const float poly_b = a.s.b * a.s.s_b / a.s.s_a;
        const float drop = power_of_two(static_cast<int>(next_lift) - static_cast<int>(lift)), next_a = drop * a.s.a, next_bx = drop / a.s.s_b;
        if (tid == 0) product(idesc_f16(128, mp, false), x_k_hi, x_k_lo, k_step, x_k_hi, x_k_lo, k_step, np, a.drop && blockIdx.x == 0u && step == 0u);
        finish();
        const float scale_a = to_a * sound();
        float gram[kItems][8];                                             // A times s_a
        if (rows_live)
#pragma unroll
            for (uint32_t c = 0; c < kItems; c += 2u)
                if (mine(c) < eights) {                                    // (eights is even)
                    float s[2][8];
                    sums(c, true, s, cut);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        gram[c][e] = scale_a * s[0][e];
                        gram[c + 1u][e] = scale_a * s[1][e];
                    }
                }
        if constexpr (!CLUSTER) {
            if (rows_live)
#pragma unroll
                for (uint32_t c = 0; c < kItems; ++c)
                    if (mine(c) < eights) put(q_hi, q_lo, c, gram[c]);
            hand_over();
        } else {
            // the parts lie where A will, fp32: eight floats of (column eight, row) side by side
            if (rows_live && row_live)
#pragma unroll
                for (uint32_t c = 0; c < kItems; ++c)
                    if (mine(c) < eights) {
                        float4* const p = reinterpret_cast<float4*>(q_hi + (mine(c) * mp + row) * 32u);
                        p[0] = make_float4(gram[c][0], gram[c][1], gram[c][2], gram[c][3]);
                        p[1] = make_float4(gram[c][4], gram[c][5], gram[c][6], gram[c][7]);
                    }
            hand_over();
            const uint32_t own = owned(rank) * panel * 2u;
            if (tid == 0) {
                expect(smem_u32(&parts_bar), own * (blocks - 1u));
                expect(smem_u32(&sums_bar), 2u * q_half);
            }
            // nobody sends before everybody expects it (and has done with the last step's)
            cluster_sync();
            if (tid < blocks && tid != rank && owned(tid))
                copy_to_block(in_block(smem_u32(parts) + rank * share, tid), smem_u32(q_hi) + tid * share, owned(tid) * panel * 2u, in_block(smem_u32(&parts_bar), tid));
            waits.wait(smem_u32(&parts_bar), step & 1u);
            // this block's share: the parts in the order of the blocks, and the sum as a pair to where this block's own part would be
            uint8_t* const stage = parts + rank * share;
            const float fill = sound() - 1.0f;                             // 0 or NaN
            for (uint32_t t = tid; t < owned(rank) * mp; t += kThreads) {
                float s[8] = { fill, fill, fill, fill, fill, fill, fill, fill };
                for (uint32_t r = 0; r < blocks; ++r) {
                    const float4* const p = reinterpret_cast<const float4*>((r == rank ? q_hi + rank * share : parts + r * share) + t * 32u);
                    const float4 u = p[0], v = p[1];
                    s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w; s[4] += v.x; s[5] += v.y; s[6] += v.z; s[7] += v.w;
                }
                uint4 hi, lo;
                split8(s, hi, lo);
                *reinterpret_cast<uint4*>(stage + t * 16u) = hi;           // (eight c, row: c panel + 16 row)
                *reinterpret_cast<uint4*>(stage + own / 2u + t * 16u) = lo;
            }
            fence_async_smem();
            cluster_sync();                                                // all parts have arrived: A may come over them
            if (tid < blocks && own) {
                const uint32_t to = rank * each_owner * panel, there = in_block(smem_u32(&sums_bar), tid);
                copy_to_block(in_block(smem_u32(q_hi) + to, tid), smem_u32(stage), own / 2u, there);
                copy_to_block(in_block(smem_u32(q_lo) + to, tid), smem_u32(stage) + own / 2u, own / 2u, there);
            }
            waits.wait(smem_u32(&sums_bar), step & 1u);
            if (rows_live && row_live)
#pragma unroll
                for (uint32_t c = 0; c < kItems; ++c)
                    if (mine(c) < eights)
                        join8(*reinterpret_cast<const uint4*>(q_hi + mine(c) * panel + row * 16u), *reinterpret_cast<const uint4*>(q_lo + mine(c) * panel + row * 16u), gram[c]);
            hand_over();
        }
        if (tid == 0) product(idesc_f16(128, mp, false), q_k_hi, q_k_lo, k_step, q_k_hi, q_k_lo, k_step, mp);      // (A is symmetric)
        finish();
        if (rows_live)
#pragma unroll
            for (uint32_t c = 0; c < kItems; c += 2u)
                if (mine(c) < eights) {
                    float s[2][8];
                    sums(c, true, s, 0.f);
#pragma unroll
                    for (uint32_t h = 0; h < 2u; ++h) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) s[h][e] = fmaf(poly_b, gram[c + h][e], poly_c * s[h][e]);
                        put(q_hi, q_lo, c + h, s[h]);
                    }
                }
        hand_over();
        if (tid == 0) product(idesc_f16(128, np, true), q_k_hi, q_k_lo, k_step, x_m_hi, x_m_lo, m_step, mp);
        finish();
        if (rows_live)
#pragma unroll
            for (uint32_t c = 0; c < kItems; c += 2u)
                if (mine(c) < jcs) {                                       // (jcs is even)
                    float s[2][8];
                    sums(c, true, s, 0.f);
#pragma unroll
                    for (uint32_t h = 0; h < 2u; ++h) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[c + h][e] = fmaf(next_a, x[c + h][e], next_bx * s[h][e]);
                        if (step + 1u < a.s.steps) put(x_hi, x_lo, c + h, x[c + h]);
                    }
                }
        hand_over();
    }
    const float back = sound() * power_of_two(-static_cast<int>(lift_at(a.s, first_lift, a.s.steps))) / a.s.s_x;
    if (g.tall) {
        // neighbouring lanes are neighbours in memory
        if (rows_live && row < m)
#pragma unroll
            for (uint32_t c = 0; c < kItems; ++c)
#pragma unroll
                for (uint32_t e = 0; e < 8u; ++e)
                    if (mine(c) < jcs && mine(c) * 8u + e < n) store<SRC, true>(a, out_index(g, which, row, j_first + mine(c) * 8u + e), x[c][e] * back, g.gain);
    } else {
        // by way of shared memory, where the pairs were: floats 0-3 of an eight in place of its high parts, 4-7 of the low ones; then 8 rows by 64
        // bytes a warp
        if (rows_live && row_live)
#pragma unroll
            for (uint32_t c = 0; c < kItems; ++c)
                if (mine(c) < jcs) {
                    *reinterpret_cast<float4*>(x_hi + mine(c) * panel + row * 16u) = make_float4(x[c][0] * back, x[c][1] * back, x[c][2] * back, x[c][3] * back);
                    *reinterpret_cast<float4*>(x_lo + mine(c) * panel + row * 16u) = make_float4(x[c][4] * back, x[c][5] * back, x[c][6] * back, x[c][7] * back);
                }
        __syncthreads();
        const uint32_t sixteens = np / 16u;
        for (uint32_t t = warp; t < sixteens * (mp / 8u); t += kThreads / 32u) {
            const uint32_t i = t / sixteens * 8u + (lane & 7u), q = lane >> 3, jc = t % sixteens * 2u + (q >> 1), j = jc * 8u + (q & 1u) * 4u;
            const float4 v = *reinterpret_cast<const float4*>((q & 1u ? x_lo : x_hi) + jc * panel + i * 16u);
            if (i < m && j < n) store4<SRC, true>(a, out_index(g, which, i, j_first + j), v, n - j, g.gain);
        }
    }
    if (abort_flag) {                                                      // no MMA may write after its tensor memory is freed
        if (tid == 0) umma_commit(smem_u32(&drain));
        mbar_wait_bounded(smem_u32(&drain), 0u, &limit);
        if (CLUSTER) {                                                     // nor a copy land in shared memory that is another block's by then
            mbar_wait_bounded(smem_u32(&parts_bar), (a.s.steps - 1u) & 1u, &limit);
            mbar_wait_bounded(smem_u32(&sums_bar), (a.s.steps - 1u) & 1u, &limit);
        }
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, 2u * kHalfCols);
    if constexpr (CLUSTER) cluster_sync();                                 // no copy between the blocks is left when one goes
    if (late) dep_wait();
}

template <bool CLUSTER>
static auto kernel_for(uint32_t source)
{
    return source == kF32 ? k_ns_small<kF32, CLUSTER> : source == kBf16 ? k_ns_small<kBf16, CLUSTER> : source == kF16 ? k_ns_small<kF16, CLUSTER> : k_ns_small<kMuon, CLUSTER>;
}

int launch_small(cudaStream_t st, uint32_t source, const Args& a, size_t smem)
{
    auto kernel = a.cluster > 1u ? kernel_for<true>(source) : kernel_for<false>(source);
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmallBytes)) != cudaSuccess) return -1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.blocks * a.cluster); cfg.blockDim = dim3(kThreads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = a.cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = a.cluster > 1u ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? 1 : -1;
}

}  // namespace ns
}  // namespace evo

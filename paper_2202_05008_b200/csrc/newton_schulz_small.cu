// Newton-Schulz iteration of matrices that fit the shared memory of an SM: one block each, all steps in one launch.
#include "newton_schulz.cuh"

namespace evo {
namespace ns {

constexpr uint32_t kThreads = 512;

// X in panels of mp rows, hi then lo; A, then B over it, the same way; 2 KB that the products may read beyond (their first operand is
// always 128 rows; the rows from mp on are other data and give sums that nothing looks at).
template <uint32_t SRC>
__global__ void __launch_bounds__(kThreads, 1) k_ns_small(const __grid_constant__ Args a)
{
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ __align__(8) uint64_t bar, drain;
    __shared__ uint32_t slot, limit;
    __shared__ volatile int abort_flag;
    __shared__ double red[kThreads / 32];
    dep_wait();
    dep_trigger();
    if (SRC == kMuon && a.skip && *a.skip == 0.0) return;
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
    uint32_t gi = 0;
    while (gi + 1u < a.groups && blockIdx.x >= a.g[gi + 1u].first_block) ++gi;
    const Group& g = a.g[gi];
    const uint32_t which = blockIdx.x - g.first_block;
    const uint32_t m = g.m, n = g.n, mp = g.mp, np = g.np, panel = mp * 16u;
    const uint32_t x_half = mp * np * 2u, q_half = mp * mp * 2u;
    uint8_t* const x_hi = smem;
    uint8_t* const x_lo = smem + x_half;
    uint8_t* const q_hi = smem + 2u * x_half;
    uint8_t* const q_lo = q_hi + q_half;

    if (tid == 0) { mbar_init(smem_u32(&bar), 1); mbar_init(smem_u32(&drain), 1); mbar_init_fence(); limit = a.wait_log2; abort_flag = 0; }
    // two accumulators of a product's columns, the large products' and the small ones'; no more tensor memory than that, so that small
    // matrices share an SM
    const uint32_t widest = max(mp, min(np, 256u));
    const uint32_t half_cols = widest <= 32u ? 32u : widest <= 64u ? 64u : widest <= 128u ? 128u : 256u, cols = 2u * half_cols;
    if (warp == 0) tmem_alloc(smem_u32(&slot), cols);

    // an item is eight j of one i; neighbouring lanes read neighbouring elements of the source
    const uint32_t jcs = np / 8u, items = jcs * mp;
    auto place = [&](uint32_t t, uint32_t& i, uint32_t& jc) {
        if (g.tall) { i = t % mp; jc = t / mp; }
        else { const uint32_t r = t % 8u, q = t / 8u; jc = q % jcs; i = q / jcs * 8u + r; }      // (mp is a multiple of 8)
    };
    double sum = 0.0;
    for (uint32_t t = tid; t < items; t += kThreads) {
        uint32_t i, jc;
        place(t, i, jc);
        if (i >= m) continue;
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            float unused;
            const uint32_t j = jc * 8u + e;
            const double x = j < n ? load<SRC>(a, in_index(g, which, i, j), &unused) : 0.f;
            sum += x * x;
        }
    }
    sum = block_sum<kThreads>(sum, red);
    uint32_t first_lift;
    const double scale = first_scale(a.s, sum, &first_lift);
    for (uint32_t t = tid; t < items; t += kThreads) {
        uint32_t i, jc;
        place(t, i, jc);
        float x[8];
#pragma unroll
        for (uint32_t e = 0; e < 8u; ++e) {
            const uint32_t j = jc * 8u + e;
            x[e] = 0.f;
            if (i < m && j < n) {
                const uint64_t at = in_index(g, which, i, j);
                float momentum;
                x[e] = static_cast<float>(scale * load<SRC>(a, at, &momentum));
                if constexpr (SRC == kMuon) store_moments(a, at, momentum);
            }
        }
        uint4 hi, lo;
        split8(x, hi, lo);
        *reinterpret_cast<uint4*>(x_hi + jc * panel + i * 16u) = hi;
        *reinterpret_cast<uint4*>(x_lo + jc * panel + i * 16u) = lo;
    }
    fence_async_smem();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = slot;
    const Waits waits{ &abort_flag, &limit, a.sticky };
    uint32_t phase = 0;
    // (128 x N) = sum over K of the products of two pairs; operands from the byte addresses on, K-adjacent core matrices ks
    // bytes apart, those along M (N) ms bytes
    auto product = [&](uint32_t idesc, uint32_t p_hi, uint32_t p_lo, uint32_t p_ks, uint32_t p_ms, uint32_t r_hi, uint32_t r_lo,
                       uint32_t r_ks, uint32_t r_ms, uint32_t K) {
        if (abort_flag) return;
        for (uint32_t k = 0; k < K / 16u; ++k) {
            const uint64_t ph = umma_smem_desc(p_hi + 2u * k * p_ks, p_ks, p_ms), pl = umma_smem_desc(p_lo + 2u * k * p_ks, p_ks, p_ms);
            const uint64_t rh = umma_smem_desc(r_hi + 2u * k * r_ks, r_ks, r_ms), rl = umma_smem_desc(r_lo + 2u * k * r_ks, r_ks, r_ms);
            umma_bf16(tmem, ph, rh, idesc, k != 0u);
            umma_bf16(tmem + half_cols, ph, rl, idesc, k != 0u);
            umma_bf16(tmem + half_cols, pl, rh, idesc, 1u);
            umma_bf16(tmem + half_cols, pl, rl, idesc, 1u);      // (the squares on A's diagonal would all miss it)
        }
        umma_commit(smem_u32(&bar));
    };
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
    const uint32_t row = (warp & 3u) * 32u + lane, lanes = (warp & 3u) << 21, part = warp >> 2;      // four warps share a quarter of the lanes
    const bool rows_live = (warp & 3u) * 32u < mp, row_live = row < mp;
    auto sums8 = [&](uint32_t c, float (&x)[8], float cut = 0.f) {
        uint32_t u[8], v[8];
        tmem_ld8_issue(tmem + lanes + c * 8u, u);
        tmem_ld8_issue(tmem + half_cols + lanes + c * 8u, v);
        asm volatile("tcgen05.wait::ld.sync.aligned;"
                     : "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]),
                       "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]) :: "memory");
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = __uint_as_float(u[e]) + fmaf(cut, __uint_as_float(u[e]), __uint_as_float(v[e]));
    };
    auto put_q = [&](uint32_t c, const float (&x)[8]) {
        uint4 hi, lo;
        split8(x, hi, lo);
        if (row_live) {
            *reinterpret_cast<uint4*>(q_hi + c * panel + row * 16u) = hi;
            *reinterpret_cast<uint4*>(q_lo + c * panel + row * 16u) = lo;
        }
        __syncwarp();
    };
    const uint32_t xh = smem_u32(x_hi), xl = smem_u32(x_lo), qh = smem_u32(q_hi), ql = smem_u32(q_lo);
    const float poly_c = a.s.c * a.s.s_b / (a.s.s_a * a.s.s_a), from_bx = 1.0f / a.s.s_b;

    for (uint32_t step = 0; step < a.s.steps; ++step) {
        const bool last = step + 1u == a.s.steps;
        const uint32_t lift = lift_at(a.s, first_lift, step), next_lift = lift_at(a.s, first_lift, step + 1u);
        const float unlift = power_of_two(-2 * static_cast<int>(lift)), to_a = unlift * (a.s.s_a / (a.s.s_x * a.s.s_x));
        const float poly_b = unlift * (a.s.b * a.s.s_b / (a.s.s_x * a.s.s_x));
        const float drop = power_of_two(static_cast<int>(next_lift) - static_cast<int>(lift));
        float gram[4][8];                                                  // columns 8 (part + 4 c) of this row
        for (uint32_t k0 = 0; k0 < np; k0 += kChunk) {
            if (tid == 0)
                product(idesc_f16(128, mp, false), xh + k0 / 8u * panel, xl + k0 / 8u * panel, panel, 128u, xh + k0 / 8u * panel,
                        xl + k0 / 8u * panel, panel, 128u, min(kChunk, np - k0));
            finish();
            if (rows_live)
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c)
                    if (part + 4u * c < mp / 8u) {
                        float x[8];
                        sums8(part + 4u * c, x, kCut * static_cast<float>(min(kChunk, np - k0) / 16u));
#pragma unroll
                        for (int e = 0; e < 8; ++e) gram[c][e] = k0 == 0u ? x[e] : gram[c][e] + x[e];
                    }
            if (k0 + kChunk < np) hand_over();
        }
        if (rows_live)
#pragma unroll
            for (uint32_t c = 0; c < 4u; ++c)
                if (part + 4u * c < mp / 8u) {
                    float x[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = to_a * gram[c][e];
                    put_q(part + 4u * c, x);
                }
        hand_over();
        if (tid == 0) product(idesc_f16(128, mp, false), qh, ql, panel, 128u, qh, ql, panel, 128u, mp);      // (A is symmetric)
        finish();
        if (rows_live)
#pragma unroll
            for (uint32_t c = 0; c < 4u; ++c)
                if (part + 4u * c < mp / 8u) {
                    float x[8];
                    sums8(part + 4u * c, x);
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[e] = fmaf(poly_b, gram[c][e], poly_c * x[e]);
                    put_q(part + 4u * c, x);
                }
        hand_over();
        for (uint32_t j0 = 0; j0 < np; j0 += 256u) {                       // columns of X do not mix
            const uint32_t w = min(256u, np - j0);
            if (tid == 0)
                product(idesc_f16(128, w, true), qh, ql, panel, 128u, xh + j0 / 8u * panel, xl + j0 / 8u * panel, 128u, panel, mp);
            finish();
            if (rows_live)
                for (uint32_t c = part; c < w / 8u; c += 4u) {
                    float s[8];
                    sums8(c, s);
                    if (row_live) {
                        uint4* const ph = reinterpret_cast<uint4*>(x_hi + (j0 / 8u + c) * panel + row * 16u);
                        uint4* const pl = reinterpret_cast<uint4*>(x_lo + (j0 / 8u + c) * panel + row * 16u);
                        float x[8];
                        join8(*ph, *pl, x);
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[e] = drop * fmaf(a.s.a, x[e], from_bx * s[e]);
                        if (!last) {
                            uint4 hi, lo;
                            split8(x, hi, lo);
                            *ph = hi;
                            *pl = lo;
                        } else if (row < m) {
                            const float back = abort_flag ? __int_as_float(0x7FC00000) : power_of_two(-static_cast<int>(next_lift)) / a.s.s_x;
#pragma unroll
                            for (uint32_t e = 0; e < 8u; ++e) {
                                const uint32_t j = j0 + c * 8u + e;
                                if (j < n) store<SRC>(a, out_index(g, which, row, j), x[e] * back, g.gain);
                            }
                        }
                    }
                    __syncwarp();
                }
            hand_over();
        }
    }
    if (abort_flag) {                                                      // no MMA may write after its tensor memory is freed
        if (tid == 0) umma_commit(smem_u32(&drain));
        mbar_wait_bounded(smem_u32(&drain), 0u, &limit);
    }
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem, cols);
}

int launch_small(cudaStream_t st, uint32_t source, const Args& a, size_t smem)
{
    void (*kernel)(const Args) = source == kF32 ? k_ns_small<kF32> : source == kBf16 ? k_ns_small<kBf16> : source == kF16 ? k_ns_small<kF16> : k_ns_small<kMuon>;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmallBytes)) != cudaSuccess) return -1;
    return launch_dependent(kernel, dim3(a.blocks), dim3(kThreads), smem, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace ns
}  // namespace evo

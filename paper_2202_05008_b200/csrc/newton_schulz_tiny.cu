// Newton-Schulz iteration of matrices of up to 32 rows (the shorter side counts as rows): all steps in one launch, X in registers
// (of the instances for 17 to 32 rows, 56 bytes a thread are spilled in clusters and 188 without).
//
// A warp owns 16 columns of X at a time, in the layout of an mma.sync accumulator (a lane has two neighbouring columns of rows g and
// g + 8, g = lane / 4).  Packed, that is the first operand of X X' and, rows 0-7 and 8-15 apart, also the second; transposed within
// the warp (movmatrix) it is the second operand of B X, whose result comes out in the layout that X has.  The warps' parts of A are
// added up in their order through shared memory, the blocks' of a cluster over distributed shared memory; then every warp has all of
// A and makes A^2 and B for itself.  A step is two barriers and a few dozen MMAs long
// and bound by the latency of its instructions (16 x 16: 1.46 us a step; 12 x 512, five steps: 16.9 us with its launch).
#include "grouped_mma.cuh"
#include "newton_schulz.cuh"

namespace evo {
namespace ns {

// an 8 x 8 matrix of halves held by a warp, transposed
__device__ __forceinline__ uint32_t turned(uint32_t x)
{
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ void cluster_sync_all()
{
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
template <typename T>
__device__ __forceinline__ T load_from_block(const T* p, uint32_t rank)
{
    uint32_t at;
    T v;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(smem_u32(p)), "r"(rank));
    if constexpr (sizeof(T) == 8) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(at) : "memory");
    else asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}

// 16 x 16 numbers in accumulator layout, v[8 columns][4], as the packed pairs of a first operand
struct Pair16 { uint32_t hi[4], lo[4]; };
__device__ __forceinline__ Pair16 pack(const float (&v)[2][4])
{
    Pair16 p;
    split2(v[0][0], v[0][1], p.hi[0], p.lo[0]);
    split2(v[0][2], v[0][3], p.hi[1], p.lo[1]);
    split2(v[1][0], v[1][1], p.hi[2], p.lo[2]);
    split2(v[1][2], v[1][3], p.hi[3], p.lo[3]);
    return p;
}
// large += hi hi', small += the three other products; b0, b1: the second operand's registers
__device__ __forceinline__ void products(float (&large)[4], float (&small)[4], const Pair16& p, uint32_t h0, uint32_t h1, uint32_t l0, uint32_t l1)
{
    gm::mma_16<__half>(large, p.hi, h0, h1);
    gm::mma_16<__half>(small, p.hi, l0, l1);
    gm::mma_16<__half>(small, p.lo, h0, h1);
    gm::mma_16<__half>(small, p.lo, l0, l1);
}

// MT: sixteens of rows; KT: sixteens of columns of a warp
template <uint32_t SRC, uint32_t MT, bool CLUSTER>
__global__ void __launch_bounds__(512) k_ns_tiny(const __grid_constant__ Args a)
{
    constexpr uint32_t KT = 4u / MT, V = MT * 2u * MT * 4u;         // V: numbers of A that a lane has
    extern __shared__ __align__(16) float parts[];                                  // [warps][V][32]
    __shared__ float sums[2][V][32];                                                // of a step and of the next (cluster)
    __shared__ double squares[16], total;
    const bool late = SRC == kMuon && a.late;
    if (!late) dep_wait();
    dep_trigger();
    if (SRC == kMuon && a.skip && __ldcg(a.skip) == 0.0) {
        if (late) dep_wait();
        return;
    }
    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, warps = blockDim.x >> 5, r = lane >> 2, q = lane & 3u;
    const uint32_t blocks = CLUSTER ? a.cluster : 1u, rank = CLUSTER ? blockIdx.x % blocks : 0u, at_block = blockIdx.x / blocks;
    uint32_t gi = 0;
    while (gi + 1u < a.groups && at_block >= a.g[gi + 1u].first_block) ++gi;
    const Group& g = a.g[gi];
    const uint32_t which = at_block - g.first_block, m = g.m, j_first = rank * g.np;
    const uint32_t n = CLUSTER ? (j_first < g.n ? min(g.np, g.n - j_first) : 0u) : g.n;

    // x[mt][kt][h][c]: rows 16 mt + r (c < 2) and + 8, columns 16 (warp + warps kt) + 8 h + 2 q + (c & 1)
    float x[MT][KT][2][4];
    double sum = 0.0;
#pragma unroll
    for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
        for (uint32_t kt = 0; kt < KT; ++kt)
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c) {
                    const uint32_t i = 16u * mt + r + 8u * (c >> 1), j = 16u * (warp + warps * kt) + 8u * h + 2u * q + (c & 1u);
                    x[mt][kt][h][c] = 0.f;
                    if (i < m && j < n) {
                        const uint64_t at = in_index(g, which, i, j_first + j);
                        float momentum;
                        x[mt][kt][h][c] = load<SRC, true>(a, at, &momentum);
                        if constexpr (SRC == kMuon) store_moments<true>(a, at, momentum);
                    }
                }
#pragma unroll
    for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
        for (uint32_t kt = 0; kt < KT; ++kt)
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c) sum += static_cast<double>(x[mt][kt][h][c]) * x[mt][kt][h][c];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if (lane == 0) squares[warp] = sum;
    __syncthreads();
    sum = 0.0;
    for (uint32_t w = 0; w < warps; ++w) sum += squares[w];
    if constexpr (CLUSTER) {
        if (tid == 0) total = sum;
        cluster_sync_all();
        sum = 0.0;
        for (uint32_t b = 0; b < blocks; ++b) sum += load_from_block(&total, b);
    }
    uint32_t first_lift;
    const double scale = first_scale(a.s, sum, &first_lift);
#pragma unroll
    for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
        for (uint32_t kt = 0; kt < KT; ++kt)
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c) x[mt][kt][h][c] = static_cast<float>(scale * x[mt][kt][h][c]);

    const uint32_t tiles = (n + 15u) / 16u, own = tiles > warp ? min(KT, (tiles - warp + warps - 1u) / warps) : 0u;
    const float poly_b = a.s.b * a.s.s_b / a.s.s_a, poly_c = a.s.c * a.s.s_b / (a.s.s_a * a.s.s_a);
    for (uint32_t step = 0; step < a.s.steps; ++step) {
        const uint32_t lift = lift_at(a.s, first_lift, step), next_lift = lift_at(a.s, first_lift, step + 1u);
        const float to_a = power_of_two(-2 * static_cast<int>(lift)) * (a.s.s_a / (a.s.s_x * a.s.s_x));
        const float drop = power_of_two(static_cast<int>(next_lift) - static_cast<int>(lift)), next_a = drop * a.s.a, next_bx = drop / a.s.s_b;
        // this warp's part of A
        {
            float large[MT][2 * MT][4] = {}, small[MT][2 * MT][4] = {};
#pragma unroll
            for (uint32_t kt = 0; kt < KT; ++kt)
                if (kt < own) {
                    Pair16 p[MT];
#pragma unroll
                    for (uint32_t mt = 0; mt < MT; ++mt) p[mt] = pack(x[mt][kt]);
#pragma unroll
                    for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
                        for (uint32_t nt = 0; nt < 2u * MT; ++nt) {
                            const Pair16& s = p[nt / 2u];
                            const uint32_t f = nt & 1u;
                            products(large[mt][nt], small[mt][nt], p[mt], s.hi[f], s.hi[f + 2u], s.lo[f], s.lo[f + 2u]);
                        }
                }
            const float cut = kCut * static_cast<float>(own);
#pragma unroll
            for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
                for (uint32_t nt = 0; nt < 2u * MT; ++nt)
#pragma unroll
                    for (uint32_t c = 0; c < 4u; ++c)
                        parts[(warp * V + (mt * 2u * MT + nt) * 4u + c) * 32u + lane] = to_a * (large[mt][nt][c] + fmaf(cut, large[mt][nt][c], small[mt][nt][c]));
        }
        __syncthreads();
        float (*const all)[32] = sums[step & 1u];
        for (uint32_t t = tid; t < V * 32u; t += blockDim.x) {
            float s = 0.f;
            for (uint32_t w = 0; w < warps; ++w) s += parts[w * V * 32u + t];
            (&all[0][0])[t] = s;
        }
        if constexpr (CLUSTER) cluster_sync_all(); else __syncthreads();
        float A[MT][2 * MT][4];
#pragma unroll
        for (uint32_t v = 0; v < V; ++v) {
            float s = 0.f;
            if constexpr (CLUSTER)
                for (uint32_t b = 0; b < blocks; ++b) s += load_from_block(&all[v][lane], b);
            else
                s = all[v][lane];
            A[v / (8u * MT)][v / 4u % (2u * MT)][v % 4u] = s;
        }
        // B = b A + c A^2, as pairs
        Pair16 bp[MT][MT];
        {
            Pair16 ap[MT][MT];
#pragma unroll
            for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
                for (uint32_t k = 0; k < MT; ++k) {
                    const float v[2][4] = { { A[mt][2 * k][0], A[mt][2 * k][1], A[mt][2 * k][2], A[mt][2 * k][3] },
                                            { A[mt][2 * k + 1][0], A[mt][2 * k + 1][1], A[mt][2 * k + 1][2], A[mt][2 * k + 1][3] } };
                    ap[mt][k] = pack(v);
                }
#pragma unroll
            for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
                for (uint32_t k = 0; k < MT; ++k) {
                    float v[2][4];
#pragma unroll
                    for (uint32_t h = 0; h < 2u; ++h) {
                        float large[4] = {}, small[4] = {};
#pragma unroll
                        for (uint32_t z = 0; z < MT; ++z) {                        // (A is symmetric: row block k is its column block)
                            const Pair16& s = ap[k][z];
                            products(large, small, ap[mt][z], s.hi[h], s.hi[h + 2u], s.lo[h], s.lo[h + 2u]);
                        }
#pragma unroll
                        for (uint32_t c = 0; c < 4u; ++c) v[h][c] = fmaf(poly_b, A[mt][2u * k + h][c], poly_c * (large[c] + small[c]));
                    }
                    bp[mt][k] = pack(v);
                }
        }
        // x <- a x + B x
#pragma unroll
        for (uint32_t kt = 0; kt < KT; ++kt)
            if (kt < own) {
                Pair16 p[MT];
#pragma unroll
                for (uint32_t mt = 0; mt < MT; ++mt) {
                    p[mt] = pack(x[mt][kt]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) { p[mt].hi[c] = turned(p[mt].hi[c]); p[mt].lo[c] = turned(p[mt].lo[c]); }
                }
#pragma unroll
                for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (uint32_t h = 0; h < 2u; ++h) {
                        float large[4] = {}, small[4] = {};
#pragma unroll
                        for (uint32_t z = 0; z < MT; ++z)
                            products(large, small, bp[mt][z], p[z].hi[2u * h], p[z].hi[2u * h + 1u], p[z].lo[2u * h], p[z].lo[2u * h + 1u]);
#pragma unroll
                        for (uint32_t c = 0; c < 4u; ++c) x[mt][kt][h][c] = fmaf(next_a, x[mt][kt][h][c], next_bx * (large[c] + small[c]));
                    }
            }
    }
    const float back = power_of_two(-static_cast<int>(lift_at(a.s, first_lift, a.s.steps))) / a.s.s_x;
#pragma unroll
    for (uint32_t mt = 0; mt < MT; ++mt)
#pragma unroll
        for (uint32_t kt = 0; kt < KT; ++kt)
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h)
#pragma unroll
                for (uint32_t c = 0; c < 4u; ++c) {
                    const uint32_t i = 16u * mt + r + 8u * (c >> 1), j = 16u * (warp + warps * kt) + 8u * h + 2u * q + (c & 1u);
                    if (i < m && j < n) store<SRC, true>(a, out_index(g, which, i, j_first + j), back * x[mt][kt][h][c], g.gain);
                }
    if constexpr (CLUSTER) cluster_sync_all();                                      // nobody reads a block's sums after it has gone
    if (late) dep_wait();
}

template <uint32_t MT, bool CLUSTER>
static auto kernel_for(uint32_t source)
{
    return source == kF32 ? k_ns_tiny<kF32, MT, CLUSTER> : source == kBf16 ? k_ns_tiny<kBf16, MT, CLUSTER> : source == kF16 ? k_ns_tiny<kF16, MT, CLUSTER> : k_ns_tiny<kMuon, MT, CLUSTER>;
}

int launch_tiny(cudaStream_t st, uint32_t source, const Args& a, uint32_t row_tiles, uint32_t warps)
{
    auto kernel = a.cluster > 1u ? (row_tiles == 1u ? kernel_for<1, true>(source) : kernel_for<2, true>(source))
                                 : (row_tiles == 1u ? kernel_for<1, false>(source) : kernel_for<2, false>(source));
    const size_t smem = static_cast<size_t>(warps) * row_tiles * row_tiles * 8u * 32u * sizeof(float);
    // (48 KB without this is what a block may have in all, the 8 KB of its sums included)
    if (smem > 32u * 1024u && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 64 * 1024) != cudaSuccess) return -1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.blocks * a.cluster); cfg.blockDim = dim3(warps * 32u); cfg.dynamicSmemBytes = smem; cfg.stream = st;
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

// Gradients of the products grouped by member: dx[r] = W_g' dz[r], dW_g = sum_r dz[r] x[r]', db_g = sum_r dz[r]; any type, size, stride and alignment.
//
// A group of a population has few rows and weights of its own: dx is bound by the weights' way from memory, dW by its own way there.  k_rows reads
// a group's weights once for up to 8 or 16 rows; k_weights makes tiles of 64 outputs x 64 or 128 inputs, or narrow ones.  Where there are too few tiles for the
// GPU, what is summed over (dx: weight rows, dW and db: rows) is split and the parts added up in a fixed order.  4,096 members of 128 x 128, 16,384 ragged rows, fp32: k_rows 60 us (4.7 TB/s; reading the
// weights alone is 41), k_weights 80 (its stores alone 40; the rest is what a block waits for before it stores), all together, overlapped, 135.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cmath>
#include <cstring>
#include <type_traits>

#include "async.cuh"
#include "grouped_gradient.h"
#include "grouped_mma.cuh"

namespace evo {
namespace {

template <typename T> __device__ __forceinline__ float to_float(T x)
{
    if constexpr (std::is_same<T, float>::value) return x;
    else if constexpr (std::is_same<T, __half>::value) return __half2float(x);
    else return __bfloat162float(x);
}
template <typename T> __device__ __forceinline__ T from_float(float x)
{
    if constexpr (std::is_same<T, float>::value) return x;
    else if constexpr (std::is_same<T, __half>::value) return __float2half_rn(x);
    else return __float2bfloat16_rn(x);
}
// Four numbers that are stored together.
template <typename T>
__device__ __forceinline__ void store4(T* p, const float (&v)[4])
{
    T raw[4];
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) raw[i] = from_float<T>(v[i]);
    if constexpr (sizeof(T) == 4) { uint4 u; memcpy(&u, raw, 16); *reinterpret_cast<uint4*>(p) = u; }
    else { uint2 u; memcpy(&u, raw, 8); *reinterpret_cast<uint2*>(p) = u; }
}

// ---- dx ----
// Warp-level products: the columns of the weights are the MMA's first operand, 16 bytes of them a lane (a warp has 32 of fp32, 64 of 16 bits), and 8 or 16 of a
// group's rows the second.  A lane takes pieces of eight weight rows into what becomes operand registers; the order of the contracted index is free as
// long as both operands share it.  fp32 numbers are two tf32 numbers each, dz of 16-bit types is one or two numbers (hi and lo), split once where it is staged in shared memory.
// The tensor core cuts its sums off, so they are taken out every 64 (fp32) or 128 weight rows and added up in fp32.
// What counts is that enough weights are under way: where they are aligned, 64 of their rows x 512 bytes are copied to shared memory asynchronously, five blocks an SM (four
// with 16 rows at a time).  Further rows are other blocks' (layers), and so are, in a group of few tiles, parts of a long column of weights (splits).
// Where there are too few tiles for the GPU a block's warps share one and split the weight rows.
constexpr uint32_t kRowWarps = 4, kStepK = 32;

template <typename T> struct Tile {
    static constexpr uint32_t kColumns = 16u / sizeof(T);             // of a lane
    static constexpr uint32_t kTiles = kColumns / 2u;                 // 16 x 8 products side by side
    static constexpr uint32_t kWarpColumns = 8u * kColumns;
    static constexpr uint32_t kAcross = kWarpColumns * kRowWarps;     // 512 bytes
    static __host__ __device__ constexpr uint32_t pitch(uint32_t chunk) { return chunk + 64u / sizeof(T); }      // of a staged row: 16 words modulo 32, so that eight lanes' pieces meet no bank twice
    static constexpr uint32_t kWeightPitch = kAcross + 32u / sizeof(T);      // of a staged weight row: 8 words modulo 32, the same for lanes of four rows
    // Piece j of lane (g, q) is weight row `row_of(j)` of a step, and where a lane finds its rows of dz beside each other: the j-th of lane q at place `place_of(row)`.
    static __device__ __forceinline__ constexpr uint32_t row_of(uint32_t j, uint32_t q) { return sizeof(T) == 4 ? 16u * (j / 4u) + 4u * (j % 4u) + q : 4u * j + q; }
    static __device__ __forceinline__ constexpr uint32_t place_of(uint32_t row)
    {
        return sizeof(T) == 4 ? row / 16u * 16u + row % 4u * 4u + row / 4u % 4u : row / 32u * 32u + row % 4u * 8u + row / 4u % 8u;
    }
};

// kStepK weight rows from k on, columns kColumns g ... of those from w on
template <typename T, bool VEC>
__device__ __forceinline__ void load_step(const T* w, uint64_t ld, uint32_t k, uint32_t end, uint32_t columns, uint4 (&v)[8])
{
    const uint32_t g = (threadIdx.x & 31u) >> 2, q = threadIdx.x & 3u;
    constexpr uint32_t C = Tile<T>::kColumns;
#pragma unroll
    for (uint32_t j = 0; j < 8u; ++j) {
        const uint32_t row = k + Tile<T>::row_of(j, q);
        v[j] = make_uint4(0u, 0u, 0u, 0u);
        if (row >= end) continue;
        const T* const from = w + static_cast<uint64_t>(row) * ld + C * g;
        if constexpr (VEC) {
            if (C * g < columns) v[j] = __ldg(reinterpret_cast<const uint4*>(from));
        } else {
            T n[C];
#pragma unroll
            for (uint32_t i = 0; i < C; ++i) n[i] = C * g + i < columns ? from[i] : from_float<T>(0.f);
            memcpy(&v[j], n, 16);
        }
    }
}

// c[tile]: columns (2 tile) and (2 tile + 1) of the lane's, rows 2q and 2q + 1
template <typename T>
struct Sums {
    float c[Tile<T>::kTiles][4], part[Tile<T>::kTiles][4], small[std::is_same<T, float>::value ? Tile<T>::kTiles : 1u][4];

    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (uint32_t m = 0; m < Tile<T>::kTiles; ++m)
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                c[m][i] = part[m][i] = 0.f;
                if constexpr (std::is_same<T, float>::value) small[m][i] = 0.f;
            }
    }
    __device__ __forceinline__ void take_out()
    {
#pragma unroll
        for (uint32_t m = 0; m < Tile<T>::kTiles; ++m)
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) {
                c[m][i] += part[m][i];
                part[m][i] = 0.f;
            }
    }
};
// weight rows [k, k + 32) of the chunk whose dz is staged in `hi` and `lo`, added to the parts of 8 rows, or of EIGHTS times as many where there are more
template <typename T, uint32_t EIGHTS>
__device__ __forceinline__ void step(const uint4 (&v)[8], const T* hi, const T* lo, uint32_t pitch, bool two, bool more, uint32_t k, Sums<T> (&sums)[EIGHTS])
{
    const uint32_t g = (threadIdx.x & 31u) >> 2, q = threadIdx.x & 3u;
    if constexpr (std::is_same<T, float>::value) {
#pragma unroll
        for (uint32_t s = 0; s < 2u; ++s) {
            uint4 bh[EIGHTS], bl[EIGHTS];
#pragma unroll
            for (uint32_t e = 0; e < EIGHTS; ++e) {
                bh[e] = *reinterpret_cast<const uint4*>(hi + (8u * e + g) * pitch + k + 16u * s + 4u * q);
                bl[e] = *reinterpret_cast<const uint4*>(lo + (8u * e + g) * pitch + k + 16u * s + 4u * q);
            }
#pragma unroll
            for (uint32_t h = 0; h < 2u; ++h) {              // weight rows 4q + 2h and 4q + 2h + 1
                const uint4 x = v[4u * s + 2u * h], y = v[4u * s + 2u * h + 1u];
                const uint32_t xs[4] = { x.x, x.y, x.z, x.w }, ys[4] = { y.x, y.y, y.z, y.w };
#pragma unroll
                for (uint32_t m = 0; m < 2u; ++m) {
                    uint32_t ah[4], al[4];
                    gm::split(__uint_as_float(xs[2u * m]), ah[0], al[0]);
                    gm::split(__uint_as_float(xs[2u * m + 1u]), ah[1], al[1]);
                    gm::split(__uint_as_float(ys[2u * m]), ah[2], al[2]);
                    gm::split(__uint_as_float(ys[2u * m + 1u]), ah[3], al[3]);
#pragma unroll
                    for (uint32_t e = 0; e < EIGHTS; ++e) {
                        if (e && !more) continue;
                        const uint32_t h0 = h ? bh[e].z : bh[e].x, h1 = h ? bh[e].w : bh[e].y, l0 = h ? bl[e].z : bl[e].x, l1 = h ? bl[e].w : bl[e].y;
                        gm::mma_tf32(sums[e].part[m], ah, h0, h1);
                        gm::mma_tf32(sums[e].small[m], ah, l0, l1);
                        gm::mma_tf32(sums[e].small[m], al, h0, h1);
                    }
                }
            }
        }
    } else {
        uint4 bh[EIGHTS], bl[EIGHTS];
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) {
            bh[e] = *reinterpret_cast<const uint4*>(hi + (8u * e + g) * pitch + k + 8u * q);
            if (two) bl[e] = *reinterpret_cast<const uint4*>(lo + (8u * e + g) * pitch + k + 8u * q);
        }
#pragma unroll
        for (uint32_t h = 0; h < 2u; ++h) {                  // weight rows 8q + 4h ... 8q + 4h + 3
            const uint32_t w[4][4] = { { v[4 * h].x, v[4 * h].y, v[4 * h].z, v[4 * h].w }, { v[4 * h + 1].x, v[4 * h + 1].y, v[4 * h + 1].z, v[4 * h + 1].w },
                                       { v[4 * h + 2].x, v[4 * h + 2].y, v[4 * h + 2].z, v[4 * h + 2].w }, { v[4 * h + 3].x, v[4 * h + 3].y, v[4 * h + 3].z, v[4 * h + 3].w } };
#pragma unroll
            for (uint32_t m = 0; m < 4u; ++m) {
                // two rows' numbers of one column beside each other
                const uint32_t a[4] = { __byte_perm(w[0][m], w[1][m], 0x5410), __byte_perm(w[0][m], w[1][m], 0x7632), __byte_perm(w[2][m], w[3][m], 0x5410),
                                        __byte_perm(w[2][m], w[3][m], 0x7632) };
#pragma unroll
                for (uint32_t e = 0; e < EIGHTS; ++e) {
                    if (e && !more) continue;
                    gm::mma_16<T>(sums[e].part[m], a, h ? bh[e].z : bh[e].x, h ? bh[e].w : bh[e].y);
                    if (!two) continue;
                    if constexpr (std::is_same<T, __half>::value) {
                        float second[4] = {};
                        gm::mma_16<T>(second, a, h ? bl[e].z : bl[e].x, h ? bl[e].w : bl[e].y);
#pragma unroll
                        for (uint32_t i = 0; i < 4u; ++i) sums[e].part[m][i] = fmaf(kDown<T>, second[i], sums[e].part[m][i]);
                    } else {
                        gm::mma_16<T>(sums[e].part[m], a, h ? bl[e].z : bl[e].x, h ? bl[e].w : bl[e].y);
                    }
                }
            }
        }
    }
}

// COPY: bytes of a copy of weights to shared memory, 16, 4 or 0: they are loaded straight into operands.  SPLIT: the block's warps share a tile.
struct RowsArgs {
    GradientArgs a;
    uint32_t layers, splits;             // blocks that share a group's rows, eight at a time; and the weight rows, a chunk at a time
    float* part;                         // splits > 1: [splits][rows][n_in]
};
// Rows [r, r + 8 EIGHTS) of the group, as far as `end`.
template <typename T, uint32_t COPY, bool SPLIT, uint32_t EIGHTS>
__device__ __forceinline__ void rows_tile(const RowsArgs& p, uint32_t group, uint32_t split, uint32_t c0, uint64_t r, uint64_t end, T* hi, T* lo, T* stage, float (*share)[EIGHTS][16][32])
{
    constexpr bool STAGED = COPY != 0u && !SPLIT;
    const GradientArgs& a = p.a;
    constexpr uint32_t kTiles = Tile<T>::kTiles, C = Tile<T>::kColumns, kChunk = STAGED ? 64u : 128u, kPitch = Tile<T>::pitch(kChunk), kThreads = 32u * kRowWarps;
    const GroupedArgs& f = a.f;
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3u, n_out = f.n_out;
    const uint32_t rows = static_cast<uint32_t>(min(static_cast<uint64_t>(8u * EIGHTS), end - r));
    const uint32_t mine = c0 + (SPLIT ? 0u : warp * Tile<T>::kWarpColumns), columns = mine < f.n_in ? f.n_in - mine : 0u;
    const bool two = f.activation == EVO_ACT_TANH, act = f.activation != EVO_ACT_NONE;
    const T* const w = static_cast<const T*>(f.w) + group * f.stride_w;
    const uint32_t k0 = SPLIT ? warp * kStepK : 0u;
    Sums<T> sums[EIGHTS];
#pragma unroll
    for (uint32_t e = 0; e < EIGHTS; ++e) sums[e].clear();
    for (uint32_t o0 = split * kChunk; o0 < n_out; o0 += p.splits * kChunk) {
        const uint32_t count = min(kChunk, n_out - o0);
        uint4 v[8];
        if constexpr (STAGED) {
            __syncthreads();
            // (512 bytes of a weight row: 32 copies of 16 bytes, or 128 of 4)
            constexpr uint32_t kCopies = 512u / COPY, kEach = COPY / sizeof(T), kMine = kChunk * kCopies / kThreads;
#pragma unroll
            for (uint32_t i = 0; i < kMine; ++i) {
                const uint32_t row = threadIdx.x / kCopies + i * (kThreads / kCopies), c = threadIdx.x % kCopies * kEach;
                const bool there = row < count && c0 + c < f.n_in;
                const uint32_t to = smem_u32(stage + row * Tile<T>::kWeightPitch + c), bytes = there ? COPY : 0u;
                const T* const from = there ? w + static_cast<uint64_t>(o0 + row) * f.ld_w + c0 + c : w;
                if constexpr (COPY == 16u) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" :: "r"(to), "l"(from), "r"(bytes) : "memory");
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else {
            load_step<T, COPY == 16u>(w + (columns ? mine : 0u), f.ld_w, o0 + k0, n_out, columns, v);
        }
        {
            // a weight row a thread: all its rows' dy and y are asked for together
            constexpr uint32_t kEach = 8u * EIGHTS * kChunk / kThreads;
            const uint32_t k = threadIdx.x % kChunk, row0 = threadIdx.x / kChunk * kEach;
            T dy[kEach], y[kEach];
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i)
                if (k < count && row0 + i < rows) {
                    dy[i] = static_cast<const T*>(a.dy)[(r + row0 + i) * a.ld_dy + o0 + k];
                    if (act) y[i] = static_cast<const T*>(f.y)[(r + row0 + i) * f.ld_y + o0 + k];
                }
            if (!STAGED) __syncthreads();
#pragma unroll
            for (uint32_t i = 0; i < kEach; ++i) {
                const float d = k < count && row0 + i < rows ? dz_unit(a, to_float(dy[i]), act ? to_float(y[i]) : 0.f) : 0.f;
                const uint32_t at = (row0 + i) * kPitch + Tile<T>::place_of(k);
                if constexpr (std::is_same<T, float>::value) {
                    uint32_t h, l;
                    gm::split(d, h, l);
                    hi[at] = __uint_as_float(h);
                    lo[at] = __uint_as_float(l);
                } else {
                    const T h = from_float<T>(d);
                    hi[at] = h;
                    if (two) lo[at] = from_float<T>(isfinite(to_float(h)) ? kUp<T> * (d - to_float(h)) : 0.f);
                }
            }
        }
        if (STAGED) asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();
#pragma unroll
        for (uint32_t n = 0; n < (SPLIT ? 1u : kChunk / kStepK); ++n) {
            const uint32_t k = k0 + n * kStepK;
            if (k >= count) break;
            if (n && sizeof(T) == 4 && n % 2u == 0u) {
#pragma unroll
                for (uint32_t e = 0; e < EIGHTS; ++e) sums[e].take_out();
            }
            if constexpr (STAGED) {
#pragma unroll
                for (uint32_t j = 0; j < 8u; ++j)
                    v[j] = *reinterpret_cast<const uint4*>(stage + (k + Tile<T>::row_of(j, q)) * Tile<T>::kWeightPitch + warp * Tile<T>::kWarpColumns + C * g);
            } else {
                if (n) load_step<T, COPY == 16u>(w + (columns ? mine : 0u), f.ld_w, o0 + k, n_out, columns, v);
            }
            step<T, EIGHTS>(v, hi, lo, kPitch, two, rows > 8u, k, sums);
        }
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e) sums[e].take_out();
    }
    if constexpr (std::is_same<T, float>::value)
#pragma unroll
        for (uint32_t e = 0; e < EIGHTS; ++e)
#pragma unroll
            for (uint32_t m = 0; m < kTiles; ++m)
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) sums[e].c[m][i] = gm::join(sums[e].c[m][i], sums[e].small[m][i]);
    if (SPLIT) {
        if (warp)
#pragma unroll
            for (uint32_t e = 0; e < EIGHTS; ++e)
#pragma unroll
                for (uint32_t m = 0; m < kTiles; ++m)
#pragma unroll
                    for (uint32_t i = 0; i < 4u; ++i) share[warp - 1u][e][m * 4u + i][lane] = sums[e].c[m][i];
        __syncthreads();
        if (warp == 0)
#pragma unroll
            for (uint32_t p = 0; p < kRowWarps - 1u; ++p)
#pragma unroll
                for (uint32_t e = 0; e < EIGHTS; ++e)
#pragma unroll
                    for (uint32_t m = 0; m < kTiles; ++m)
#pragma unroll
                        for (uint32_t i = 0; i < 4u; ++i) sums[e].c[m][i] += share[p][e][m * 4u + i][lane];
        __syncthreads();
        if (warp) return;
    }
#pragma unroll
    for (uint32_t e = 0; e < EIGHTS; ++e)
#pragma unroll
        for (uint32_t i = 0; i < 2u; ++i) {
            const uint32_t row = 8u * e + 2u * q + i;
            if (row >= rows) continue;
            if (p.splits > 1u) {
                float* const to = p.part + (split * f.rows + r + row) * f.n_in + mine + C * g;
#pragma unroll
                for (uint32_t j = 0; j < C; ++j)
                    if (C * g + j < columns) to[j] = f.scale * sums[e].c[j / 2u][i + 2u * (j & 1u)];
            } else {
                T* const to = static_cast<T*>(a.dx) + (r + row) * a.ld_dx + mine + C * g;
#pragma unroll
                for (uint32_t j = 0; j < C; ++j)
                    if (C * g + j < columns) to[j] = from_float<T>(f.scale * sums[e].c[j / 2u][i + 2u * (j & 1u)]);
            }
        }
}

template <typename T, uint32_t COPY, bool SPLIT, uint32_t EIGHTS>
__global__ void __launch_bounds__(32 * kRowWarps, (COPY && !SPLIT ? 6 : 5) - EIGHTS) k_rows(const __grid_constant__ RowsArgs p)
{
    constexpr bool kStaged = COPY != 0u && !SPLIT;
    constexpr uint32_t kPitch = Tile<T>::pitch(kStaged ? 64u : 128u), kWide = SPLIT ? Tile<T>::kWarpColumns : Tile<T>::kAcross;
    __shared__ __align__(16) T hi[8 * EIGHTS * kPitch], lo[8 * EIGHTS * kPitch], stage[kStaged ? 64u * Tile<T>::kWeightPitch : 8u];
    __shared__ float share[SPLIT ? kRowWarps - 1 : 1][EIGHTS][16][32];
    dep_begin(p.a);
    const uint32_t across = (p.a.f.n_in + kWide - 1u) / kWide;
    const uint32_t group = blockIdx.x / across, c0 = blockIdx.x % across * kWide;
    // (the last rows first: few groups have them, and those take longest)
    uint32_t split = 0, layer = gridDim.y - 1u - blockIdx.y;
    if (p.splits > 1u) { split = layer % p.splits; layer /= p.splits; }
    uint64_t first, end;
    group_rows(p.a.f, group, &first, &end);
    for (uint64_t r = first + 8u * EIGHTS * layer; r < end; r += 8u * EIGHTS * p.layers) rows_tile<T, COPY, SPLIT, EIGHTS>(p, group, split, c0, r, end, hi, lo, stage, share);
    dep_end(p.a);
}

// The parts of rows that belong to a group, added up in their order.
template <typename T>
__global__ void __launch_bounds__(256) k_add_rows(const __grid_constant__ RowsArgs p)
{
    dep_wait();
    dep_trigger();
    const GroupedArgs& f = p.a.f;
    uint64_t first, end, skip;
    group_rows(f, 0u, &first, &skip);
    group_rows(f, f.groups - 1u, &skip, &end);
    const uint64_t each = f.rows * f.n_in;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256u + threadIdx.x; i < each; i += static_cast<uint64_t>(gridDim.x) * 256u) {
        const uint64_t row = i / f.n_in;
        if (row < first || row >= end) continue;
        float s = 0.f;
#pragma unroll 4
        for (uint32_t k = 0; k < p.splits; ++k) s += p.part[k * each + i];
        static_cast<T*>(p.a.dx)[row * p.a.ld_dx + i % f.n_in] = from_float<T>(s);
    }
}

// ---- dW and db ----
struct WeightsArgs {
    GradientArgs a;
    uint32_t all, sets, splits, out_tiles, in_tiles;
    float* part_w; float* part_b;                            // [splits][sets][n_out][n_in], [splits][sets][n_out]
};
constexpr uint32_t kStep = 16;                               // rows at a time

// Tiles of TO outputs x TI inputs; a thread has 4 inputs (side by side with VEC, where four can be stored together) of TO TI / 1,024 outputs.
template <typename T, uint32_t TO, uint32_t TI, bool VEC>
__global__ void __launch_bounds__(256, 4) k_weights(const __grid_constant__ WeightsArgs p)
{
    constexpr uint32_t kAcross = TI / 4u, kEach = TO * TI / 1024u;
    __shared__ __align__(16) float dz[kStep][TO], xs[kStep][TI];
    const GradientArgs& a = p.a;
    dep_begin(a);
    const uint32_t n_in = a.f.n_in, n_out = a.f.n_out;
    uint32_t at = blockIdx.x;
    const uint32_t i0 = at % p.in_tiles * TI; at /= p.in_tiles;
    const uint32_t o0 = at % p.out_tiles * TO; at /= p.out_tiles;
    const uint32_t split = at % p.splits, set = at / p.splits;
    uint64_t r, end;
    set_rows(a, p.all, set, split, p.splits, &r, &end);
    const uint32_t tx = threadIdx.x % kAcross, ty = threadIdx.x / kAcross;
    const bool bias = a.db && i0 == 0u && threadIdx.x < TO;
    float sum[kEach][4] = {}, sum_b = 0.f;
    for (; r < end; r += kStep) {
        const uint32_t rows = end - r < kStep ? static_cast<uint32_t>(end - r) : kStep;
        // Rows are asked for, and put where the block's threads find them, 4 D at a time: no more than there are (with four of them, most of the instructions are
        // those of the other twelve).
        auto stage = [&](auto fours) {
            constexpr uint32_t D = decltype(fours)::value;
            constexpr uint32_t kZ = (4u * D * TO + 255u) / 256u, kX = (4u * D * TI + 255u) / 256u;
            T dy[kZ], y[kZ], x[kX];
            const uint32_t o = o0 + threadIdx.x % TO, i = i0 + threadIdx.x % TI;
#pragma unroll
            for (uint32_t k = 0; k < kZ; ++k) {
                const uint32_t row = threadIdx.x / TO + 256u / TO * k;
                if (row < rows && o < n_out) {
                    dy[k] = static_cast<const T*>(a.dy)[(r + row) * a.ld_dy + o];
                    if (a.f.activation != EVO_ACT_NONE) y[k] = static_cast<const T*>(a.f.y)[(r + row) * a.f.ld_y + o];
                }
            }
#pragma unroll
            for (uint32_t k = 0; k < kX; ++k) {
                const uint32_t row = threadIdx.x / TI + 256u / TI * k;
                if (row < rows && i < n_in) x[k] = static_cast<const T*>(a.f.x)[(r + row) * a.f.ld_x + i];
            }
            __syncthreads();
#pragma unroll
            for (uint32_t k = 0; k < kZ; ++k) {
                const uint32_t row = threadIdx.x / TO + 256u / TO * k;
                dz[row][threadIdx.x % TO] = row < rows && o < n_out ? dz_of(a, to_float(dy[k]), a.f.activation == EVO_ACT_NONE ? 0.f : to_float(y[k])) : 0.f;
            }
#pragma unroll
            for (uint32_t k = 0; k < kX; ++k) {
                const uint32_t row = threadIdx.x / TI + 256u / TI * k;
                xs[row][threadIdx.x % TI] = row < rows && i < n_in ? to_float(x[k]) : 0.f;
            }
            __syncthreads();
        };
        if (rows <= 4u) stage(std::integral_constant<uint32_t, 1>());
        else if (rows <= 8u) stage(std::integral_constant<uint32_t, 2>());
        else stage(std::integral_constant<uint32_t, 4>());
        if (bias) {
            float s = 0.f;
#pragma unroll
            for (uint32_t k = 0; k < kStep; ++k) s += k < rows ? dz[k][threadIdx.x] : 0.f;
            sum_b += s;
        }
#pragma unroll 4
        for (uint32_t k = 0; k < rows; ++k) {
            float xx[4];
            if constexpr (VEC) {
                const float4 v = *reinterpret_cast<const float4*>(&xs[k][4u * tx]);
                xx[0] = v.x; xx[1] = v.y; xx[2] = v.z; xx[3] = v.w;
            } else {
#pragma unroll
                for (uint32_t j = 0; j < 4u; ++j) xx[j] = xs[k][tx + kAcross * j];
            }
#pragma unroll
            for (uint32_t i = 0; i < kEach; i += 4u) {
                const float4 v = *reinterpret_cast<const float4*>(&dz[k][kEach * ty + i]);
                const float dd[4] = { v.x, v.y, v.z, v.w };
#pragma unroll
                for (uint32_t e = 0; e < 4u; ++e)
#pragma unroll
                    for (uint32_t j = 0; j < 4u; ++j) sum[i + e][j] = fmaf(dd[e], xx[j], sum[i + e][j]);
            }
        }
    }
    const uint64_t part = static_cast<uint64_t>(split) * p.sets + set;
    if (bias && o0 + threadIdx.x < n_out) {
        const uint32_t o = o0 + threadIdx.x;
        if (p.splits > 1u) p.part_b[part * n_out + o] = sum_b;
        else static_cast<T*>(a.db)[set * a.stride_db + o] = from_float<T>(sum_b);
    }
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t o = o0 + kEach * ty + i;
        if (o >= n_out) break;
        float* const to_part = p.part_w + (part * n_out + o) * n_in;
        T* const to = static_cast<T*>(a.dw) + set * a.stride_dw + o * a.ld_dw;
        if constexpr (VEC) {
            const uint32_t c = i0 + 4u * tx;
            if (c >= n_in) break;
            if (p.splits > 1u) store4(to_part + c, sum[i]);
            else store4(to + c, sum[i]);
        } else {
#pragma unroll
            for (uint32_t j = 0; j < 4u; ++j) {
                const uint32_t c = i0 + tx + kAcross * j;
                if (c >= n_in) break;
                if (p.splits > 1u) to_part[c] = sum[i][j];
                else to[c] = from_float<T>(sum[i][j]);
            }
        }
    }
    dep_end(a);
}

// db alone: 256 / R threads side by side with N columns each, R rows at a time.
struct BiasArgs {
    GradientArgs a;
    uint32_t all, sets, splits, tiles;
    float* part;
    const uint16_t* laid;                                    // dz as laid out for the tensor cores, or NULL
    uint32_t parts, pitch;
};
template <typename T, uint32_t N, uint32_t R>
__global__ void __launch_bounds__(256) k_bias(const __grid_constant__ BiasArgs p)
{
    constexpr uint32_t kWide = 256u / R;
    __shared__ float sums[R][kWide * N];
    const GradientArgs& a = p.a;
    dep_begin(a);
    uint32_t at = blockIdx.x;
    const uint32_t c0 = at % p.tiles * kWide * N; at /= p.tiles;
    const uint32_t split = at % p.splits, set = at / p.splits;
    uint64_t first, end;
    set_rows(a, p.all, set, split, p.splits, &first, &end);
    const uint32_t c = c0 + threadIdx.x % kWide * N, n_out = a.f.n_out;
    const bool act = a.f.activation != EVO_ACT_NONE;
    float sum[N] = {};
    if (p.laid) {                                            // dz / scale is there, in parts (N 8: aligned)
        constexpr uint32_t kAsk = 8;
        const uint64_t rows = (end > first ? end - first : 0u) * p.parts;               // (the parts of a row lie one behind the other, like rows)
        const uint16_t* const from = p.laid + first * p.parts * p.pitch + c;
        if (c < n_out)
            for (uint64_t r = threadIdx.x / kWide; r < rows; r += R * kAsk) {
                uint4 u[kAsk];
#pragma unroll
                for (uint32_t k = 0; k < kAsk; ++k) u[k] = r + R * k < rows ? __ldg(reinterpret_cast<const uint4*>(from + (r + R * k) * p.pitch)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (uint32_t k = 0; k < kAsk; ++k) {
                    const uint32_t w[4] = { u[k].x, u[k].y, u[k].z, u[k].w };
                    const float factor = std::is_same<T, __half>::value && p.parts == 2u && ((r + R * k) & 1u) ? kDown<T> : 1.f;      // (a second part)
#pragma unroll
                    for (uint32_t e = 0; e < N; ++e) {
                        const uint16_t bits = static_cast<uint16_t>(w[e / 2u] >> (e % 2u * 16u));
                        if constexpr (std::is_same<T, __half>::value) sum[e] = fmaf(factor, __half2float(__ushort_as_half(bits)), sum[e]);
                        else sum[e] += __uint_as_float(static_cast<uint32_t>(bits) << 16);
                    }
                }
            }
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) sum[e] *= a.f.scale;
    } else if (c < n_out) {
        constexpr uint32_t kAsk = N == 1u ? 8u : 4u;
        for (uint64_t r = first + threadIdx.x / kWide; r < end; r += R * kAsk) {
            T dy[kAsk][N], y[kAsk][N];
#pragma unroll
            for (uint32_t k = 0; k < kAsk; ++k) {
                const uint64_t row = r + R * k;
                if (row >= end) break;
                const T* const from = static_cast<const T*>(a.dy) + row * a.ld_dy + c;
                const T* const from_y = static_cast<const T*>(a.f.y) + row * a.f.ld_y + c;
                if constexpr (N * sizeof(T) != 16u) {
                    dy[k][0] = from[0];
                    if (act) y[k][0] = from_y[0];
                } else {
                    const uint4 u = __ldg(reinterpret_cast<const uint4*>(from));
                    memcpy(dy[k], &u, 16);
                    if (act) { const uint4 v = __ldg(reinterpret_cast<const uint4*>(from_y)); memcpy(y[k], &v, 16); }
                }
            }
#pragma unroll
            for (uint32_t k = 0; k < kAsk; ++k) {
                if (r + R * k >= end) break;
#pragma unroll
                for (uint32_t e = 0; e < N; ++e) sum[e] += dz_of(a, to_float(dy[k][e]), act ? to_float(y[k][e]) : 0.f);
            }
        }
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) sums[threadIdx.x / kWide][threadIdx.x % kWide * N + e] = sum[e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < kWide * N; i += 256u) {
        if (c0 + i >= n_out) break;
        float s = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < R; ++k) s += sums[k][i];
        if (p.splits > 1u) p.part[(static_cast<uint64_t>(split) * p.sets + set) * n_out + c0 + i] = s;
        else static_cast<T*>(a.db)[set * a.stride_db + c0 + i] = from_float<T>(s);
    }
    dep_end(a);
}

// The splits' parts, added up in their order: rows of `n` numbers, `rows` of them a set.
template <typename T>
__global__ void __launch_bounds__(256) k_add_parts(const float* __restrict__ part, uint32_t splits, uint32_t sets, uint32_t rows, uint32_t n, T* __restrict__ to, uint64_t stride,
                                                   uint64_t ld)
{
    dep_wait();
    dep_trigger();
    const uint64_t each = static_cast<uint64_t>(sets) * rows * n;
    for (uint64_t i = static_cast<uint64_t>(blockIdx.x) * 256u + threadIdx.x; i < each; i += static_cast<uint64_t>(gridDim.x) * 256u) {
        float s = 0.f;
        for (uint32_t k = 0; k < splits; ++k) s += part[k * each + i];
        const uint64_t row = i / n;
        to[row / rows * stride + row % rows * ld + i % n] = from_float<T>(s);
    }
}

// ---- plans ----
// Splits of the rows: as many as fill the GPU twice, of no fewer than 128 rows on average.
uint32_t splits_for(const GradientArgs& a, bool all, uint64_t tiles)
{
    const uint64_t sets = all ? 1u : a.f.groups, blocks = sets * tiles, rows = a.f.rows / sets;
    if (blocks >= kSms) return 1u;
    const uint64_t most = 2u * kSms / blocks, want = rows / 128u;
    return static_cast<uint32_t>(want < 2u ? 1u : want < most ? want : most);
}
// db alone is read in little time, but a block's rows one after the other: no more than 64 rows a split on average, of up to 16, while the GPU has room.
uint32_t bias_splits(const GradientArgs& a)
{
    const uint64_t sets = a.sum_b ? 1u : a.f.groups, blocks = sets * ((a.f.n_out + 255u) / 256u), rows = a.f.rows / sets;
    uint32_t splits = 1;
    while (splits < 16u && blocks * splits < 4u * kSms && rows > 64u * splits) splits *= 2u;
    return splits;
}
// 16-bit rows that are whole pieces of 16 bytes (the same wherever the arrays lie: workspaces are planned before they do)
bool whole_pieces(const GradientArgs& a) { return ((a.f.n_in | a.f.n_out) & 7u) == 0u; }
// Whether tcgen05 pays for dx: rows a group from which it does.  fp32 weights, and those that TMA cannot address, are laid out first, whatever the rows; the walk over many
// groups takes a warp longer than the products; few tiles leave SMs without one, which k_rows' splits do not; and a tile takes 128 inputs x 64 outputs at a time, however
// few there are.  us, tcgen05 / k_rows, rows a group in brackets:
//   fp32     200 groups of 256 -> 256 (32) 63.6 / 53.1, (64) 69.3 / 98; 32 of 1,024 -> 1,024 (32) 139 / 88, (64) 144 / 163; 1 of 4,096 -> 4,096 (64) 175 / 127;
//            1,000 of 64 -> 64 (64) 75 / 48; 300 of 207 -> 379 (32) 134 / 131; 4,096 of 128 -> 128 (64) 421 / 300
//   16 bits  200 of 256 -> 256 (2) 13.1 / 10.6, (5) 13.1 / 15.9; 1,000 of 64 -> 64 (16) 26.4 / 17.6, (32) 27.5 / 31.6; 4,096 of 128 -> 128 (16) 109 / 100; 32 of 1,024 -> 1,024
//            (2) 16.6 / 22.2, (8) 16.6 / 39.4; 1 of 4,096 -> 4,096 (10) 25.8 / 24.1, (64) 26 / 75; not aligned: 300 of 207 -> 379 (5) 60.8 / 36.7, (8) 61.3 / 64.5; 3,000 of
//            20 -> 30 (16) 94.6 / 65.2, (32) 102 / 105; 10 of 1,887 -> 3,200 (1) 56 / 117
// Over 374 shapes (270 of them drawn) the choice takes 1.03 times the faster side's time in the geometric mean; tcgen05 always 1.8 times, k_rows always 1.16.  It is a fit, and the lines above
// are not all on its side: 1,000 of 64 -> 64 fp32 go to tcgen05 from 63 rows on (75 us for 48), 32 of 1,024 -> 1,024 fp32 from 35 on, where the two meet near 54, and 16 bits from 2.5 (2 rows: 22.2 us for
// 16.6).
bool dx_on_tensor_cores(uint32_t type, const GradientArgs& a)
{
    const GroupedArgs& f = a.f;
    if (f.rows >= (1ull << 31) || static_cast<uint64_t>(f.groups) * f.n_out >= (1ull << 31)) return false;
    const double groups = f.groups, across = (f.n_in + 127u) / 128u, idle = std::fmax(0.0, 1.0 - std::fmin(groups, static_cast<double>(f.rows)) * across / kSms), few = idle * idle * idle * idle;
    const double size = static_cast<double>(f.n_in) * f.n_out, more = std::fmin(16.0, 8192.0 * across * ((f.n_out + 63u) / 64u) / size) - 1.0;
    const double least = type == EVO_F32 ? 34.0 + groups / 40.0 + 120.0 * few + 4.0 * more
                       : whole_pieces(a) ? 2.0 + std::fmin(groups / 60.0, 16.0) + 80.0 * few + more
                       : 8.0 * std::fmin(1.0, 3e5 / size) + std::fmin(groups / 60.0, 16.0) + 160.0 * few * std::fmin(1.0, 1e5 / size) + 2.0 * more;
    return static_cast<double>(f.rows) >= least * groups;
}
// The same for dW.  A tile is 128 outputs x up to 256 inputs, however many there are; where there are few tiles k_weights takes long groups 16 rows at a time.  tcgen05 / k_weights:
//   fp32     200 of 256 -> 256 (8) 29.5 / 20.6, (16) 31.0 / 33.1; 32 of 1,024 -> 1,024 (16) 58.7 / 62.6; 1 of 4,096 -> 4,096 (16) 36.5 / 27.8, (32) 40.2 / 45.4;
//            1,000 of 64 -> 64 (64) 74 / 46; 7 of 171 -> 7 (107) 20.8 / 47.4
//   16 bits  200 of 256 -> 256 (2) 10.0 / 10.9; 1,000 of 64 -> 64 (8) 17.3 / 9.7, (16) 12.0 / 15.4, (32) 13.1 / 26.4; 4 of 2,048 -> 2,048 (2) 17.6 / 11.1, (8) 17.5 / 19.5;
//            not aligned: 300 of 207 -> 379 (8) 32.6 / 40.5; 3,000 of 20 -> 30 (32) 71 / 51, (64) 112 / 92
// Over the same shapes 1.02 times the faster side's time; tcgen05 always 1.7 times, k_weights always 1.3.
bool dw_on_tensor_cores(uint32_t type, const GradientArgs& a)
{
    const GroupedArgs& f = a.f;
    if (f.rows >= (1ull << 31)) return false;
    const double sets = a.sum_w ? 1.0 : f.groups, tiles = static_cast<double>((f.n_out + 127u) / 128u) * ((f.n_in + 255u) / 256u);
    const double waste = tiles * 32768.0 / (static_cast<double>(f.n_in) * f.n_out);
    double least = type == EVO_F32 ? 18.0 * std::fmin(std::fmax(0.5 * waste, 1.0), 12.0) : (whole_pieces(a) ? 2.0 : 6.0) + 2.0 * std::fmin(waste, 12.0);
    if (tiles * sets < kSms) least = std::fmin(least, 48.0);
    return static_cast<double>(f.rows) >= least * sets;
}
// A tile of k_weights: where there are few outputs (a policy's actions) or few inputs, most of a square one would be nothing.  fp32, us, square / narrow: 320
// groups of 137 -> 7, 9,292 rows 30.7 / 16.9; 1,000 of 256 -> 16, 32,000 rows 58.5 / 27.2; 2,000 of 16 -> 256, a row each 24.9 / 10.8; but long groups are better served by more
// tiles: 64 of 4 -> 128, 60,000 rows 170 / 286.
struct Shape { uint32_t outputs, inputs; };
Shape tile_of(const GradientArgs& a)
{
    if (a.f.n_out <= 16u && a.f.n_in > 64u) return { 16u, 256u };
    if (a.f.n_in <= 16u && a.f.n_out > 64u && a.f.rows <= 16ull * a.f.groups) return { 256u, 16u };
    return { 64u, a.f.n_in <= 64u ? 64u : 128u };
}
uint64_t tiles_of(uint64_t n, uint32_t each) { return (n + each - 1u) / each; }
// How dx is spread over blocks without tcgen05: the columns of a warp's tile shared by the block's warps (split), rows eight at a time over `layers`, weight rows a chunk at a time over
// `splits`, as far as there is room on the GPU.
struct RowsPlan { uint32_t eights, split, layers, splits; };
RowsPlan rows_plan(uint32_t type, const GradientArgs& a)
{
    const GroupedArgs& f = a.f;
    const uint64_t all = type == EVO_F32 ? 128u : 256u, wide = all / kRowWarps, used = f.rows < f.groups ? f.rows : f.groups;
    RowsPlan p;
    // (16 rows at a time read and split the weights half as often: us, 8 / 16 at a time, rows a group in brackets: fp32, 200 groups of 256 -> 256 (5) 19.0 / 17.2, (16) 34.8 / 29.5, (64)
    // 127 / 98; 32 of 1,024 -> 1,024 (8) 58 / 65, (32) 122 / 96; not aligned, 100 of 414 -> 378 (2) 17.5 / 25.3, (5) 37.5 / 27.4; 16 bits, 4,096 of 128 -> 128 (8) 59 / 72, (32)
    // 180 / 185; not aligned, 300 of 207 -> 379 (2) 32.8 / 39.7, (5) 57.9 / 36.7, (12) 81.8 / 68.8)
    const bool aligned = f.n_in % (type == EVO_F32 ? 4u : 8u) == 0u;
    p.eights = f.rows > (aligned ? 10ull : 4ull) * f.groups && (type == EVO_F32 || !aligned) ? 2u : 1u;
    const uint64_t passes = (f.rows / f.groups + 8u * p.eights - 1u) / (8u * p.eights);
    uint64_t blocks = used * ((f.n_in + all - 1u) / all);
    // (with two rows a group on average few have nine, and the blocks that find none cost more)
    const uint64_t most_layers = f.rows > 2ull * f.groups ? 2u * passes : 1u, room = 8u * kSms;
    uint64_t layers = blocks ? room / blocks : 1u;
    layers = layers < 2u ? 2u : layers;
    layers = layers < most_layers ? layers : most_layers;
    p.split = blocks * layers < 4u * kSms && f.n_out > kStepK;
    if (p.split) blocks = used * ((f.n_in + wide - 1u) / wide);
    const uint64_t chunks = (f.n_out + (p.split ? 127u : 63u)) / (p.split ? 128u : 64u);
    uint64_t splits = 1;
    // (a block waits most of the time, for one chunk after the other: more of them than fit at a time, us with 4 / 8 / 16 an SM: fp32, 10 groups of 1,887 -> 3,200, 23 rows each
    // 387 / 383 / 195; 32 of 1,024 -> 1,024, 10 rows each 54 / 54 / 43; 1 of 4,096 -> 4,096, 10 rows 61 / 39 / 39)
    if (chunks > 2u) splits = 16u * kSms / (blocks * layers + 1u);
    splits = splits > chunks / 2u ? chunks / 2u : splits;
    p.layers = static_cast<uint32_t>(layers < 1u ? 1u : layers);
    p.splits = static_cast<uint32_t>(splits < 2u ? 1u : splits > 32u ? 32u : splits);
    return p;
}
struct Plan {
    TcPlan tc;
    RowsPlan rows;
    bool both;                           // dW and db in one launch of k_weights
    uint32_t w_splits, b_splits;
    size_t tc_bytes, x_bytes, w_bytes, b_bytes;
};
size_t padded(size_t n) { return (n + 255u) / 256u * 256u; }
Plan plan_for(uint32_t type, const GradientArgs& a, bool any_address)
{
    Plan p;
    const Shape tile = tile_of(a);
    const bool dx = a.dx && a.f.rows && dx_on_tensor_cores(type, a), dw = a.dw && a.f.rows && dw_on_tensor_cores(type, a);
    p.both = a.dw && !dw && a.db && a.sum_w == a.sum_b;
    p.w_splits = !a.dw ? 1u : dw ? splits_for(a, a.sum_w, ((a.f.n_out + 127ull) / 128u) * ((a.f.n_in + 255ull) / 256u)) : splits_for(a, a.sum_w, tiles_of(a.f.n_out, tile.outputs) * tiles_of(a.f.n_in, tile.inputs));
    p.b_splits = p.both ? p.w_splits : a.db ? bias_splits(a) : 1u;
    p.tc = grouped_gradient_tc_plan(type, a, dx, dw, p.w_splits, any_address);
    const uint64_t w_sets = a.sum_w ? 1u : a.f.groups, b_sets = a.sum_b ? 1u : a.f.groups;
    p.tc_bytes = padded(p.tc.bytes());
    p.rows = rows_plan(type, a);
    p.x_bytes = a.dx && a.f.rows && !dx && p.rows.splits > 1u ? padded(4u * p.rows.splits * a.f.rows * a.f.n_in) : 0u;
    p.w_bytes = p.w_splits > 1u ? padded(4u * p.w_splits * w_sets * a.f.n_out * a.f.n_in) : 0u;
    p.b_bytes = p.b_splits > 1u ? padded(4u * p.b_splits * b_sets * a.f.n_out) : 0u;
    return p;
}

template <typename T, uint32_t EIGHTS>
int launch_rows(cudaStream_t st, const GradientArgs& a, const RowsPlan& plan, float* part)
{
    const GroupedArgs& f = a.f;
    const uint32_t wide = plan.split ? Tile<T>::kWarpColumns : Tile<T>::kAcross;
    const uint64_t blocks = static_cast<uint64_t>(f.groups) * ((f.n_in + wide - 1u) / wide);
    if (blocks > 0x7FFFFFFFull) return -2;
    RowsArgs p;
    p.a = a; p.layers = plan.layers; p.splits = plan.splits; p.part = part;
    const uint64_t bits = reinterpret_cast<uintptr_t>(f.w) | (f.n_in | f.ld_w | f.stride_w) * sizeof(T);
    auto kernel = bits % 16u == 0u ? (plan.split ? k_rows<T, 16, true, EIGHTS> : k_rows<T, 16, false, EIGHTS>)
                : plan.split ? k_rows<T, 0, true, EIGHTS> : bits % 4u == 0u ? k_rows<T, 4, false, EIGHTS> : k_rows<T, 0, false, EIGHTS>;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks), plan.layers * plan.splits), dim3(32 * kRowWarps), 0, st, p) == cudaSuccess ? 1 : -1;
}
template <typename T>
bool add_rows(cudaStream_t st, const GradientArgs& a, const RowsPlan& plan, float* part)
{
    RowsArgs p;
    p.a = a; p.layers = plan.layers; p.splits = plan.splits; p.part = part;
    const uint64_t blocks = (a.f.rows * a.f.n_in + 255u) / 256u;
    return launch_dependent(k_add_rows<T>, dim3(static_cast<uint32_t>(blocks < 8u * kSms ? blocks : 8u * kSms)), dim3(256), 0, st, p) == cudaSuccess;
}

template <typename T>
bool add_parts(cudaStream_t st, const float* part, uint32_t splits, uint32_t sets, uint32_t rows, uint32_t n, void* to, uint64_t stride, uint64_t ld)
{
    const uint64_t blocks = (static_cast<uint64_t>(sets) * rows * n + 255u) / 256u;
    return launch_dependent(k_add_parts<T>, dim3(static_cast<uint32_t>(blocks < 8u * kSms ? blocks : 8u * kSms)), dim3(256), 0, st, part, splits, sets, rows, n, static_cast<T*>(to),
                            stride, ld) == cudaSuccess;
}

template <typename T>
int launch_weights(cudaStream_t st, const GradientArgs& in, bool bias, uint32_t splits, float* part_w, float* part_b)
{
    WeightsArgs p;
    p.a = in;
    if (!bias) p.a.db = nullptr;
    p.all = in.sum_w;
    p.sets = p.all ? 1u : in.f.groups;
    p.splits = splits;
    const Shape tile = tile_of(in);
    p.out_tiles = static_cast<uint32_t>(tiles_of(in.f.n_out, tile.outputs));
    p.in_tiles = static_cast<uint32_t>(tiles_of(in.f.n_in, tile.inputs));
    p.part_w = part_w; p.part_b = part_b;
    const uint64_t blocks = static_cast<uint64_t>(p.sets) * splits * p.out_tiles * p.in_tiles;
    if (blocks > 0x7FFFFFFFull) return -2;
    const bool four = in.f.n_in % 4u == 0u && (splits > 1u || (reinterpret_cast<uintptr_t>(in.dw) % (4u * sizeof(T)) == 0u && (in.ld_dw | in.stride_dw) % 4u == 0u));
    auto kernel = tile.outputs == 16u ? (four ? k_weights<T, 16, 256, true> : k_weights<T, 16, 256, false>)
                : tile.outputs == 256u ? (four ? k_weights<T, 256, 16, true> : k_weights<T, 256, 16, false>)
                : tile.inputs == 64u ? (four ? k_weights<T, 64, 64, true> : k_weights<T, 64, 64, false>) : (four ? k_weights<T, 64, 128, true> : k_weights<T, 64, 128, false>);
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st, p) == cudaSuccess ? 1 : -1;
}

// columns of a thread of k_bias: 16 bytes, where rows start and end on them
template <typename T>
uint32_t bias_columns(const GradientArgs& a)
{
    constexpr uint32_t N = 16u / sizeof(T);
    const bool act = a.f.activation != EVO_ACT_NONE;
    const uintptr_t address = reinterpret_cast<uintptr_t>(a.dy) | (act ? reinterpret_cast<uintptr_t>(a.f.y) : 0u);
    return address % 16u == 0u && (a.f.n_out | a.ld_dy | (act ? a.f.ld_y : 0u)) % N == 0u ? N : 1u;
}
template <typename T>
int launch_bias(cudaStream_t st, const GradientArgs& in, uint32_t splits, float* part, const TcPlan& tc, const void* work)
{
    BiasArgs p;
    p.a = in;
    p.all = in.sum_b; p.sets = p.all ? 1u : in.f.groups; p.splits = splits; p.part = part;
    p.laid = tc.lay_dz ? static_cast<const uint16_t*>(work) : nullptr;      // (the first of the workspace)
    p.parts = tc.dz_parts; p.pitch = tc.pitch_dz;
    const uint32_t n = p.laid ? 8u : bias_columns<T>(in);
    // (many groups of few rows: wide rows one at a time: 1,095 of 1,597, 17 rows in all 62 -> 10.6 us, 4,096 of 512, a row each 31 -> 10.6)
    const bool one = splits == 1u && in.f.rows <= 4ull * p.sets && in.f.n_out > 32u * n;
    p.tiles = static_cast<uint32_t>(tiles_of(in.f.n_out, (one ? 256u : 32u) * n));
    const uint64_t blocks = static_cast<uint64_t>(p.sets) * splits * p.tiles;
    if (blocks > 0x7FFFFFFFull) return -2;
    auto kernel = one ? (n == 1u ? k_bias<T, 1, 1> : n == 4u ? k_bias<T, 4, 1> : k_bias<T, 8, 1>) : n == 1u ? k_bias<T, 1, 8> : n == 4u ? k_bias<T, 4, 8> : k_bias<T, 8, 8>;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st, p) == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_type(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work)
{
    const Plan plan = plan_for(type, a, false);
    uint8_t* const at = static_cast<uint8_t*>(work);
    float* const part_x = reinterpret_cast<float*>(at + plan.tc_bytes);
    float* const part_w = reinterpret_cast<float*>(at + plan.tc_bytes + plan.x_bytes);
    float* const part_b = reinterpret_cast<float*>(at + plan.tc_bytes + plan.x_bytes + plan.w_bytes);
    const uint32_t w_sets = a.sum_w ? 1u : a.f.groups, b_sets = a.sum_b ? 1u : a.f.groups;
    int launches = 0, n = 0;
    // (the first kernel waits at its beginning)
    auto late = [&](GradientArgs b) { b.late = launches > 0; return b; };
    if (plan.tc.dx || plan.tc.dw) {
        n = launch_grouped_gradient_tc(st, type, a, plan.tc, plan.w_splits, part_w, work);
        if (n < 0) return n;
        launches += n;
    }
    if (a.dx && a.f.rows && !plan.tc.dx) {
        n = plan.rows.eights == 2u ? launch_rows<T, 2>(st, late(a), plan.rows, part_x) : launch_rows<T, 1>(st, late(a), plan.rows, part_x);
        if (n < 0) return n;
        launches += n;
    }
    if (a.dw && !plan.tc.dw) {
        n = launch_weights<T>(st, late(a), plan.both, plan.w_splits, part_w, part_b);
        if (n < 0) return n;
        launches += n;
    }
    if (a.db && !plan.both) {
        n = launch_bias<T>(st, late(a), plan.b_splits, part_b, plan.tc, work);
        if (n < 0) return n;
        launches += n;
    }
    if (plan.x_bytes) {
        if (!add_rows<T>(st, a, plan.rows, part_x)) return -1;
        ++launches;
    }
    if (plan.w_splits > 1u) {
        if (!add_parts<T>(st, part_w, plan.w_splits, w_sets, a.f.n_out, a.f.n_in, a.dw, a.stride_dw, a.ld_dw)) return -1;
        ++launches;
    }
    if (plan.b_splits > 1u) {
        if (!add_parts<T>(st, part_b, plan.b_splits, b_sets, 1u, a.f.n_out, a.db, a.stride_db, 0u)) return -1;
        ++launches;
    }
    return launches;
}

}  // namespace

size_t grouped_gradient_bytes(uint32_t type, const GradientArgs& a, bool any_address)
{
    const Plan p = plan_for(type, a, any_address);
    return p.tc_bytes + p.x_bytes + p.w_bytes + p.b_bytes;
}

int launch_grouped_gradient(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work)
{
    return type == EVO_F32 ? launch_type<float>(st, type, a, work) : type == EVO_BF16 ? launch_type<__nv_bfloat16>(st, type, a, work) : launch_type<__half>(st, type, a, work);
}

}  // namespace evo

// Gradients of the products grouped by member: dx[r] = W_g' dz[r], dW_g = sum_r dz[r] x[r]', db_g = sum_r dz[r]; any type, size, stride and alignment.
//
// A group of a population has few rows and weights of its own: dx is bound by the weights' way from memory, dW by its own way there.  k_rows reads
// a group's weights once for up to 8 rows, which are multiplied in fp32 on the CUDA cores; k_weights makes tiles of 64 outputs x 64 or 128 inputs.  Where there are too few tiles for the
// GPU and many rows, the rows are split and the parts added up in a fixed order.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>
#include <type_traits>

#include "grouped_gradient.h"

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
template <typename T>
__device__ __forceinline__ float dz_at(const GradientArgs& a, uint64_t row, uint32_t o)
{
    const float dy = to_float(static_cast<const T*>(a.dy)[row * a.ld_dy + o]);
    return dz_of(a, dy, a.f.activation == EVO_ACT_NONE ? 0.f : to_float(static_cast<const T*>(a.f.y)[row * a.f.ld_y + o]));
}

// Four numbers that lie together, as fp32.
template <typename T>
__device__ __forceinline__ void load4(const T* p, float (&v)[4])
{
    T raw[4];
    if constexpr (sizeof(T) == 4) { const uint4 u = __ldg(reinterpret_cast<const uint4*>(p)); memcpy(raw, &u, 16); }
    else { const uint2 u = __ldg(reinterpret_cast<const uint2*>(p)); memcpy(raw, &u, 8); }
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) v[i] = to_float(raw[i]);
}
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
// 4 columns a thread, `wide` threads side by side and the others on other weight rows: their sums are added up at the end.  A thread asks for kAhead rows of
// weights before it needs the first, and for the first ones before dz is there.
constexpr uint32_t kRows = 8, kChunk = 256, kThreads = 256, kAhead = 8;

template <typename T, bool VEC>
__global__ void __launch_bounds__(kThreads, 2) k_rows(const __grid_constant__ GradientArgs a, uint32_t wide)
{
    __shared__ __align__(16) float dz[kChunk][kRows];
    __shared__ __align__(16) float sums[kThreads][4 * kRows];
    dep_wait();
    dep_trigger();
    const GroupedArgs& f = a.f;
    const uint32_t n_in = f.n_in, n_out = f.n_out, tiles = (n_in + 4u * wide - 1u) / (4u * wide);
    const uint32_t group = blockIdx.x / tiles, c0 = blockIdx.x % tiles * 4u * wide, tx = threadIdx.x % wide, ty = threadIdx.x / wide, slices = kThreads / wide;
    uint64_t first, end;
    group_rows(f, group, &first, &end);
    const T* const w = static_cast<const T*>(f.w) + group * f.stride_w + c0;
    for (uint64_t r = first; r < end; r += kRows) {
        const uint32_t rows = static_cast<uint32_t>(min(static_cast<uint64_t>(kRows), end - r));
        float sum[4][kRows];
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i)
#pragma unroll
            for (uint32_t k = 0; k < kRows; ++k) sum[i][k] = 0.f;
        for (uint32_t o0 = 0; o0 < n_out; o0 += kChunk) {
            const uint32_t count = min(kChunk, n_out - o0);
            float v[kAhead][4];
            auto ask = [&](uint32_t o) {
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    const uint32_t k = o + j * slices;
                    const T* const from = w + static_cast<uint64_t>(o0 + k) * f.ld_w;
                    if constexpr (VEC) {
                        if (k < count && c0 + 4u * tx < n_in) load4(from + 4u * tx, v[j]);
                        else v[j][0] = v[j][1] = v[j][2] = v[j][3] = 0.f;
                    } else {
#pragma unroll
                        for (uint32_t i = 0; i < 4u; ++i) v[j][i] = k < count && c0 + tx + wide * i < n_in ? to_float(from[tx + wide * i]) : 0.f;
                    }
                }
            };
            ask(ty);
            __syncthreads();
            const uint32_t padded = (count + 31u) / 32u * 32u;              // (a warp's loads are one row's)
#pragma unroll 2
            for (uint32_t i = threadIdx.x; i < padded * kRows; i += kThreads) {
                const uint32_t o = i % padded, row = i / padded;
                dz[o][row] = o < count && row < rows ? dz_at<T>(a, r + row, o0 + o) : 0.f;
            }
            __syncthreads();
            for (uint32_t o = ty; o < count; o += slices * kAhead) {
                if (o != ty) ask(o);
#pragma unroll
                for (uint32_t j = 0; j < kAhead; ++j) {
                    if (o + j * slices >= count) break;
                    const float4 d0 = *reinterpret_cast<const float4*>(&dz[o + j * slices][0]), d1 = *reinterpret_cast<const float4*>(&dz[o + j * slices][4]);
                    const float d[kRows] = { d0.x, d0.y, d0.z, d0.w, d1.x, d1.y, d1.z, d1.w };
#pragma unroll
                    for (uint32_t i = 0; i < 4u; ++i)
#pragma unroll
                        for (uint32_t k = 0; k < kRows; ++k) sum[i][k] = fmaf(v[j][i], d[k], sum[i][k]);
                }
            }
        }
        // sums[ty][row][column]
        __syncthreads();
        float* const flat = &sums[0][0];
#pragma unroll
        for (uint32_t k = 0; k < kRows; ++k)
            if (k < rows) {
                float* const to = flat + (ty * kRows + k) * 4u * wide;
                if constexpr (VEC) {
                    *reinterpret_cast<float4*>(to + 4u * tx) = make_float4(sum[0][k], sum[1][k], sum[2][k], sum[3][k]);
                } else {
#pragma unroll
                    for (uint32_t i = 0; i < 4u; ++i) to[tx + wide * i] = sum[i][k];
                }
            }
        __syncthreads();
        for (uint32_t i = threadIdx.x; i < rows * 4u * wide; i += kThreads) {
            const uint32_t c = i % (4u * wide), row = i / (4u * wide);
            float s = 0.f;
#pragma unroll 8
            for (uint32_t y = 0; y < slices; ++y) s += flat[(y * kRows + row) * 4u * wide + c];
            if (c0 + c < n_in) static_cast<T*>(a.dx)[(r + row) * a.ld_dx + c0 + c] = from_float<T>(s);
        }
    }
}

// ---- dW and db ----
struct WeightsArgs {
    GradientArgs a;
    uint32_t all, sets, splits, out_tiles, in_tiles;
    float* part_w; float* part_b;                            // [splits][sets][n_out][n_in], [splits][sets][n_out]
};
constexpr uint32_t kTile = 64, kStep = 16;                   // outputs of a tile, rows at a time

// Tiles of 64 outputs x TI inputs; a thread has 4 inputs (side by side with VEC, where four can be stored together) of TI / 16 outputs.
template <typename T, uint32_t TI, bool VEC>
__global__ void __launch_bounds__(256, 3) k_weights(const __grid_constant__ WeightsArgs p)
{
    constexpr uint32_t kAcross = TI / 4u, kEach = TI / 16u;
    __shared__ __align__(16) float dz[kStep][kTile], xs[kStep][TI];
    dep_wait();
    dep_trigger();
    const GradientArgs& a = p.a;
    const uint32_t n_in = a.f.n_in, n_out = a.f.n_out;
    uint32_t at = blockIdx.x;
    const uint32_t i0 = at % p.in_tiles * TI; at /= p.in_tiles;
    const uint32_t o0 = at % p.out_tiles * kTile; at /= p.out_tiles;
    const uint32_t split = at % p.splits, set = at / p.splits;
    uint64_t r, end;
    set_rows(a, p.all, set, split, p.splits, &r, &end);
    const uint32_t tx = threadIdx.x % kAcross, ty = threadIdx.x / kAcross;
    const bool bias = a.db && i0 == 0u && threadIdx.x < kTile;
    float sum[kEach][4] = {}, sum_b = 0.f;
    for (; r < end; r += kStep) {
        float d[4], x[TI / 16u];
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k) {
            const uint32_t row = threadIdx.x / kTile + 4u * k, o = o0 + threadIdx.x % kTile;
            d[k] = r + row < end && o < n_out ? dz_at<T>(a, r + row, o) : 0.f;
        }
#pragma unroll
        for (uint32_t k = 0; k < TI / 16u; ++k) {
            const uint32_t row = threadIdx.x / TI + 256u / TI * k, i = i0 + threadIdx.x % TI;
            x[k] = r + row < end && i < n_in ? to_float(static_cast<const T*>(a.f.x)[(r + row) * a.f.ld_x + i]) : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k) dz[threadIdx.x / kTile + 4u * k][threadIdx.x % kTile] = d[k];
#pragma unroll
        for (uint32_t k = 0; k < TI / 16u; ++k) xs[threadIdx.x / TI + 256u / TI * k][threadIdx.x % TI] = x[k];
        __syncthreads();
        if (bias) {
            float s = 0.f;
#pragma unroll
            for (uint32_t k = 0; k < kStep; ++k) s += dz[k][threadIdx.x];
            sum_b += s;
        }
        const uint32_t rows = end - r < kStep ? static_cast<uint32_t>(end - r) : kStep;
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
}

// db alone: 32 threads side by side with N columns each, 8 rows at a time.
struct BiasArgs {
    GradientArgs a;
    uint32_t all, sets, splits, tiles;
    float* part;
};
template <typename T, uint32_t N>
__global__ void __launch_bounds__(256) k_bias(const __grid_constant__ BiasArgs p)
{
    __shared__ float sums[8][32 * N];
    dep_wait();
    dep_trigger();
    const GradientArgs& a = p.a;
    uint32_t at = blockIdx.x;
    const uint32_t c0 = at % p.tiles * 32u * N; at /= p.tiles;
    const uint32_t split = at % p.splits, set = at / p.splits;
    uint64_t first, end;
    set_rows(a, p.all, set, split, p.splits, &first, &end);
    const uint32_t c = c0 + threadIdx.x % 32u * N, n_out = a.f.n_out;
    const bool act = a.f.activation != EVO_ACT_NONE;
    float sum[N] = {};
    if (c < n_out) {
        constexpr uint32_t kAsk = 4;
        for (uint64_t r = first + threadIdx.x / 32u; r < end; r += 8u * kAsk) {
            T dy[kAsk][N], y[kAsk][N];
#pragma unroll
            for (uint32_t k = 0; k < kAsk; ++k) {
                const uint64_t row = r + 8u * k;
                if (row >= end) break;
                const T* const from = static_cast<const T*>(a.dy) + row * a.ld_dy + c;
                const T* const from_y = static_cast<const T*>(a.f.y) + row * a.f.ld_y + c;
                if constexpr (N == 1u) {
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
                if (r + 8u * k >= end) break;
#pragma unroll
                for (uint32_t e = 0; e < N; ++e) sum[e] += dz_of(a, to_float(dy[k][e]), act ? to_float(y[k][e]) : 0.f);
            }
        }
    }
#pragma unroll
    for (uint32_t e = 0; e < N; ++e) sums[threadIdx.x / 32u][threadIdx.x % 32u * N + e] = sum[e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < 32u * N; i += 256u) {
        if (c0 + i >= n_out) break;
        float s = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < 8u; ++k) s += sums[k][i];
        if (p.splits > 1u) p.part[(static_cast<uint64_t>(split) * p.sets + set) * n_out + c0 + i] = s;
        else static_cast<T*>(a.db)[set * a.stride_db + c0 + i] = from_float<T>(s);
    }
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
bool dx_on_tensor_cores(uint32_t type, const GradientArgs& a)
{
    return a.f.rows < (1ull << 31) && static_cast<uint64_t>(a.f.groups) * a.f.n_out < (1ull << 31) && a.f.rows >= 24ull * a.f.groups;
}
bool dw_on_tensor_cores(uint32_t type, const GradientArgs& a)
{
    return a.f.rows < (1ull << 31) && a.f.rows >= 24ull * (a.sum_w ? 1u : a.f.groups);
}
uint32_t inputs_of_a_tile(const GradientArgs& a) { return a.f.n_in <= 64u ? 64u : 128u; }
struct Plan {
    TcPlan tc;
    bool both;                           // dW and db in one launch of k_weights
    uint32_t w_splits, b_splits;
    size_t tc_bytes, w_bytes, b_bytes;
};
size_t padded(size_t n) { return (n + 255u) / 256u * 256u; }
Plan plan_for(uint32_t type, const GradientArgs& a, bool any_address)
{
    Plan p;
    const uint64_t out_tiles = (a.f.n_out + kTile - 1u) / kTile, in_tiles = (a.f.n_in + inputs_of_a_tile(a) - 1u) / inputs_of_a_tile(a);
    const bool dx = a.dx && a.f.rows && dx_on_tensor_cores(type, a), dw = a.dw && a.f.rows && dw_on_tensor_cores(type, a);
    p.both = a.dw && !dw && a.db && a.sum_w == a.sum_b;
    p.w_splits = !a.dw ? 1u : dw ? splits_for(a, a.sum_w, ((a.f.n_out + 127ull) / 128u) * ((a.f.n_in + 255ull) / 256u)) : splits_for(a, a.sum_w, out_tiles * in_tiles);
    p.b_splits = p.both ? p.w_splits : a.db ? splits_for(a, a.sum_b, (a.f.n_out + 127u) / 128u) : 1u;
    p.tc = grouped_gradient_tc_plan(type, a, dx, dw, p.w_splits, any_address);
    const uint64_t w_sets = a.sum_w ? 1u : a.f.groups, b_sets = a.sum_b ? 1u : a.f.groups;
    p.tc_bytes = padded(p.tc.bytes());
    p.w_bytes = p.w_splits > 1u ? padded(4u * p.w_splits * w_sets * a.f.n_out * a.f.n_in) : 0u;
    p.b_bytes = p.b_splits > 1u ? padded(4u * p.b_splits * b_sets * a.f.n_out) : 0u;
    return p;
}

template <typename T>
int launch_rows(cudaStream_t st, const GradientArgs& a)
{
    const GroupedArgs& f = a.f;
    uint32_t wide = 8u;                                      // columns of a block: as the row needs, fewer where there are few groups
    while (wide < 64u && wide * 4u < f.n_in) wide *= 2u;
    const uint64_t used = f.rows < f.groups ? f.rows : f.groups;
    while (wide > 8u && used * ((f.n_in + 4u * wide - 1u) / (4u * wide)) < 2u * kSms) wide /= 2u;
    const uint64_t blocks = static_cast<uint64_t>(f.groups) * ((f.n_in + 4u * wide - 1u) / (4u * wide));
    if (blocks > 0x7FFFFFFFull) return -2;
    const bool aligned = (reinterpret_cast<uintptr_t>(f.w) & (4u * sizeof(T) - 1u)) == 0u && ((f.n_in | f.ld_w | f.stride_w) & 3u) == 0u;
    auto kernel = aligned ? k_rows<T, true> : k_rows<T, false>;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, st, a, wide) == cudaSuccess ? 1 : -1;
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
    p.out_tiles = (in.f.n_out + kTile - 1u) / kTile;
    const uint32_t wide = inputs_of_a_tile(in);
    p.in_tiles = (in.f.n_in + wide - 1u) / wide;
    p.part_w = part_w; p.part_b = part_b;
    const uint64_t blocks = static_cast<uint64_t>(p.sets) * splits * p.out_tiles * p.in_tiles;
    if (blocks > 0x7FFFFFFFull) return -2;
    const bool four = in.f.n_in % 4u == 0u && (splits > 1u || (reinterpret_cast<uintptr_t>(in.dw) % (4u * sizeof(T)) == 0u && (in.ld_dw | in.stride_dw) % 4u == 0u));
    auto kernel = wide == 64u ? (four ? k_weights<T, 64, true> : k_weights<T, 64, false>) : (four ? k_weights<T, 128, true> : k_weights<T, 128, false>);
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
int launch_bias(cudaStream_t st, const GradientArgs& in, uint32_t splits, float* part)
{
    BiasArgs p;
    p.a = in;
    p.all = in.sum_b; p.sets = p.all ? 1u : in.f.groups; p.splits = splits; p.part = part;
    const uint32_t n = bias_columns<T>(in);
    p.tiles = (in.f.n_out + 32u * n - 1u) / (32u * n);
    const uint64_t blocks = static_cast<uint64_t>(p.sets) * splits * p.tiles;
    if (blocks > 0x7FFFFFFFull) return -2;
    auto kernel = n == 1u ? k_bias<T, 1> : k_bias<T, 16u / sizeof(T)>;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(256), 0, st, p) == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_type(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work)
{
    const Plan plan = plan_for(type, a, false);
    uint8_t* const at = static_cast<uint8_t*>(work);
    float* const part_w = reinterpret_cast<float*>(at + plan.tc_bytes);
    float* const part_b = reinterpret_cast<float*>(at + plan.tc_bytes + plan.w_bytes);
    const uint32_t w_sets = a.sum_w ? 1u : a.f.groups, b_sets = a.sum_b ? 1u : a.f.groups;
    int launches = 0, n = 0;
    if (plan.tc.dx || plan.tc.dw) {
        n = launch_grouped_gradient_tc(st, type, a, plan.tc, plan.w_splits, part_w, work);
        if (n < 0) return n;
        launches += n;
    }
    if (a.dx && a.f.rows && !plan.tc.dx) {
        n = launch_rows<T>(st, a);
        if (n < 0) return n;
        launches += n;
    }
    if (a.dw && !plan.tc.dw) {
        n = launch_weights<T>(st, a, plan.both, plan.w_splits, part_w, part_b);
        if (n < 0) return n;
        launches += n;
    }
    if (a.db && !plan.both) {
        n = launch_bias<T>(st, a, plan.b_splits, part_b);
        if (n < 0) return n;
        launches += n;
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
    return p.tc_bytes + p.w_bytes + p.b_bytes;
}

int launch_grouped_gradient(cudaStream_t st, uint32_t type, const GradientArgs& a, void* work)
{
    return type == EVO_F32 ? launch_type<float>(st, type, a, work) : type == EVO_BF16 ? launch_type<__nv_bfloat16>(st, type, a, work) : launch_type<__half>(st, type, a, work);
}

}  // namespace evo

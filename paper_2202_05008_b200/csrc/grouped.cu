// Products grouped by member, y[r] = scale act(W_g x[r] + b_g), on warp-level tensor-core products: any type, size, stride and alignment.
//
// A group of a population has few rows and weights of its own, so the kernel is bound by the weights' way from memory: a warp
// takes 16 outputs and reads their weight rows once, straight into the MMA's operand registers; the group's rows are the
// MMA's columns (8, or 32 where more are left).  Where there are too few such tiles to fill the GPU the four warps of a block
// share one and split the contracted index.
#include <cstring>
#include <type_traits>

#include "grouped.h"
#include "grouped_mma.cuh"

namespace evo {
namespace {

constexpr uint32_t kWarps = 4;
// The tensor core cuts its sums off (2.7e-5 of 4,096 16-bit numbers of one sign): beyond kLong of the contracted index they are taken out every kPart, by instances of
// their own (a loop around the loop over the contracted index keeps the loads from running ahead: 1,262 groups of 5 rows, 3,536 -> 8, bf16: 150 us without, 250 with)
constexpr uint32_t kPart = 4096, kLong = 8192;

template <typename T> __device__ __forceinline__ float to_float(T x);
template <> __device__ __forceinline__ float to_float(float x) { return x; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_float(float x) { return __float2half_rn(x); }

// Sixteen bytes of a row from element k on; elements from n_in on are 0 (what lies there is another row, or a bias).
template <typename T, bool VEC>
__device__ __forceinline__ uint4 load16(const T* row, uint32_t k, uint32_t n_in)
{
    constexpr uint32_t N = 16u / sizeof(T);
    uint4 r = make_uint4(0u, 0u, 0u, 0u);
    if constexpr (VEC) {
        if (k < n_in) r = *reinterpret_cast<const uint4*>(row + k);          // (n_in is a multiple of N)
    } else {
        T v[N];
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) v[e] = k + e < n_in ? row[k + e] : from_float<T>(0.f);
        memcpy(&r, v, 16);
    }
    return r;
}

// Sums of 16 outputs x 8 NT rows over [k0, k1): c[t] holds (output g, rows 2q, 2q + 1), (output g + 8, the same) of the t-th eight rows.
template <typename T, bool VEC, uint32_t NT>
__device__ __forceinline__ void tile_sums(const T* w0, const T* w1, const T* const (&x)[NT], uint32_t k0, uint32_t k1, uint32_t n_in, float (&c)[NT][4])
{
    const uint32_t q = threadIdx.x & 3u;
    if constexpr (std::is_same<T, float>::value) {
        constexpr uint32_t kAhead = NT == 1u ? 8u : 4u;          // sixteens whose weights are asked for together
        float small[NT][4], less[NT][4];
#pragma unroll
        for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = small[t][i] = less[t][i] = 0.f;
        for (uint32_t k = k0; k < k1; k += 16u * kAhead) {
            float large[NT][4];
#pragma unroll
            for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) large[t][i] = 0.f;
            uint4 u[kAhead], v[kAhead];
#pragma unroll
            for (uint32_t s = 0; s < kAhead; ++s) {
                u[s] = load16<T, VEC>(w0, k + 16u * s + 4u * q, n_in);
                v[s] = load16<T, VEC>(w1, k + 16u * s + 4u * q, n_in);
            }
#pragma unroll
            for (uint32_t s = 0; s < kAhead; ++s) {
                if (k + 16u * s >= k1) break;
                if (s == 4u)
#pragma unroll
                    for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) { c[t][i] += large[t][i]; large[t][i] = 0.f; }
                const uint32_t wu[4] = { u[s].x, u[s].y, u[s].z, u[s].w }, wv[4] = { v[s].x, v[s].y, v[s].z, v[s].w };
                uint32_t hi[2][4], lo[2][4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    gm::split(__uint_as_float(wu[2 * h]), hi[h][0], lo[h][0]);
                    gm::split(__uint_as_float(wv[2 * h]), hi[h][1], lo[h][1]);
                    gm::split(__uint_as_float(wu[2 * h + 1]), hi[h][2], lo[h][2]);
                    gm::split(__uint_as_float(wv[2 * h + 1]), hi[h][3], lo[h][3]);
                }
#pragma unroll
                for (uint32_t t = 0; t < NT; ++t) {
                    const uint4 r = load16<T, VEC>(x[t], k + 16u * s + 4u * q, n_in);
                    const uint32_t xs[4] = { r.x, r.y, r.z, r.w };
                    uint32_t xh[4], xl[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) gm::split(__uint_as_float(xs[e]), xh[e], xl[e]);
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        gm::mma_tf32(large[t], hi[h], xh[2 * h], xh[2 * h + 1]);
                        gm::mma_tf32(small[t], hi[h], xl[2 * h], xl[2 * h + 1]);
                        gm::mma_tf32(NT == 1u ? less[t] : small[t], lo[h], xh[2 * h], xh[2 * h + 1]);      // (32 rows have no registers for a third sum)
                    }
                }
            }
#pragma unroll
            for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) c[t][i] += large[t][i];
        }
#pragma unroll
        for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = gm::join(c[t][i], small[t][i] + less[t][i]);
    } else {
#pragma unroll
        for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = 0.f;
        for (uint32_t k = k0; k < k1; k += 128u) {
            uint4 u[4], v[4];
#pragma unroll
            for (uint32_t s = 0; s < 4u; ++s) {
                u[s] = load16<T, VEC>(w0, k + 32u * s + 8u * q, n_in);
                v[s] = load16<T, VEC>(w1, k + 32u * s + 8u * q, n_in);
            }
#pragma unroll
            for (uint32_t s = 0; s < 4u; ++s) {
                if (k + 32u * s >= k1) break;
                const uint32_t a0[4] = { u[s].x, v[s].x, u[s].y, v[s].y }, a1[4] = { u[s].z, v[s].z, u[s].w, v[s].w };
#pragma unroll
                for (uint32_t t = 0; t < NT; ++t) {
                    const uint4 r = load16<T, VEC>(x[t], k + 32u * s + 8u * q, n_in);
                    gm::mma_16<T>(c[t], a0, r.x, r.y);
                    gm::mma_16<T>(c[t], a1, r.z, r.w);
                }
            }
        }
    }
}

__device__ __forceinline__ float activate(float x, uint32_t activation, float scale)
{
    if (activation == EVO_ACT_TANH) x = gm::tanh32(x);
    if (activation == EVO_ACT_RELU) x = x < 0.f ? 0.f : x;                   // (a NaN stays one)
    return scale * x;
}

// rows [r, r + 8 NT) of the group, as far as `end`; SPLIT: the block's warps share the tile
template <typename T, bool VEC, uint32_t NT, bool SPLIT, bool LONG>
__device__ __forceinline__ void tile(const GroupedArgs& a, uint32_t group, uint32_t o0, uint64_t r, uint64_t end, float (*part)[32][4 * 4])
{
    const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5, g = lane >> 2, q = lane & 3u;
    const T* const w = static_cast<const T*>(a.w) + group * a.stride_w;
    // what is beyond the last output or row is read as the last one, and not stored
    const T* const w0 = w + static_cast<uint64_t>(min(o0 + g, a.n_out - 1u)) * a.ld_w;
    const T* const w1 = w + static_cast<uint64_t>(min(o0 + g + 8u, a.n_out - 1u)) * a.ld_w;
    const T* x[NT];
#pragma unroll
    for (uint32_t t = 0; t < NT; ++t) {
        const uint64_t row = r + 8u * t + g;
        x[t] = static_cast<const T*>(a.x) + (row < end ? row : end - 1u) * a.ld_x;
    }
    uint32_t k0 = 0, k1 = a.n_in;
    if (SPLIT) {
        const uint32_t per = (a.n_in + 128u * kWarps - 1u) / (128u * kWarps) * 128u;
        k0 = min(warp * per, a.n_in);
        k1 = min(k0 + per, a.n_in);
    }
    float c[NT][4];
    if constexpr (LONG) {
#pragma unroll
        for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) c[t][i] = 0.f;
        for (uint32_t k = k0; k < k1; k += kPart) {
            float part[NT][4];
            tile_sums<T, VEC, NT>(w0, w1, x, k, min(k + kPart, k1), a.n_in, part);
#pragma unroll
            for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) c[t][i] += part[t][i];
        }
    } else {
        tile_sums<T, VEC, NT>(w0, w1, x, k0, k1, a.n_in, c);
    }
    if (SPLIT) {
        if (warp)
#pragma unroll
            for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                for (uint32_t i = 0; i < 4u; ++i) part[warp - 1u][lane][t * 4u + i] = c[t][i];
        __syncthreads();
        if (warp == 0)
#pragma unroll
            for (uint32_t p = 0; p < kWarps - 1u; ++p)
#pragma unroll
                for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
                    for (uint32_t i = 0; i < 4u; ++i) c[t][i] += part[p][lane][t * 4u + i];
        __syncthreads();
        if (warp) return;
    }
    const T* const b = a.b ? static_cast<const T*>(a.b) + group * a.stride_b : nullptr;
#pragma unroll
    for (uint32_t h = 0; h < 2u; ++h) {
        const uint32_t o = o0 + g + 8u * h;
        if (o >= a.n_out) continue;
        const float bias = b ? to_float(b[o]) : 0.f;
#pragma unroll
        for (uint32_t t = 0; t < NT; ++t)
#pragma unroll
            for (uint32_t i = 0; i < 2u; ++i) {
                const uint64_t row = r + 8u * t + 2u * q + i;
                if (row < end) static_cast<T*>(a.y)[row * a.ld_y + o] = from_float<T>(activate(c[t][2u * h + i] + bias, a.activation, a.scale));
            }
    }
}

// fp32, at most 128 of the contracted index, aligned; up to 8 rows: the weights and biases are asked for first, then the rows, which the block's warps
// share through shared memory: one latency for all of them
constexpr uint32_t kShort = 128;
__device__ __forceinline__ void short_tile(const GroupedArgs& a, uint32_t group, uint32_t o0, uint64_t r, uint64_t end, float (*rows)[kShort + 4])
{
    const uint32_t lane = threadIdx.x & 31u, g = lane >> 2, q = lane & 3u;
    const float* const w = static_cast<const float*>(a.w) + group * a.stride_w;
    const float* const w0 = w + static_cast<uint64_t>(min(o0 + g, a.n_out - 1u)) * a.ld_w;
    const float* const w1 = w + static_cast<uint64_t>(min(o0 + g + 8u, a.n_out - 1u)) * a.ld_w;
    const float* const b = a.b ? static_cast<const float*>(a.b) + group * a.stride_b : nullptr;
    uint4 u[8], v[8];
#pragma unroll
    for (uint32_t s = 0; s < 8u; ++s) {
        u[s] = load16<float, true>(w0, 16u * s + 4u * q, a.n_in);
        v[s] = load16<float, true>(w1, 16u * s + 4u * q, a.n_in);
    }
    const float b0 = b && o0 + g < a.n_out ? b[o0 + g] : 0.f, b1 = b && o0 + g + 8u < a.n_out ? b[o0 + g + 8u] : 0.f;
#pragma unroll
    for (uint32_t t = 0; t < 2u; ++t) {
        const uint32_t x = threadIdx.x + 128u * t, row = x >> 5, k = (x & 31u) * 4u;
        const uint64_t from = r + row < end ? r + row : end - 1u;
        *reinterpret_cast<uint4*>(&rows[row][k]) = load16<float, true>(static_cast<const float*>(a.x) + from * a.ld_x, k, a.n_in);
    }
    __syncthreads();
    float large[4] = {}, small[4] = {}, less[4] = {}, sum[4] = {};
#pragma unroll
    for (uint32_t s = 0; s < 8u; ++s) {
        if (16u * s >= a.n_in) break;
        if (s == 4u)
#pragma unroll
            for (int i = 0; i < 4; ++i) { sum[i] = large[i]; large[i] = 0.f; }
        const uint32_t wu[4] = { u[s].x, u[s].y, u[s].z, u[s].w }, wv[4] = { v[s].x, v[s].y, v[s].z, v[s].w };
        const float4 z = *reinterpret_cast<const float4*>(&rows[g][16u * s + 4u * q]);
        uint32_t xh[4], xl[4];
        gm::split(z.x, xh[0], xl[0]); gm::split(z.y, xh[1], xl[1]); gm::split(z.z, xh[2], xl[2]); gm::split(z.w, xh[3], xl[3]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t hi[4], lo[4];
            gm::split(__uint_as_float(wu[2 * h]), hi[0], lo[0]);
            gm::split(__uint_as_float(wv[2 * h]), hi[1], lo[1]);
            gm::split(__uint_as_float(wu[2 * h + 1]), hi[2], lo[2]);
            gm::split(__uint_as_float(wv[2 * h + 1]), hi[3], lo[3]);
            gm::mma_tf32(large, hi, xh[2 * h], xh[2 * h + 1]);
            gm::mma_tf32(small, hi, xl[2 * h], xl[2 * h + 1]);
            gm::mma_tf32(less, lo, xh[2 * h], xh[2 * h + 1]);
        }
    }
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
        const uint32_t o = o0 + g + 8u * (i >> 1);
        const uint64_t row = r + 2u * q + (i & 1u);
        if (o >= a.n_out || row >= end) continue;
        float y = gm::join(sum[i] + large[i], small[i] + less[i]) + (i >> 1 ? b1 : b0);
        if (a.activation == EVO_ACT_TANH) y = gm::tanh32(y);
        if (a.activation == EVO_ACT_RELU) y = y < 0.f ? 0.f : y;
        static_cast<float*>(a.y)[row * a.ld_y + o] = a.scale * y;
    }
}
__global__ void __launch_bounds__(kWarps * 32, 5) k_grouped_short(const __grid_constant__ GroupedArgs a)
{
    __shared__ float rows[8][kShort + 4];
    dep_wait();
    dep_trigger();
    const uint32_t per = (a.n_out + 16u * kWarps - 1u) / (16u * kWarps);
    const uint32_t group = blockIdx.x / per, o0 = blockIdx.x % per * 16u * kWarps + (threadIdx.x >> 5) * 16u;
    uint64_t r, end;
    group_rows(a, group, &r, &end);
    for (; r < end; r += 8u) {
        short_tile(a, group, o0, r, end, rows);              // (a warp without outputs works on the last one's weights and stores nothing)
        __syncthreads();
    }
}

template <typename T, bool VEC, bool SPLIT, bool LONG>
__global__ void __launch_bounds__(kWarps * 32) k_grouped(const __grid_constant__ GroupedArgs a)
{
    __shared__ float part[SPLIT ? kWarps - 1 : 1][32][4 * 4];
    dep_wait();
    dep_trigger();
    const uint32_t per = (a.n_out + (SPLIT ? 16u : 16u * kWarps) - 1u) / (SPLIT ? 16u : 16u * kWarps);
    const uint32_t group = blockIdx.x / per, o0 = blockIdx.x % per * (SPLIT ? 16u : 16u * kWarps) + (SPLIT ? 0u : (threadIdx.x >> 5) * 16u);
    uint64_t r, end;
    group_rows(a, group, &r, &end);
    if (!SPLIT && o0 >= a.n_out) return;
    while (r < end) {
        if (end - r > 8u) { tile<T, VEC, 4, SPLIT, LONG>(a, group, o0, r, end, part); r += 32u; }
        else { tile<T, VEC, 1, SPLIT, LONG>(a, group, o0, r, end, part); r += 8u; }
    }
}

template <typename T, bool VEC>
int launch(cudaStream_t st, const GroupedArgs& a, bool split)
{
    const uint64_t per = split ? (a.n_out + 15u) / 16u : (a.n_out + 16u * kWarps - 1u) / (16u * kWarps), blocks = per * a.groups;
    if (blocks > 0x7FFFFFFFull) return -2;
    if constexpr (std::is_same<T, float>::value && VEC)
        if (!split && a.n_in <= kShort && a.rows <= 8ull * a.groups)
            return launch_dependent(k_grouped_short, dim3(static_cast<uint32_t>(blocks)), dim3(kWarps * 32), 0, st, a) == cudaSuccess ? 1 : -1;
    auto kernel = split ? k_grouped<T, VEC, true, false> : k_grouped<T, VEC, false, false>;
    if constexpr (!std::is_same<T, float>::value)
        if (a.n_in > kLong) kernel = split ? k_grouped<T, VEC, true, true> : k_grouped<T, VEC, false, true>;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kWarps * 32), 0, st, a) == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_type(cudaStream_t st, const GroupedArgs& a)
{
    constexpr uint64_t kStep = 16u / sizeof(T);
    const bool aligned = ((reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.w)) & 15u) == 0u &&
                         (a.n_in | a.ld_x | a.ld_w | a.stride_w) % kStep == 0u;
    // groups that can have rows, and the blocks that they make without splitting the sums
    const uint64_t used = a.rows < a.groups ? a.rows : a.groups;
    const bool split = used * ((a.n_out + 16u * kWarps - 1u) / (16u * kWarps)) < 4u * kSms && a.n_in > 128u;
    return aligned ? launch<T, true>(st, a, split) : launch<T, false>(st, a, split);
}

}  // namespace

size_t grouped_bytes(uint32_t type, const GroupedArgs& a) { return grouped_tc_addressable(type, a) ? 0u : grouped_tc_bytes(type, a); }

int launch_grouped(cudaStream_t st, uint32_t type, const GroupedArgs& a, void* work)
{
    if (work || grouped_tc_takes(type, a)) return launch_grouped_tc(st, type, a, work);
    return type == EVO_F32 ? launch_type<float>(st, a) : type == EVO_BF16 ? launch_type<__nv_bfloat16>(st, a) : launch_type<__half>(st, a);
}

}  // namespace evo

// Rows in sorted order and back: take, combine and the gradient of combine.
//
// All three go by the rows of the unsorted side, so that each of them is read or written once, and the sorted rows that it has are found by
// their places.  A row is `lanes` threads' (a power of two up to a block), each with every lanes-th piece of up to 16 bytes; pieces are as wide as addresses, pitches and
// length allow.  Bound by memory: no number is moved twice.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>
#include <type_traits>

#include "routing.h"

namespace evo {
namespace {

constexpr uint32_t kThreads = 256;

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

template <uint32_t BYTES> struct Bytes;
template <> struct Bytes<16> { using type = uint4; };
template <> struct Bytes<8> { using type = uint2; };
template <> struct Bytes<4> { using type = uint32_t; };
template <> struct Bytes<2> { using type = uint16_t; };

template <typename T, uint32_t N>
struct Piece {                                               // N numbers that are loaded and stored together
    using Raw = typename Bytes<sizeof(T) * N>::type;
    T v[N];
    __device__ __forceinline__ void load(const T* p) { const Raw r = __ldg(reinterpret_cast<const Raw*>(p)); memcpy(v, &r, sizeof(r)); }
    __device__ __forceinline__ void store(T* p) const { Raw r; memcpy(&r, v, sizeof(r)); *reinterpret_cast<Raw*>(p) = r; }
};

struct Where { uint64_t row; uint32_t lane; bool live; };
__device__ __forceinline__ Where whose(const RowSetArgs& a, uint32_t lanes)
{
    Where w;
    w.row = static_cast<uint64_t>(blockIdx.x) * (kThreads / lanes) + threadIdx.x / lanes;
    w.lane = threadIdx.x & (lanes - 1u);
    w.live = w.row < a.count;
    return w;
}
// (a place outside of the sorted rows is none)
__device__ __forceinline__ bool place_of(const RowSetArgs& a, uint64_t row, uint32_t j, uint32_t* place)
{
    *place = static_cast<uint32_t>(a.place[row * a.ld_place + j]);
    return *place < a.sorted_rows;
}

template <typename T, uint32_t N>
__global__ void __launch_bounds__(kThreads) k_take(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    if (!w.live) return;
    const T* const from = static_cast<const T*>(a.rows) + w.row * a.ld_rows;
    constexpr uint32_t kAhead = 4;
    for (uint32_t c = w.lane * N; c < a.cols; c += lanes * N * kAhead) {
        Piece<T, N> x[kAhead];
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i)
            if (c + i * lanes * N < a.cols) x[i].load(from + c + i * lanes * N);
        for (uint32_t j = 0; j < a.choices; ++j) {
            uint32_t place;
            if (!place_of(a, w.row, j, &place)) continue;
            T* const to = static_cast<T*>(a.sorted) + place * a.ld_sorted;
            const float weight = a.weights ? a.weights[w.row * a.ld_weights + j] : 1.f;
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i)
                if (c + i * lanes * N < a.cols) {
                    Piece<T, N> y = x[i];
                    if (a.weights)
#pragma unroll
                        for (uint32_t e = 0; e < N; ++e) y.v[e] = from_float<T>(weight * to_float(x[i].v[e]));
                    y.store(to + c + i * lanes * N);
                }
        }
    }
}

template <typename T, uint32_t N>
__global__ void __launch_bounds__(kThreads) k_combine(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    if (!w.live) return;
    T* const to = static_cast<T*>(a.rows) + w.row * a.ld_rows;
    constexpr uint32_t kAhead = 4;                           // choices whose rows are asked for together
    for (uint32_t c = w.lane * N; c < a.cols; c += lanes * N) {
        float sum[N];
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) sum[e] = 0.f;
        for (uint32_t j = 0; j < a.choices; j += kAhead) {
            Piece<T, N> y[kAhead];
            bool live[kAhead];
            float weight[kAhead];
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i) {
                uint32_t place = 0;
                live[i] = j + i < a.choices && place_of(a, w.row, j + i, &place);
                if (live[i]) {
                    y[i].load(static_cast<const T*>(a.sorted) + place * a.ld_sorted + c);
                    weight[i] = a.weights ? a.weights[w.row * a.ld_weights + j + i] : 1.f;
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < kAhead; ++i)
                if (live[i])
#pragma unroll
                    for (uint32_t e = 0; e < N; ++e) sum[e] = fmaf(weight[i], to_float(y[i].v[e]), sum[e]);
        }
        Piece<T, N> r;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) r.v[e] = from_float<T>(sum[e]);
        r.store(to + c);
    }
}

// JU: choices that are worked on together, each with a sum of its own
template <typename T, uint32_t N, uint32_t JU>
__global__ void __launch_bounds__(kThreads) k_combine_backward(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    __shared__ float part[kThreads / 32u][JU];
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    const T* const from = static_cast<const T*>(a.rows) + (w.live ? w.row : 0u) * a.ld_rows;
    for (uint32_t j = 0; j < a.choices; j += JU) {
        uint32_t place[JU];
        bool live[JU];
        float weight[JU], dot[JU];
#pragma unroll
        for (uint32_t i = 0; i < JU; ++i) {
            place[i] = 0;
            live[i] = w.live && j + i < a.choices && place_of(a, w.row, j + i, &place[i]);
            weight[i] = live[i] ? a.weights[w.row * a.ld_weights + j + i] : 0.f;
            dot[i] = 0.f;
        }
        if (w.live)
            for (uint32_t c = w.lane * N; c < a.cols; c += lanes * N) {
                Piece<T, N> x, y[JU];
                x.load(from + c);
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i)
                    if (live[i]) y[i].load(static_cast<const T*>(a.sorted) + place[i] * a.ld_sorted + c);
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i)
                    if (live[i]) {
                        Piece<T, N> d;
#pragma unroll
                        for (uint32_t e = 0; e < N; ++e) {
                            const float g = to_float(x.v[e]);
                            dot[i] = fmaf(g, to_float(y[i].v[e]), dot[i]);
                            d.v[e] = from_float<T>(weight[i] * g);
                        }
                        d.store(static_cast<T*>(a.d_sorted) + place[i] * a.ld_d_sorted + c);
                    }
            }
        // the sums of the row's threads
#pragma unroll
        for (uint32_t i = 0; i < JU; ++i)
            for (uint32_t d = min(lanes, 32u) / 2u; d > 0u; d /= 2u) dot[i] += __shfl_xor_sync(0xffffffffu, dot[i], d);
        if (lanes > 32u) {
            const uint32_t warp = threadIdx.x >> 5, warps = lanes / 32u;
            if ((threadIdx.x & 31u) == 0u)
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i) part[warp][i] = dot[i];
            __syncthreads();
            if (w.lane == 0u)
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i)
                    for (uint32_t k = 1; k < warps; ++k) dot[i] += part[warp + k][i];
            __syncthreads();
        }
        if (w.live && w.lane == 0u)
#pragma unroll
            for (uint32_t i = 0; i < JU; ++i)
                if (j + i < a.choices) a.d_weights[w.row * a.ld_d_weights + j + i] = dot[i];
    }
}

// the widest pieces that everything allows
uint32_t numbers_of_a_piece(uint32_t size, const RowSetArgs& a)
{
    uint64_t bits = reinterpret_cast<uintptr_t>(a.rows) | reinterpret_cast<uintptr_t>(a.sorted) | reinterpret_cast<uintptr_t>(a.d_sorted) |
                    (static_cast<uint64_t>(a.cols) | a.ld_rows | a.ld_sorted | a.ld_d_sorted) * size;
    for (uint32_t bytes = 16u; bytes > size; bytes /= 2u)
        if (bits % bytes == 0u) return bytes / size;
    return 1u;
}

// threads of a row: a few pieces each
uint32_t lanes_for(const RowSetArgs& a, uint32_t numbers, uint32_t pieces_each)
{
    const uint32_t pieces = (a.cols + numbers - 1u) / numbers;
    uint32_t lanes = 1;
    while (lanes < kThreads && lanes * pieces_each < pieces) lanes *= 2u;
    return lanes;
}

template <class F>
int by_type(uint32_t type, uint32_t n, F f)
{
    if (type == EVO_F32) return n == 4u ? f(float(), std::integral_constant<uint32_t, 4>()) : n == 2u ? f(float(), std::integral_constant<uint32_t, 2>())
                                        : f(float(), std::integral_constant<uint32_t, 1>());
    auto half = [&](auto t) {
        return n == 8u ? f(t, std::integral_constant<uint32_t, 8>()) : n == 4u ? f(t, std::integral_constant<uint32_t, 4>())
             : n == 2u ? f(t, std::integral_constant<uint32_t, 2>()) : f(t, std::integral_constant<uint32_t, 1>());
    };
    return type == EVO_BF16 ? half(__nv_bfloat16()) : half(__half());
}

int launch(cudaStream_t st, void (*kernel)(RowSetArgs, uint32_t), const RowSetArgs& a, uint32_t lanes)
{
    const uint64_t per = kThreads / lanes, blocks = (a.count + per - 1u) / per;
    if (blocks > 0x7FFFFFFFull) return -2;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, st, a, lanes) == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_take(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    const uint32_t n = numbers_of_a_piece(type == EVO_F32 ? 4u : 2u, a);
    return by_type(type, n, [&](auto t, auto k) { return launch(st, k_take<decltype(t), decltype(k)::value>, a, lanes_for(a, n, 4u)); });
}
int launch_combine(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    const uint32_t n = numbers_of_a_piece(type == EVO_F32 ? 4u : 2u, a);
    return by_type(type, n, [&](auto t, auto k) { return launch(st, k_combine<decltype(t), decltype(k)::value>, a, lanes_for(a, n, 1u)); });
}
int launch_combine_backward(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    const uint32_t n = numbers_of_a_piece(type == EVO_F32 ? 4u : 2u, a);
    return by_type(type, n, [&](auto t, auto k) {
        using T = decltype(t);
        constexpr uint32_t N = decltype(k)::value;
        auto kernel = a.choices == 1u ? k_combine_backward<T, N, 1> : a.choices == 2u ? k_combine_backward<T, N, 2>
                    : a.choices <= 4u ? k_combine_backward<T, N, 4> : k_combine_backward<T, N, 8>;
        return launch(st, kernel, a, lanes_for(a, n, 1u));
    });
}

}  // namespace evo

// Rows in sorted order and back: take, combine and the gradient of combine.
//
// All three go by the rows of the unsorted side, so that each of them is read or written once, and the sorted rows that it has are found by
// their places.  A row is `lanes` threads' (a power of two up to a block), each with every lanes-th piece of 16 bytes.  Bound by memory: no number is moved twice.
// Rows of bf16: take of 32,768 x 2,048 for four choices 101 us, 6.5 TB/s; combine of 40,000 x 2,048, two choices, 86 us, 5.6 TB/s; its gradient, 16,384 x 1,024, eight
// choices, 99 us, 5.7 TB/s; fp16, 5,003 x 1,001, three choices, where no two rows begin alike, 17.1 us,
// 3.9 TB/s.
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
    __device__ __forceinline__ void scale(float f)
    {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) v[e] = from_float<T>(f * to_float(v[e]));
    }
    __device__ __forceinline__ float dot(const Piece& other, float sum) const
    {
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) sum = fmaf(to_float(v[e]), to_float(other.v[e]), sum);
        return sum;
    }
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

// ---- rows that are whole pieces of 16 bytes everywhere (N numbers a piece), or short ones (N 1) ----
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
                    if (a.weights) y.scale(weight);
                    y.store(to + c + i * lanes * N);
                }
        }
    }
}

// K choices of U pieces are asked for together
template <typename T, uint32_t N, uint32_t K, uint32_t U>
__global__ void __launch_bounds__(kThreads) k_combine(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    if (!w.live) return;
    T* const to = static_cast<T*>(a.rows) + w.row * a.ld_rows;
    for (uint32_t c0 = w.lane * N; c0 < a.cols; c0 += lanes * N * U) {
        float sum[U][N];
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) sum[u][e] = 0.f;
        for (uint32_t j = 0; j < a.choices; j += K) {
            Piece<T, N> y[K][U];
            bool live[K];
            float weight[K];
#pragma unroll
            for (uint32_t i = 0; i < K; ++i) {
                uint32_t place = 0;
                live[i] = j + i < a.choices && place_of(a, w.row, j + i, &place);
                if (live[i]) {
                    const T* const from = static_cast<const T*>(a.sorted) + place * a.ld_sorted + c0;
#pragma unroll
                    for (uint32_t u = 0; u < U; ++u)
                        if (c0 + u * lanes * N < a.cols) y[i][u].load(from + u * lanes * N);
                    weight[i] = a.weights ? a.weights[w.row * a.ld_weights + j + i] : 1.f;
                }
            }
#pragma unroll
            for (uint32_t i = 0; i < K; ++i)
                if (live[i])
#pragma unroll
                    for (uint32_t u = 0; u < U; ++u)
#pragma unroll
                        for (uint32_t e = 0; e < N; ++e) sum[u][e] = fmaf(weight[i], to_float(y[i][u].v[e]), sum[u][e]);
        }
#pragma unroll
        for (uint32_t u = 0; u < U; ++u)
            if (c0 + u * lanes * N < a.cols) {
                Piece<T, N> r;
#pragma unroll
                for (uint32_t e = 0; e < N; ++e) r.v[e] = from_float<T>(sum[u][e]);
                r.store(to + c0 + u * lanes * N);
            }
    }
}

// Sums of a row's threads, which the first of them stores.  The whole block calls it.
template <uint32_t JU>
__device__ __forceinline__ void store_dots(const RowSetArgs& a, const Where& w, uint32_t lanes, uint32_t j, float (&dot)[JU], float (*part)[JU])
{
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
#pragma unroll(JU > 2u ? 2 : 4)
            for (uint32_t c = w.lane * N; c < a.cols; c += lanes * N) {
                Piece<T, N> x, y[JU];
                x.load(from + c);
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i)
                    if (live[i]) y[i].load(static_cast<const T*>(a.sorted) + place[i] * a.ld_sorted + c);
#pragma unroll
                for (uint32_t i = 0; i < JU; ++i)
                    if (live[i]) {
                        dot[i] = x.dot(y[i], dot[i]);
                        Piece<T, N> d = x;
                        d.scale(weight[i]);
                        d.store(static_cast<T*>(a.d_sorted) + place[i] * a.ld_d_sorted + c);
                    }
            }
        store_dots<JU>(a, w, lanes, j, dot, part);
    }
}

// ---- rows of any alignment ----
// Pieces are those of the row that is written.  A piece that lies across two aligned ones of a row that is read is put together from both; at the ends of the array, where
// one of them would reach out of it, from single numbers.
template <typename T>
struct Any {
    static constexpr uint32_t N = 16u / sizeof(T);
    const uint8_t* first; const uint8_t* end;                // of the array

    __device__ __forceinline__ Any(const void* p, uint64_t rows, uint64_t ld, uint32_t cols)
        : first(static_cast<const uint8_t*>(p)), end(first + ((rows - 1u) * ld + cols) * sizeof(T)) {}
    __device__ __forceinline__ void load(const T* at, Piece<T, N>& to) const
    {
        const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(at) & 15u);
        const uint8_t* const base = reinterpret_cast<const uint8_t*>(at) - off;
        if (off == 0u) { to.load(at); return; }
        if (base < first || base + 32u > end) {
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) to.v[e] = at[e];
            return;
        }
        const uint4 a = __ldg(reinterpret_cast<const uint4*>(base)), b = __ldg(reinterpret_cast<const uint4*>(base) + 1);
        uint32_t w[8] = { a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w };
        if (off & 8u)
#pragma unroll
            for (uint32_t i = 0; i < 6u; ++i) w[i] = w[i + 2u];
        if (off & 4u)
#pragma unroll
            for (uint32_t i = 0; i < 5u; ++i) w[i] = w[i + 1u];
        if constexpr (sizeof(T) == 2)
#pragma unroll
            for (uint32_t i = 0; i < 4u; ++i) w[i] = __funnelshift_r(w[i], w[i + 1u], (off & 2u) * 8u);
        memcpy(to.v, w, 16);
    }
};
// A row of `cols` numbers from `to` on: `head` numbers up to the first 16-byte boundary, pieces, and the rest.  Thread t < singles() has the number single(t).
template <typename T>
struct Cut {
    static constexpr uint32_t N = 16u / sizeof(T);
    uint32_t head, pieces, cols;
    __device__ __forceinline__ Cut(const T* to, uint32_t n)
        : head(min(static_cast<uint32_t>((16u - (reinterpret_cast<uintptr_t>(to) & 15u)) & 15u) / static_cast<uint32_t>(sizeof(T)), n)), pieces((n - head) / N), cols(n) {}
    __device__ __forceinline__ uint32_t singles() const { return cols - pieces * N; }
    __device__ __forceinline__ uint32_t single(uint32_t t) const { return t < head ? t : t + pieces * N; }
};

template <typename T>
__global__ void __launch_bounds__(kThreads) k_take_any(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    constexpr uint32_t N = 16u / sizeof(T);
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    if (!w.live) return;
    const Any<T> any(a.rows, a.count, a.ld_rows, a.cols);
    const T* const from = static_cast<const T*>(a.rows) + w.row * a.ld_rows;
    for (uint32_t j = 0; j < a.choices; ++j) {
        uint32_t place;
        if (!place_of(a, w.row, j, &place)) continue;
        T* const to = static_cast<T*>(a.sorted) + place * a.ld_sorted;
        const float weight = a.weights ? a.weights[w.row * a.ld_weights + j] : 1.f;
        const Cut<T> cut(to, a.cols);
#pragma unroll 2
        for (uint32_t u = w.lane; u < cut.pieces; u += lanes) {
            Piece<T, N> x;
            any.load(from + cut.head + u * N, x);
            if (a.weights) x.scale(weight);
            x.store(to + cut.head + u * N);
        }
        for (uint32_t t = w.lane; t < cut.singles(); t += lanes) {
            const T x = from[cut.single(t)];
            to[cut.single(t)] = a.weights ? from_float<T>(weight * to_float(x)) : x;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_combine_any(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    constexpr uint32_t N = 16u / sizeof(T);
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    if (!w.live) return;
    const Any<T> any(a.sorted, a.sorted_rows, a.ld_sorted, a.cols);
    T* const to = static_cast<T*>(a.rows) + w.row * a.ld_rows;
    const Cut<T> cut(to, a.cols);
    for (uint32_t u = w.lane; u < cut.pieces; u += lanes) {
        float sum[N] = {};
#pragma unroll 2
        for (uint32_t j = 0; j < a.choices; ++j) {
            uint32_t place;
            if (!place_of(a, w.row, j, &place)) continue;
            const float weight = a.weights ? a.weights[w.row * a.ld_weights + j] : 1.f;
            Piece<T, N> y;
            any.load(static_cast<const T*>(a.sorted) + place * a.ld_sorted + cut.head + u * N, y);
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) sum[e] = fmaf(weight, to_float(y.v[e]), sum[e]);
        }
        Piece<T, N> r;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) r.v[e] = from_float<T>(sum[e]);
        r.store(to + cut.head + u * N);
    }
    for (uint32_t t = w.lane; t < cut.singles(); t += lanes) {
        float sum = 0.f;
        for (uint32_t j = 0; j < a.choices; ++j) {
            uint32_t place;
            if (!place_of(a, w.row, j, &place)) continue;
            sum = fmaf(a.weights ? a.weights[w.row * a.ld_weights + j] : 1.f, to_float(static_cast<const T*>(a.sorted)[place * a.ld_sorted + cut.single(t)]), sum);
        }
        to[cut.single(t)] = from_float<T>(sum);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_combine_backward_any(const __grid_constant__ RowSetArgs a, uint32_t lanes)
{
    constexpr uint32_t N = 16u / sizeof(T);
    __shared__ float part[kThreads / 32u][1];
    dep_wait();
    dep_trigger();
    const Where w = whose(a, lanes);
    const Any<T> any_x(a.rows, a.count, a.ld_rows, a.cols), any_y(a.sorted, a.sorted_rows, a.ld_sorted, a.cols);
    const T* const from = static_cast<const T*>(a.rows) + (w.live ? w.row : 0u) * a.ld_rows;
    for (uint32_t j = 0; j < a.choices; ++j) {
        uint32_t place = 0;
        float dot[1] = { 0.f };
        if (w.live && place_of(a, w.row, j, &place)) {
            const float weight = a.weights[w.row * a.ld_weights + j];
            const T* const y = static_cast<const T*>(a.sorted) + place * a.ld_sorted;
            T* const to = static_cast<T*>(a.d_sorted) + place * a.ld_d_sorted;
            const Cut<T> cut(to, a.cols);
#pragma unroll 2
            for (uint32_t u = w.lane; u < cut.pieces; u += lanes) {
                Piece<T, N> x, z;
                any_x.load(from + cut.head + u * N, x);
                any_y.load(y + cut.head + u * N, z);
                dot[0] = x.dot(z, dot[0]);
                x.scale(weight);
                x.store(to + cut.head + u * N);
            }
            for (uint32_t t = w.lane; t < cut.singles(); t += lanes) {
                const float x = to_float(from[cut.single(t)]);
                dot[0] = fmaf(x, to_float(y[cut.single(t)]), dot[0]);
                to[cut.single(t)] = from_float<T>(weight * x);
            }
        }
        store_dots<1>(a, w, lanes, j, dot, part);
    }
}

// ---- choices ----
// kPieces: 16 bytes everywhere; kShort: rows of less than 128 bytes, a number a thread; kAny (5,003 rows of 1,001 numbers of fp16, three choices: take 11.1 us number by number, 9.6 so; combine 26.3, 11.4; its
// gradient 37.7, 17.1)
enum Way { kPieces, kShort, kAny };
Way way_of(uint32_t size, const RowSetArgs& a)
{
    const uint64_t bits = reinterpret_cast<uintptr_t>(a.rows) | reinterpret_cast<uintptr_t>(a.sorted) | reinterpret_cast<uintptr_t>(a.d_sorted) |
                          (static_cast<uint64_t>(a.cols) | a.ld_rows | a.ld_sorted | a.ld_d_sorted) * size;
    return bits % 16u == 0u ? kPieces : a.cols * size < 128u ? kShort : kAny;
}

// threads of a row: `pieces_each` pieces a thread
uint32_t lanes_for(const RowSetArgs& a, uint32_t numbers, uint32_t pieces_each)
{
    const uint32_t pieces = (a.cols + numbers - 1u) / numbers;
    uint32_t lanes = 1;
    while (lanes < kThreads && lanes * pieces_each < pieces) lanes *= 2u;
    // few rows are spread over more threads
    while (lanes < kThreads && lanes < pieces && a.count * lanes < 512u * kSms) lanes *= 2u;
    return lanes;
}

template <class F>
int by_type(uint32_t type, F f) { return type == EVO_F32 ? f(float()) : type == EVO_BF16 ? f(__nv_bfloat16()) : f(__half()); }

int launch(cudaStream_t st, void (*kernel)(RowSetArgs, uint32_t), const RowSetArgs& a, uint32_t lanes)
{
    const uint64_t per = kThreads / lanes, blocks = (a.count + per - 1u) / per;
    if (blocks > 0x7FFFFFFFull) return -2;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(kThreads), 0, st, a, lanes) == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_take(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr uint32_t N = 16u / sizeof(T);
        const Way way = way_of(sizeof(T), a);
        return way == kPieces ? launch(st, k_take<T, N>, a, lanes_for(a, N, 4u)) : way == kShort ? launch(st, k_take<T, 1>, a, lanes_for(a, 1u, 4u))
                              : launch(st, k_take_any<T>, a, lanes_for(a, N, 2u));
    });
}
int launch_combine(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr uint32_t N = 16u / sizeof(T);
        const Way way = way_of(sizeof(T), a);
        if (way == kAny) return launch(st, k_combine_any<T>, a, lanes_for(a, N, 2u));
        if (way == kShort) return launch(st, k_combine<T, 1, 4, 1>, a, lanes_for(a, 1u, 1u));
        return a.choices == 1u ? launch(st, k_combine<T, N, 1, 4>, a, lanes_for(a, N, 8u)) : a.choices == 2u ? launch(st, k_combine<T, N, 2, 4>, a, lanes_for(a, N, 8u))
                               : launch(st, k_combine<T, N, 4, 2>, a, lanes_for(a, N, 8u));
    });
}
int launch_combine_backward(cudaStream_t st, uint32_t type, const RowSetArgs& a)
{
    return by_type(type, [&](auto t) {
        using T = decltype(t);
        constexpr uint32_t N = 16u / sizeof(T);
        const Way way = way_of(sizeof(T), a);
        // (2 / 4 / 8 pieces a thread, each of two or three loads: 5,003 x 1,001 of fp16, three choices 19.1 / 17.1 / 23 us, 20,000 x 333 of fp32, two 52.6 / 39.1 / 37.8)
        if (way == kAny) return launch(st, k_combine_backward_any<T>, a, lanes_for(a, N, 4u));
        if (way == kShort) return launch(st, k_combine_backward<T, 1, 4>, a, lanes_for(a, 1u, 1u));
        auto kernel = a.choices == 1u ? k_combine_backward<T, N, 1> : a.choices == 2u ? k_combine_backward<T, N, 2> : k_combine_backward<T, N, 4>;
        return launch(st, kernel, a, lanes_for(a, N, 8u));
    });
}

}  // namespace evo

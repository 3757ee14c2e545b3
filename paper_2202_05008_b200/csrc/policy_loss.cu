// Clipped policy loss of rows of logits and its gradient, one pass over the logits.
//
//   e_v = exp(x_v - max), s = sum e_v, logp = x_a - max - log s;  gradient_v = w c ([v = a] - e_v / s)
// A row stays in registers between its two uses (the sum and the gradient), so that it is read once and its gradient written once: that
// traffic is the bound for long rows, the launch for few short ones.  Rows of up to 256 actions are a part of a warp's, number by number; longer ones a warp's or a block's, in
// pieces of 16 bytes from the row's first 16-byte boundary on (the ends in single numbers), where logits and gradient lie alike; other rows, and rows longer than a block's
// registers hold, are read twice, the second time mostly from L2.
// One thread has the row's scalars in fp64: the ratio may lie close to a border, and 1 - p of the chosen action is a difference.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>
#include <type_traits>

#include "policy_loss.h"

namespace evo {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

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
// e^(x - top), 1 for the maximum itself.  (The difference first: x log2 e may leave fp32's range, and all of a row may be the type's lowest number.)
__device__ __forceinline__ float exp_below(float x, float top)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"((x - top) * kLog2e));
    return y;
}

struct Row { int64_t action; double weight; bool live; };
__device__ __forceinline__ Row row_of(const PolicyArgs& a, uint64_t row)
{
    Row r;
    r.action = a.wide ? static_cast<const int64_t*>(a.action)[row] : static_cast<const int32_t*>(a.action)[row];
    r.weight = a.weights ? static_cast<double>(a.weights[row]) : a.even;
    r.live = r.action >= 0 && r.action < static_cast<int64_t>(a.n) && r.weight != 0.0;
    return r;
}

// What follows from the row's maximum and s = sum of e^(x - top).  `all`: the factor of e^(x - top) in the gradient, `chosen`: the gradient of the action.
__device__ __forceinline__ void finish_row(const PolicyArgs& a, uint64_t row, const Row& r, float chosen_logit, float top, float s, float* all, float* chosen)
{
    const double logp = static_cast<double>(chosen_logit) - static_cast<double>(top) - log(static_cast<double>(s));
    const double adv = a.advantage[row], ratio = exp(logp - static_cast<double>(a.old_logp[row]));
    const bool clipped = adv >= 0.0 ? ratio > 1.0 + a.clip_high : ratio < 1.0 - a.clip_low;
    double loss = -adv * (clipped ? (adv >= 0.0 ? 1.0 + a.clip_high : 1.0 - a.clip_low) : ratio);
    double c = clipped ? 0.0 : -adv * ratio;
    if (!(ratio == ratio)) loss = c = ratio;                 // (a NaN compares as not clipped for either sign, but 0 times it is one too)
    if (a.ref_logp) {
        const double d = static_cast<double>(a.ref_logp[row]) - logp, e = expm1(d);
        loss += a.kl * (e - d);
        c -= a.kl * e;
    }
    c *= r.weight;
    *all = static_cast<float>(-c / static_cast<double>(s));
    *chosen = static_cast<float>(-c * expm1(logp));
    if (a.logp) a.logp[row] = static_cast<float>(logp);
    if (a.row_loss) a.row_loss[row] = r.weight * loss;
}
__device__ __forceinline__ void padded_row(const PolicyArgs& a, uint64_t row)
{
    if (a.logp) a.logp[row] = 0.f;
    if (a.row_loss) a.row_loss[row] = 0.0;
}

// Up to L E actions: L lanes a row, E numbers each.
template <typename T, uint32_t L, uint32_t E>
__global__ void __launch_bounds__(128) k_policy_short(const __grid_constant__ PolicyArgs a)
{
    dep_wait();
    dep_trigger();
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * (128u / L) + threadIdx.x / L;
    const uint32_t lane = threadIdx.x % L;
    Row r;
    r.live = false;
    if (row < a.rows) r = row_of(a, row);
    const T* const x = static_cast<const T*>(a.logits) + (r.live ? row : 0u) * a.ld;
    float v[E], top = -INFINITY;
#pragma unroll
    for (uint32_t i = 0; i < E; ++i) v[i] = r.live && lane + L * i < a.n ? to_float(x[lane + L * i]) : -INFINITY;
    const float chosen_logit = r.live ? to_float(x[r.action]) : 0.f;
#pragma unroll
    for (uint32_t i = 0; i < E; ++i) top = fmaxf(top, v[i]);
#pragma unroll
    for (uint32_t d = L / 2u; d > 0u; d /= 2u) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    float s = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < E; ++i)
        if (lane + L * i < a.n) {
            v[i] = exp_below(v[i], top);
            s += v[i];
        }
#pragma unroll
    for (uint32_t d = L / 2u; d > 0u; d /= 2u) s += __shfl_xor_sync(0xffffffffu, s, d);
    float all = 0.f, chosen = 0.f;
    if (lane == 0u && row < a.rows) {
        if (r.live) finish_row(a, row, r, chosen_logit, top, s, &all, &chosen);
        else padded_row(a, row);
    }
    all = __shfl_sync(0xffffffffu, all, 0, L);
    chosen = __shfl_sync(0xffffffffu, chosen, 0, L);
    if (row >= a.rows || !a.gradient) return;
    T* const g = static_cast<T*>(a.gradient) + row * a.ld_gradient;
#pragma unroll
    for (uint32_t i = 0; i < E; ++i) {
        const uint32_t k = lane + L * i;
        if (k < a.n) g[k] = from_float<T>(!r.live ? 0.f : k == static_cast<uint64_t>(r.action) ? chosen : all * v[i]);
    }
}

// Maximum or sum over a block (one warp: no shared memory)
template <uint32_t THREADS, bool MAX>
__device__ __forceinline__ float over_block(float x, float* part)
{
#pragma unroll
    for (uint32_t d = 16u; d > 0u; d /= 2u) {
        const float y = __shfl_xor_sync(0xffffffffu, x, d);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    if constexpr (THREADS > 32u) {
        if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = x;
        __syncthreads();
        x = part[threadIdx.x & 31u & (THREADS / 32u - 1u)];
#pragma unroll
        for (uint32_t d = THREADS / 64u; d > 0u; d /= 2u) {
            const float y = __shfl_xor_sync(0xffffffffu, x, d);
            x = MAX ? fmaxf(x, y) : x + y;
        }
    }
    return x;
}

template <typename T> struct Sixteen {
    static constexpr uint32_t N = 16u / sizeof(T);
    T v[N];
    __device__ __forceinline__ void load(const T* p) { const uint4 r = *reinterpret_cast<const uint4*>(p); memcpy(v, &r, 16); }
    __device__ __forceinline__ void store(T* p) const { uint4 r; memcpy(&r, v, 16); *reinterpret_cast<uint4*>(p) = r; }
};

// A row in the registers of THREADS threads, NV pieces of 16 bytes and one single number each.
template <typename T, uint32_t THREADS, uint32_t NV>
__global__ void __launch_bounds__(THREADS < 128u ? 128u : THREADS) k_policy_row(const __grid_constant__ PolicyArgs a)
{
    constexpr uint32_t N = Sixteen<T>::N, kRows = THREADS < 128u ? 128u / THREADS : 1u;
    __shared__ float part[2][32], factors[2];
    dep_wait();
    dep_trigger();
    const uint64_t row = static_cast<uint64_t>(blockIdx.x) * kRows + threadIdx.x / THREADS;
    const uint32_t t = threadIdx.x % THREADS;
    if (row >= a.rows) return;                               // (whole warps)
    const Row r = row_of(a, row);
    const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
    T* const g = static_cast<T*>(a.gradient) + row * a.ld_gradient;
    // numbers in front of the first 16-byte boundary, pieces, and numbers behind them
    const uintptr_t address = reinterpret_cast<uintptr_t>(a.gradient ? static_cast<const void*>(g) : x);
    const uint32_t head = min(static_cast<uint32_t>((16u - (address & 15u)) & 15u) / static_cast<uint32_t>(sizeof(T)), a.n);
    const uint32_t pieces = (a.n - head) / N, tail = (a.n - head) % N;
    const bool has_single = t < head + tail;
    const uint32_t single = t < head ? t : head + pieces * N + (t - head);
    Sixteen<T> v[NV];
    if (!r.live) {
        if (t == 0u) padded_row(a, row);
        if (!a.gradient) return;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) v[0].v[e] = from_float<T>(0.f);
#pragma unroll
        for (uint32_t i = 0; i < NV; ++i)
            if (t + THREADS * i < pieces) v[0].store(g + head + (t + THREADS * i) * N);
        if (has_single) g[single] = from_float<T>(0.f);
        return;
    }
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < pieces) v[i].load(x + head + (t + THREADS * i) * N);
    const float alone = has_single ? to_float(x[single]) : -INFINITY;
    const float chosen_logit = t == 0u ? to_float(x[r.action]) : 0.f;
    float top = alone;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < pieces)
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) top = fmaxf(top, to_float(v[i].v[e]));
    top = over_block<THREADS, true>(top, part[0]);
    float s = has_single ? exp_below(alone, top) : 0.f;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < pieces) {
            float sum = 0.f;
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) sum += exp_below(to_float(v[i].v[e]), top);
            s += sum;
        }
    s = over_block<THREADS, false>(s, part[1]);
    float all = 0.f, chosen = 0.f;
    if (t == 0u) finish_row(a, row, r, chosen_logit, top, s, &all, &chosen);
    if (!a.gradient) return;
    if constexpr (THREADS > 32u) {
        if (t == 0u) { factors[0] = all; factors[1] = chosen; }
        __syncthreads();
        all = factors[0]; chosen = factors[1];
    } else {
        all = __shfl_sync(0xffffffffu, all, 0);
        chosen = __shfl_sync(0xffffffffu, chosen, 0);
    }
    // (the action's number is stored by the thread that has stored over it)
    const uint32_t action = static_cast<uint32_t>(r.action);
    bool mine = has_single && single == action;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < pieces) {
            Sixteen<T> y;
#pragma unroll
            for (uint32_t e = 0; e < N; ++e) y.v[e] = from_float<T>(all * exp_below(to_float(v[i].v[e]), top));
            y.store(g + head + (t + THREADS * i) * N);
            mine = mine || (action >= head && (action - head) / N == t + THREADS * i);
        }
    if (has_single) g[single] = from_float<T>(all * exp_below(alone, top));
    if (mine) g[action] = from_float<T>(chosen);
}

// Any length and alignment: a block a row, which is read twice, in pieces of N numbers (N 1: number by number).
constexpr uint32_t kLongThreads = 512;
template <typename T, bool PIECES>
__global__ void __launch_bounds__(kLongThreads) k_policy_long(const __grid_constant__ PolicyArgs a)
{
    constexpr uint32_t N = Sixteen<T>::N;
    __shared__ float part[2][32], factors[2];
    dep_wait();
    dep_trigger();
    const uint64_t row = blockIdx.x;
    const uint32_t t = threadIdx.x;
    const Row r = row_of(a, row);
    const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
    T* const g = static_cast<T*>(a.gradient) + row * a.ld_gradient;
    const uintptr_t address = reinterpret_cast<uintptr_t>(a.gradient ? static_cast<const void*>(g) : x);
    const uint32_t head = PIECES ? min(static_cast<uint32_t>((16u - (address & 15u)) & 15u) / static_cast<uint32_t>(sizeof(T)), a.n) : a.n;
    const uint32_t pieces = (a.n - head) / N, behind = head + pieces * N;
    if (!r.live) {
        if (t == 0u) padded_row(a, row);
        if (!a.gradient) return;
        Sixteen<T> zero;
#pragma unroll
        for (uint32_t e = 0; e < N; ++e) zero.v[e] = from_float<T>(0.f);
        for (uint32_t i = t; i < pieces; i += kLongThreads) zero.store(g + head + i * N);
        for (uint32_t k = t; k < head; k += kLongThreads) g[k] = zero.v[0];
        for (uint32_t k = behind + t; k < a.n; k += kLongThreads) g[k] = zero.v[0];
        return;
    }
    const float chosen_logit = t == 0u ? to_float(x[r.action]) : 0.f;
    // the thread's maximum, and its sum with that taken off (0 while it has seen forbidden actions alone)
    float top = -INFINITY, s = 0.f;
    auto add = [&](const float* v, uint32_t count) {
        float most = v[0];
        for (uint32_t e = 1; e < count; ++e) most = fmaxf(most, v[e]);
        if (most > top) { s *= exp_below(top, most); top = most; }
        const float off = top == -INFINITY ? 0.f : top;
        float sum = 0.f;
        for (uint32_t e = 0; e < count; ++e) sum += exp_below(v[e], off);
        s += sum;
    };
    constexpr uint32_t kAhead = 4;
    for (uint32_t i = t; i < pieces; i += kLongThreads * kAhead) {
        Sixteen<T> v[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + kLongThreads * k < pieces) v[k].load(x + head + (i + kLongThreads * k) * N);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + kLongThreads * k < pieces) {
                float f[N];
#pragma unroll
                for (uint32_t e = 0; e < N; ++e) f[e] = to_float(v[k].v[e]);
                add(f, N);
            }
    }
    for (uint32_t k = t; k < head; k += kLongThreads) { const float f = to_float(x[k]); add(&f, 1u); }
    for (uint32_t k = behind + t; k < a.n; k += kLongThreads) { const float f = to_float(x[k]); add(&f, 1u); }
    const float most = over_block<kLongThreads, true>(top, part[0]);
    s = over_block<kLongThreads, false>(s * exp_below(top, most), part[1]);
    float all = 0.f, chosen = 0.f;
    if (t == 0u) finish_row(a, row, r, chosen_logit, most, s, &all, &chosen);
    if (!a.gradient) return;
    if (t == 0u) { factors[0] = all; factors[1] = chosen; }
    __syncthreads();
    all = factors[0]; chosen = factors[1];
    const uint32_t action = static_cast<uint32_t>(r.action);
    for (uint32_t i = t; i < pieces; i += kLongThreads * kAhead) {
        Sixteen<T> v[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + kLongThreads * k < pieces) v[k].load(x + head + (i + kLongThreads * k) * N);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + kLongThreads * k < pieces) {
                const uint32_t at = head + (i + kLongThreads * k) * N;
                Sixteen<T> y;
#pragma unroll
                for (uint32_t e = 0; e < N; ++e) y.v[e] = from_float<T>(at + e == action ? chosen : all * exp_below(to_float(v[k].v[e]), most));
                y.store(g + at);
            }
    }
    for (uint32_t k = t; k < head; k += kLongThreads) g[k] = from_float<T>(k == action ? chosen : all * exp_below(to_float(x[k]), most));
    for (uint32_t k = behind + t; k < a.n; k += kLongThreads) g[k] = from_float<T>(k == action ? chosen : all * exp_below(to_float(x[k]), most));
}

// The sum over the rows: always the same parts in the same order.
__global__ void __launch_bounds__(1024) k_policy_sum(const double* __restrict__ rows, uint64_t n, float* __restrict__ loss)
{
    __shared__ double part[32];
    dep_wait();
    dep_trigger();
    double s[4] = {};
    for (uint64_t i = threadIdx.x; i < n; i += 4096u)
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k)
            if (i + 1024u * k < n) s[k] += rows[i + 1024u * k];
    double sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (uint32_t d = 16u; d > 0u; d /= 2u) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x < 32u) {
        sum = part[threadIdx.x];
#pragma unroll
        for (uint32_t d = 16u; d > 0u; d /= 2u) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (threadIdx.x == 0u) *loss = static_cast<float>(sum);
    }
}

template <typename T>
int launch_rows(cudaStream_t st, const PolicyArgs& a)
{
    constexpr uint32_t N = Sixteen<T>::N;
    void (*kernel)(PolicyArgs) = nullptr;
    uint32_t threads = 128, per = 1;
    const bool alike = !a.gradient || ((reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.gradient)) % 16u == 0u &&
                                       (a.rows < 2u || (a.ld - a.ld_gradient) * sizeof(T) % 16u == 0u));
    if (a.n <= 32u) { kernel = k_policy_short<T, 8, 4>; per = 16u; }
    else if (a.n <= 256u) { kernel = k_policy_short<T, 32, 8>; per = 4u; }
    else if (!alike) { kernel = k_policy_long<T, false>; threads = kLongThreads; }
    else if (a.n <= 32u * 4u * N) { kernel = k_policy_row<T, 32, 4>; per = 4u; }
    else if (a.n <= 128u * 4u * N) kernel = k_policy_row<T, 128, 4>;
    else if (a.n <= 128u * 8u * N) kernel = k_policy_row<T, 128, 8>;
    else if (a.n <= 512u * 4u * N) { kernel = k_policy_row<T, 512, 4>; threads = 512u; }
    else if (a.n <= 512u * 8u * N) { kernel = k_policy_row<T, 512, 8>; threads = 512u; }
    else if (a.n <= 512u * 16u * N) { kernel = k_policy_row<T, 512, 16>; threads = 512u; }
    else { kernel = k_policy_long<T, true>; threads = kLongThreads; }
    const uint64_t blocks = (a.rows + per - 1u) / per;
    if (blocks > 0x7FFFFFFFull) return -2;
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(threads), 0, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_policy_loss(cudaStream_t st, uint32_t type, const PolicyArgs& a)
{
    int n = 0;
    if (a.rows) {
        n = type == EVO_F32 ? launch_rows<float>(st, a) : type == EVO_BF16 ? launch_rows<__nv_bfloat16>(st, a) : launch_rows<__half>(st, a);
        if (n < 0) return n;
    }
    if (!a.loss) return n;
    return launch_dependent(k_policy_sum, dim3(1), dim3(1024), 0, st, a.row_loss, a.rows, a.loss) == cudaSuccess ? n + 1 : -1;
}

}  // namespace evo

// Clipped policy loss of rows of logits and its gradient.
//
//   e_v = exp(x_v - max), s = sum e_v, logp = x_a - max - log s;  gradient_v = w c ([v = a] - e_v / s)
// Rows of up to 256 actions are a part of a warp's, number by number, and rows of up to 4 KB a warp's, in pieces of 16 bytes from the row's first 16-byte boundary on (the ends in single
// numbers): they stay in registers between their two uses, the sum and the gradient.  Longer rows are a block's and are read twice, the second time mostly from L2.  So are all rows above 256
// actions whose logits and gradient do not begin alike modulo 16 bytes, number by number.  A lane, or one thread of a block, has a row's scalars.
// Many short rows are bound by those and by issue (4,000,000 of 64: fp32 470 us, 4.4 TB/s, bf16 586; 100,000 of 300 bf16 83, of 900 106, of 2,000 158, 5.1 TB/s), long ones by memory and the
// exponentials (8,192 of 32,000 bf16 196 to 211), few by the launch and by a row's way through one block (1 to 148 rows of 130,000 bf16 20 us a call).  Rows that do not lie alike take
// two to six times as long: bf16 of pitch 50,304, 4,096 of 50,257 340 us against 165, 100,000 of 300 in a pitch of 304 509 against 83.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <cstring>
#include <type_traits>

#include "async.cuh"
#include "policy_loss.h"

namespace evo {
namespace {

constexpr uint32_t kMostBlocks = 8;          // of a cluster
constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = static_cast<float>(1.4426950408889634 - static_cast<double>(kLog2e)), kLn2f = 0.69314718055994530942f;
constexpr double kLn2 = 0.69314718055994530942;

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
// Two at once: additions and products of pairs are one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long*>(&r))
        : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*reinterpret_cast<unsigned long long*>(&r))
        : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)));
    return r;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(*reinterpret_cast<unsigned long long*>(&r))
        : "l"(*reinterpret_cast<const unsigned long long*>(&a)), "l"(*reinterpret_cast<const unsigned long long*>(&b)), "l"(*reinterpret_cast<const unsigned long long*>(&c)));
    return r;
}
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float power2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// what has a power that is 0 anyway is cut off (an infinite difference has no rest); a NaN stays one
__device__ __forceinline__ float no_less(float t)
{
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(t), "f"(-256.f));
    return r;
}

// e^(x - top), 1 for the maximum itself; numbers below 2^-126 are 0.  (The difference first: x log2 e may leave fp32's range, and all of a row may be the type's lowest number.)
// y = (x - top) log2 e is rounded, which of a large difference R is R 1.25 2^-24 of the result.  WHOLE (fp32): what y leaves is put right, e^(x - top) = 2^y (1 + ln 2 rest), so that
// the difference's own rounding is what is left.  Numbers of 16 bits do without: R would have to be in the hundreds to be seen in them, and a long row of bf16 is bound by issue (8,192 of
// 32,000: 197 us without, 264 with; of fp32 4,096 of 32,000 200 and 202, 100,000 of 900 150 and 158, 1,000,000 of 12 63).
template <typename T> constexpr bool kWhole = std::is_same<T, float>::value;
template <bool WHOLE>
__device__ __forceinline__ float exp_below(float x, float top)
{
    if constexpr (!WHOLE) return power2((x - top) * kLog2e);
    const float t = no_less(x - top), y = t * kLog2e, r = power2(y);
    return fmaf(r * kLn2f, fmaf(t, kLog2eRest, fmaf(t, kLog2e, -y)), r);
}
template <bool WHOLE>
__device__ __forceinline__ float2 exp_below2(float2 x, float top)
{
    float2 t = add2(x, both(-top));
    if constexpr (WHOLE) t = make_float2(no_less(t.x), no_less(t.y));
    const float2 y = mul2(t, both(kLog2e)), r = make_float2(power2(y.x), power2(y.y));
    if constexpr (!WHOLE) return r;
    return fma2(mul2(r, both(kLn2f)), fma2(t, both(kLog2eRest), fma2(t, both(kLog2e), make_float2(-y.x, -y.y))), r);
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

// e^x in fp32's precision and fp64's range: its product with a weight or an advantage may be an fp32 number where it is none itself.
__device__ __forceinline__ double exp_far(double x)
{
    if (fabs(x) < 80.0) return static_cast<double>(expf(static_cast<float>(x)));
    if (!(fabs(x) < 700.0)) return x > 0.0 ? static_cast<double>(INFINITY) : x < 0.0 ? 0.0 : x;      // (a NaN)
    const double k = rint(x * static_cast<double>(kLog2e));
    return scalbn(static_cast<double>(expf(static_cast<float>(fma(-kLn2, k, x)))), static_cast<int>(k));
}

// What follows from the row's maximum and s = sum of e^(x - top), 1 at least.  `all`: the factor of e^(x - top) in the gradient, `chosen`: the gradient of the action.
// Differences are taken in fp64, functions of them in fp32: log s of its exponent and of a number close to 1, the ratio's borders as logarithms, 1 - p as an expm1,
// e^d - 1 - d as its series where it is a small difference.  Returns the row's share of the loss.
__device__ __forceinline__ double finish_row(const PolicyArgs& a, uint64_t row, const Row& r, float chosen_logit, float top, float s, float* all, float* chosen)
{
    const uint32_t bits = __float_as_uint(s);
    const int32_t exponent = static_cast<int32_t>(bits - 0x3F400000u) >> 23;      // s = m 2^exponent, m from 0.75 up to 1.5
    const float m = __uint_as_float(bits - (static_cast<uint32_t>(exponent) << 23));
    double logp = static_cast<double>(chosen_logit) - static_cast<double>(top) - fma(kLn2, static_cast<double>(exponent), static_cast<double>(logf(m)));
    if (!(s >= 1.f)) logp = static_cast<double>(s);          // (a NaN)
    const double log_ratio = logp - static_cast<double>(a.old_logp[row]);
    const float adv = a.advantage[row];
    const double ratio = exp_far(log_ratio);
    const bool clipped = adv >= 0.f ? log_ratio > a.log_high : log_ratio < a.log_low;
    double loss = -static_cast<double>(adv) * (clipped ? (adv >= 0.f ? 1.0 + a.clip_high : 1.0 - a.clip_low) : ratio);
    double c = clipped ? 0.0 : -static_cast<double>(adv) * ratio;
    if (a.ref_logp) {
        const double far = static_cast<double>(a.ref_logp[row]) - logp;
        const float d = static_cast<float>(far), near = expm1f(d);
        double e = near, rest = near - d;
        if (d >= 80.f) {
            e = exp_far(far) - 1.0;
            rest = e - far;
        } else if (fabsf(d) < 0.5f) {                        // (what is left out is below 4e-8 of it)
            float q = 1.f / 40320.f;
            q = fmaf(q, d, 1.f / 5040.f); q = fmaf(q, d, 1.f / 720.f); q = fmaf(q, d, 1.f / 120.f); q = fmaf(q, d, 1.f / 24.f); q = fmaf(q, d, 1.f / 6.f); q = fmaf(q, d, 0.5f);
            rest = d * d * q;
        }
        loss += a.kl * rest;
        c -= a.kl * e;
    }
    c *= r.weight;
    *all = static_cast<float>(-c) / s;
    *chosen = static_cast<float>(-c) * expm1f(static_cast<float>(logp));
    if (a.logp) a.logp[row] = static_cast<float>(logp);
    loss *= r.weight;
    if (a.row_loss) a.row_loss[row] = loss;
    return loss;
}
__device__ __forceinline__ void padded_row(const PolicyArgs& a, uint64_t row)
{
    if (a.logp) a.logp[row] = 0.f;
    if (a.row_loss) a.row_loss[row] = 0.0;
}

// Up to L E actions: L lanes a row, E numbers each; a warp has R times 32 / L rows one behind the other, and a lane finishes each of them (a
// row's scalars in fp64 cost more than its numbers: 4 million rows of 64 took 2,870 us with a row a time, fp32 470 and bf16 586 so).
// ONE: the grid is one cluster, whose blocks' shares of the loss meet in the first one's shared memory, added up in their order: no second launch (1,024 rows of 12: a call
// from Python 21 -> 18.7 us, on the device 5.4 -> 4.7).
template <typename T, uint32_t L, uint32_t E, uint32_t R, bool ONE>
__global__ void __launch_bounds__(128) k_policy_short(const __grid_constant__ PolicyArgs a)
{
    constexpr uint32_t kAcross = 32u / L, kRows = kAcross * R;
    static_assert(kRows <= 32u, "a lane a row");
    dep_wait();
    dep_trigger();
    if constexpr (ONE) {
        __syncwarp();                                        // (.aligned: a warp comes to it as one)
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");         // (that the first block has begun)
    }
    const uint32_t all_lanes = threadIdx.x % 32u, lane = all_lanes % L, nth = all_lanes / L;
    const uint64_t first = (static_cast<uint64_t>(blockIdx.x) * 4u + threadIdx.x / 32u) * kRows;
    if (!ONE && first >= a.rows) return;                     // (whole warps)
    // the lane's own row
    const uint64_t mine = first + all_lanes;
    Row r;
    r.live = false; r.action = 0; r.weight = 0.0;
    float chosen_logit = 0.f;
    if (all_lanes < kRows && mine < a.rows) {
        r = row_of(a, mine);
        if (r.live) chosen_logit = to_float(static_cast<const T*>(a.logits)[mine * a.ld + r.action]);
    }
    float v[R][E], my_top = 0.f, my_sum = 1.f;
    const uint32_t live = __ballot_sync(0xffffffffu, r.live);
#pragma unroll
    for (uint32_t p = 0; p < R; ++p) {
        const uint32_t row = p * kAcross + nth;
        const T* const x = static_cast<const T*>(a.logits) + (first + row) * a.ld;
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) v[p][i] = live >> row & 1u && lane + L * i < a.n ? to_float(x[lane + L * i]) : -INFINITY;
    }
#pragma unroll
    for (uint32_t p = 0; p < R; ++p) {
        float top = -INFINITY, s = 0.f;
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) top = fmaxf(top, v[p][i]);
#pragma unroll
        for (uint32_t d = L / 2u; d > 0u; d /= 2u) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
#pragma unroll
        for (uint32_t i = 0; i < E; i += 2u) {               // (behind the row's end minus infinity)
            const float2 e = exp_below2<kWhole<T>>(make_float2(v[p][i], v[p][i + 1u]), top);
            v[p][i] = e.x;
            v[p][i + 1u] = e.y;
            s += e.x;
            s += e.y;
        }
#pragma unroll
        for (uint32_t d = L / 2u; d > 0u; d /= 2u) s += __shfl_xor_sync(0xffffffffu, s, d);
        const float t = __shfl_sync(0xffffffffu, top, all_lanes % kAcross * L), u = __shfl_sync(0xffffffffu, s, all_lanes % kAcross * L);
        if (all_lanes / kAcross == p) { my_top = t; my_sum = u; }
    }
    float all = 0.f, chosen = 0.f;
    double loss = 0.0;
    if (all_lanes < kRows && mine < a.rows) {
        if (r.live) loss = finish_row(a, mine, r, chosen_logit, my_top, my_sum, &all, &chosen);
        else padded_row(a, mine);
    }
    if constexpr (ONE) {
        __shared__ double warps[4], blocks[kMostBlocks];
#pragma unroll
        for (uint32_t d = 16u; d > 0u; d /= 2u) loss += __shfl_xor_sync(0xffffffffu, loss, d);
        if (all_lanes == 0u) warps[threadIdx.x / 32u] = loss;
        __syncwarp();
        asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        __syncthreads();
        if (threadIdx.x == 0u) {
            uint32_t there;
            asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(there) : "r"(smem_u32(blocks + blockIdx.x)));
            asm volatile("st.shared::cluster.f64 [%0], %1;" :: "r"(there), "d"((warps[0] + warps[1]) + (warps[2] + warps[3])) : "memory");
        }
        __syncwarp();
        asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
        if (blockIdx.x == 0u && threadIdx.x == 0u) {
            loss = 0.0;
            for (uint32_t k = 0; k < gridDim.x; ++k) loss += blocks[k];
            *a.loss = static_cast<float>(loss);
        }
    }
    if (!a.gradient) return;
#pragma unroll
    for (uint32_t p = 0; p < R; ++p) {
        const uint32_t row = p * kAcross + nth;
        const float f = __shfl_sync(0xffffffffu, all, row), c = __shfl_sync(0xffffffffu, chosen, row);
        const uint32_t action = __shfl_sync(0xffffffffu, static_cast<uint32_t>(r.action), row);
        if (first + row >= a.rows) continue;
        T* const g = static_cast<T*>(a.gradient) + (first + row) * a.ld_gradient;
#pragma unroll
        for (uint32_t i = 0; i < E; ++i) {
            const uint32_t k = lane + L * i;
            if (k < a.n) g[k] = from_float<T>(!(live >> row & 1u) ? 0.f : k == action ? c : f * v[p][i]);
        }
    }
}

template <bool MAX>
__device__ __forceinline__ float over_warp(float x)
{
#pragma unroll
    for (uint32_t d = 16u; d > 0u; d /= 2u) {
        const float y = __shfl_xor_sync(0xffffffffu, x, d);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    return x;
}
// Maximum or sum over a block; `part` has room for its warps.
template <uint32_t THREADS, bool MAX>
__device__ __forceinline__ float over_block(float x, float* part)
{
    constexpr uint32_t kWarps = THREADS / 32u;
    x = over_warp<MAX>(x);
    if ((threadIdx.x & 31u) == 0u) part[threadIdx.x / 32u] = x;
    __syncthreads();
    x = part[threadIdx.x % kWarps];
#pragma unroll
    for (uint32_t d = kWarps / 2u; d > 0u; d /= 2u) {
        const float y = __shfl_xor_sync(0xffffffffu, x, d);
        x = MAX ? fmaxf(x, y) : x + y;
    }
    return x;
}

// 16 bytes of a row: kept as they were loaded, since numbers taken apart are twice the registers.
template <typename T> struct Sixteen {
    static constexpr uint32_t N = 16u / sizeof(T);
    uint32_t w[4];
    __device__ __forceinline__ void load(const T* p) { const uint4 r = *reinterpret_cast<const uint4*>(p); w[0] = r.x; w[1] = r.y; w[2] = r.z; w[3] = r.w; }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]); }
    __device__ __forceinline__ void numbers(float2 (&f)[N / 2u]) const
    {
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            if constexpr (std::is_same<T, float>::value) (i % 2u ? f[i / 2u].y : f[i / 2u].x) = __uint_as_float(w[i]);
            else if constexpr (std::is_same<T, __half>::value) f[i] = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            else f[i] = make_float2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
        }
    }
    __device__ __forceinline__ void round(const float2 (&f)[N / 2u])
    {
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            if constexpr (std::is_same<T, float>::value) {
                w[i] = __float_as_uint(i % 2u ? f[i / 2u].y : f[i / 2u].x);
            } else if constexpr (std::is_same<T, __half>::value) {
                const __half2 two = __floats2half2_rn(f[i].x, f[i].y);
                w[i] = *reinterpret_cast<const uint32_t*>(&two);
            } else {
                const __nv_bfloat162 two = __floats2bfloat162_rn(f[i].x, f[i].y);
                w[i] = *reinterpret_cast<const uint32_t*>(&two);
            }
        }
    }
    // the larger of each pair of numbers, in the type itself (of a number and a NaN the number)
    __device__ __forceinline__ void larger(const Sixteen& other)
    {
#pragma unroll
        for (uint32_t i = 0; i < 4u; ++i) {
            if constexpr (std::is_same<T, float>::value) {
                w[i] = __float_as_uint(fmaxf(__uint_as_float(w[i]), __uint_as_float(other.w[i])));
            } else if constexpr (std::is_same<T, __half>::value) {
                const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&w[i]), *reinterpret_cast<const __half2*>(&other.w[i]));
                w[i] = *reinterpret_cast<const uint32_t*>(&m);
            } else {
                const __nv_bfloat162 m = __hmax2(*reinterpret_cast<const __nv_bfloat162*>(&w[i]), *reinterpret_cast<const __nv_bfloat162*>(&other.w[i]));
                w[i] = *reinterpret_cast<const uint32_t*>(&m);
            }
        }
    }
    __device__ __forceinline__ float largest() const
    {
        float2 f[N / 2u];
        numbers(f);
        float top = fmaxf(f[0].x, f[0].y);
#pragma unroll
        for (uint32_t i = 1; i < N / 2u; ++i) top = fmaxf(top, fmaxf(f[i].x, f[i].y));
        return top;
    }
    // sum of e^(x - top)
    __device__ __forceinline__ float sum_below(float top) const
    {
        float2 f[N / 2u], sum = make_float2(0.f, 0.f);
        numbers(f);
#pragma unroll
        for (uint32_t i = 0; i < N / 2u; ++i) sum = add2(sum, exp_below2<kWhole<T>>(f[i], top));
        return sum.x + sum.y;
    }
    // every number to factor e^(x - top)
    __device__ __forceinline__ void scale_below(float top, float factor)
    {
        float2 f[N / 2u];
        numbers(f);
#pragma unroll
        for (uint32_t i = 0; i < N / 2u; ++i) f[i] = mul2(exp_below2<kWhole<T>>(f[i], top), make_float2(factor, factor));
        round(f);
    }
};

// A row in the registers of a warp, NV pieces of 16 bytes and one single number a lane; the scalars of a block's eight rows are finished by a warp side by side.
template <typename T, uint32_t NV>
__global__ void __launch_bounds__(256, 4) k_policy_row(const __grid_constant__ PolicyArgs a)
{
    constexpr uint32_t N = Sixteen<T>::N, THREADS = 32, kRows = 8;
    __shared__ float tops[kRows], sums[kRows], alls[kRows], chosens[kRows];
    dep_wait();
    dep_trigger();
    const uint32_t t = threadIdx.x % THREADS, nth = threadIdx.x / THREADS;
    const uint64_t first = static_cast<uint64_t>(blockIdx.x) * kRows, row = first + nth;
    const bool exists = row < a.rows;
    bool live = false;
    uint32_t action = 0;
    if (exists) {
        const Row r = row_of(a, row);
        live = r.live;
        action = static_cast<uint32_t>(r.action);
    }
    const T* const x = static_cast<const T*>(a.logits) + row * a.ld;
    T* const g = static_cast<T*>(a.gradient) + row * a.ld_gradient;
    // numbers in front of the first 16-byte boundary, pieces, and numbers behind them
    const uintptr_t address = reinterpret_cast<uintptr_t>(a.gradient ? static_cast<const void*>(g) : x);
    const uint32_t head = min(static_cast<uint32_t>((16u - (address & 15u)) & 15u) / static_cast<uint32_t>(sizeof(T)), a.n);
    const uint32_t pieces = (a.n - head) / N, tail = (a.n - head) % N;
    const bool has_single = exists && t < head + tail;
    const uint32_t single = t < head ? t : head + pieces * N + (t - head);
    const uint32_t mine = live ? pieces : 0u;                // (of a row that is padding nothing is read)
    Sixteen<T> v[NV];
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < mine) v[i].load(x + head + (t + THREADS * i) * N);
    const float alone = has_single && live ? to_float(x[single]) : -INFINITY;
    // the first warp has the rows' scalars, a lane each
    Row r;
    float chosen_logit = 0.f;
    const bool finishes = threadIdx.x < kRows && first + threadIdx.x < a.rows;
    if (finishes) {
        r = row_of(a, first + threadIdx.x);
        if (r.live) chosen_logit = to_float(static_cast<const T*>(a.logits)[(first + threadIdx.x) * a.ld + r.action]);
    }
    float top = alone;
    if (t < mine) {
        Sixteen<T> most = v[0];
#pragma unroll
        for (uint32_t i = 1; i < NV; ++i)
            if (t + THREADS * i < mine) most.larger(v[i]);
        top = fmaxf(top, most.largest());
    }
    top = over_warp<true>(top);
    float s = has_single && live ? exp_below<kWhole<T>>(alone, top) : 0.f;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < mine) s += v[i].sum_below(top);
    s = over_warp<false>(s);
    if (t == 0u) { tops[nth] = top; sums[nth] = s; }
    __syncthreads();
    if (finishes) {
        float all = 0.f, chosen = 0.f;
        if (r.live) finish_row(a, first + threadIdx.x, r, chosen_logit, tops[threadIdx.x], sums[threadIdx.x], &all, &chosen);
        else padded_row(a, first + threadIdx.x);
        alls[threadIdx.x] = all;
        chosens[threadIdx.x] = chosen;
    }
    if (!a.gradient) return;
    __syncthreads();
    if (!exists) return;
    const float all = alls[nth], chosen = chosens[nth];
    // (the action's number is stored by the thread that has stored over it)
    bool own = has_single && single == action;
#pragma unroll
    for (uint32_t i = 0; i < NV; ++i)
        if (t + THREADS * i < pieces) {
            if (live) v[i].scale_below(top, all);
            else v[i].w[0] = v[i].w[1] = v[i].w[2] = v[i].w[3] = 0u;
            v[i].store(g + head + (t + THREADS * i) * N);
            own = own || (action >= head && (action - head) / N == t + THREADS * i);
        }
    if (has_single) g[single] = from_float<T>(live ? all * exp_below<kWhole<T>>(alone, top) : 0.f);
    if (own && live) g[action] = from_float<T>(chosen);
}

// Any length and alignment: a block a row, which is read twice, the second time from L2 as a rule (holding it in registers or shared memory leaves fewer rows in flight and
// measured slower: 32,000 of bf16 230 us in registers, 198 like this), in pieces of 16 bytes or (PIECES false) number by number.
template <typename T, bool PIECES, uint32_t THREADS>
__global__ void __launch_bounds__(THREADS) k_policy_long(const __grid_constant__ PolicyArgs a)
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
        zero.w[0] = zero.w[1] = zero.w[2] = zero.w[3] = 0u;
        for (uint32_t i = t; i < pieces; i += THREADS) zero.store(g + head + i * N);
        for (uint32_t k = t; k < head; k += THREADS) g[k] = from_float<T>(0.f);
        for (uint32_t k = behind + t; k < a.n; k += THREADS) g[k] = from_float<T>(0.f);
        return;
    }
    const float chosen_logit = t == 0u ? to_float(x[r.action]) : 0.f;
    // the thread's maximum, and its sum with that taken off (0 while it has seen forbidden actions alone)
    float top = -INFINITY, s = 0.f;
    auto raise = [&](float most) {
        if (most > top) { s *= exp_below<kWhole<T>>(top, most); top = most; }
        return top == -INFINITY ? 0.f : top;
    };
    constexpr uint32_t kAhead = 4;
    for (uint32_t i = t; i < pieces; i += THREADS * kAhead) {
        Sixteen<T> v[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + THREADS * k < pieces) v[k].load(x + head + (i + THREADS * k) * N);
        Sixteen<T> most = v[0];
#pragma unroll
        for (uint32_t k = 1; k < kAhead; ++k)
            if (i + THREADS * k < pieces) most.larger(v[k]);
        const float off = raise(most.largest());
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + THREADS * k < pieces) s += v[k].sum_below(off);
    }
    auto add = [&](float x) { s += exp_below<kWhole<T>>(x, raise(x)); };
    for (uint32_t k = t; k < head; k += THREADS) add(to_float(x[k]));
    for (uint32_t k = behind + t; k < a.n; k += THREADS) add(to_float(x[k]));
    const float most = over_block<THREADS, true>(top, part[0]);
    s = over_block<THREADS, false>(s * exp_below<kWhole<T>>(top, most), part[1]);
    float all = 0.f, chosen = 0.f;
    if (t == 0u) finish_row(a, row, r, chosen_logit, most, s, &all, &chosen);
    if (!a.gradient) return;
    if (t == 0u) { factors[0] = all; factors[1] = chosen; }
    __syncthreads();
    all = factors[0]; chosen = factors[1];
    const uint32_t action = static_cast<uint32_t>(r.action);
    for (uint32_t i = t; i < pieces; i += THREADS * kAhead) {
        Sixteen<T> v[kAhead];
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + THREADS * k < pieces) v[k].load(x + head + (i + THREADS * k) * N);
#pragma unroll
        for (uint32_t k = 0; k < kAhead; ++k)
            if (i + THREADS * k < pieces) {
                const uint32_t at = head + (i + THREADS * k) * N;
                v[k].scale_below(most, all);
                v[k].store(g + at);
                if (action >= at && action - at < N) g[action] = from_float<T>(chosen);
            }
    }
    for (uint32_t k = t; k < head; k += THREADS) g[k] = from_float<T>(k == action ? chosen : all * exp_below<kWhole<T>>(to_float(x[k]), most));
    for (uint32_t k = behind + t; k < a.n; k += THREADS) g[k] = from_float<T>(k == action ? chosen : all * exp_below<kWhole<T>>(to_float(x[k]), most));
}

// The sum over the rows, always of the same parts in the same order: a block's share of them to parts[block], or, of one block, the loss.
__global__ void __launch_bounds__(1024) k_policy_sum(const double* __restrict__ rows, uint64_t n, uint64_t share, double* __restrict__ parts, float* __restrict__ loss)
{
    __shared__ double part[32];
    dep_wait();
    dep_trigger();
    const uint64_t first = blockIdx.x * share, end = min(first + share, n);
    double s[4] = {};
    for (uint64_t i = first + threadIdx.x; i < end; i += 4096u)
#pragma unroll
        for (uint32_t k = 0; k < 4u; ++k)
            if (i + 1024u * k < end) s[k] += rows[i + 1024u * k];
    double sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (uint32_t d = 16u; d > 0u; d /= 2u) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if ((threadIdx.x & 31u) == 0u) part[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x < 32u) {
        sum = part[threadIdx.x];
#pragma unroll
        for (uint32_t d = 16u; d > 0u; d /= 2u) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (threadIdx.x == 0u) {
            if (loss) *loss = static_cast<float>(sum);
            else parts[blockIdx.x] = sum;
        }
    }
}
// One block up to 8,192 rows, else 256 and one for their parts.
constexpr uint64_t kOneBlock = 8192, kSumBlocks = 256;

template <typename T>
int launch_rows(cudaStream_t st, const PolicyArgs& a, bool one)
{
    constexpr uint32_t N = Sixteen<T>::N;
    void (*kernel)(PolicyArgs) = nullptr;
    uint32_t threads = 128, per = 1;
    const bool alike = !a.gradient || ((reinterpret_cast<uintptr_t>(a.logits) - reinterpret_cast<uintptr_t>(a.gradient)) % 16u == 0u &&
                                       (a.rows < 2u || (a.ld - a.ld_gradient) * sizeof(T) % 16u == 0u));
    const uint32_t pieces = a.n / N;
    if (a.n <= 32u) { kernel = one ? k_policy_short<T, 8, 4, 8, true> : k_policy_short<T, 8, 4, 8, false>; per = 128u; }
    else if (a.n <= 64u) { kernel = one ? k_policy_short<T, 16, 4, 8, true> : k_policy_short<T, 16, 4, 8, false>; per = 64u; }
    else if (a.n <= 128u) { kernel = one ? k_policy_short<T, 32, 4, 8, true> : k_policy_short<T, 32, 4, 8, false>; per = 32u; }
    else if (a.n <= 256u) { kernel = one ? k_policy_short<T, 32, 8, 4, true> : k_policy_short<T, 32, 8, 4, false>; per = 16u; }
    else if (!alike) { kernel = k_policy_long<T, false, 512>; threads = 512u; }
    else if (pieces <= 64u) { kernel = k_policy_row<T, 2>; threads = 256u; per = 8u; }
    else if (pieces <= 128u) { kernel = k_policy_row<T, 4>; threads = 256u; per = 8u; }
    else if (pieces <= 256u) { kernel = k_policy_row<T, 8>; threads = 256u; per = 8u; }
    else {
        // 192 bytes a thread, more in rows that a block of 512 has no more threads for; 64 / 128 / 256 / 512 / 1,024 threads, us for half a GB of bf16: rows of 6,000
        // 186 / 205 / 270, 12,000 224 / 182 / 208, 24,000 235 / 227 / 185 / 223, 48,000 - / - / 223 / 191 / 314, 130,000 - / - / 248 / 230 / 233; fp32, 130,000 - / - / - / 251 / 234.
        // Few rows are spread over more threads.
        const uint64_t bytes = static_cast<uint64_t>(a.n) * sizeof(T);
        threads = 64u;
        while (threads < 512u && (bytes > 192u * threads || a.rows * threads < 1024u * kSms)) threads *= 2u;
        if (bytes > (200u << 10)) threads = 1024u;
        kernel = threads == 64u ? k_policy_long<T, true, 64> : threads == 128u ? k_policy_long<T, true, 128> : threads == 256u ? k_policy_long<T, true, 256>
               : threads == 512u ? k_policy_long<T, true, 512> : k_policy_long<T, true, 1024>;
    }
    const uint64_t blocks = (a.rows + per - 1u) / per;
    if (blocks > 0x7FFFFFFFull) return -2;
    if (one) {
        uint32_t cluster = 1;
        while (cluster < blocks) cluster *= 2u;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(cluster); cfg.blockDim = dim3(threads); cfg.stream = st;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr; cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, kernel, a) == cudaSuccess ? 1 : -1;
    }
    return launch_dependent(kernel, dim3(static_cast<uint32_t>(blocks)), dim3(threads), 0, st, a) == cudaSuccess ? 1 : -1;
}

}  // namespace

int launch_policy_loss(cudaStream_t st, uint32_t type, const PolicyArgs& in)
{
    PolicyArgs a = in;
    int n = 0;
    // short rows that one cluster of k_policy_short has
    const bool together = a.loss && a.rows && a.rows <= kMostBlocks * (a.n <= 32u ? 128u : a.n <= 64u ? 64u : a.n <= 128u ? 32u : a.n <= 256u ? 16u : 0u);
    if (together) a.row_loss = nullptr;
    if (a.rows) {
        n = type == EVO_F32 ? launch_rows<float>(st, a, together) : type == EVO_BF16 ? launch_rows<__nv_bfloat16>(st, a, together) : launch_rows<__half>(st, a, together);
        if (n < 0) return n;
    }
    if (!a.loss || together) return n;
    const dim3 one(1), threads(1024);
    if (a.rows <= kOneBlock)
        return launch_dependent(k_policy_sum, one, threads, 0, st, a.row_loss, a.rows, a.rows, static_cast<double*>(nullptr), a.loss) == cudaSuccess ? n + 1 : -1;
    double* const parts = a.row_loss + a.rows;
    const uint64_t share = (a.rows + kSumBlocks - 1u) / kSumBlocks;
    if (launch_dependent(k_policy_sum, dim3(static_cast<uint32_t>(kSumBlocks)), threads, 0, st, a.row_loss, a.rows, share, parts, static_cast<float*>(nullptr)) != cudaSuccess) return -1;
    return launch_dependent(k_policy_sum, one, threads, 0, st, parts, kSumBlocks, kSumBlocks, static_cast<double*>(nullptr), a.loss) == cudaSuccess ? n + 2 : -1;
}

size_t policy_loss_bytes(uint64_t rows) { return static_cast<size_t>((8u * (rows + (rows > kOneBlock ? kSumBlocks : 0u)) + 255u) / 256u * 256u); }

}  // namespace evo

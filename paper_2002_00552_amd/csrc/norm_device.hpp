// What the norm kernels share on the device: sums over lanes, the statistics of a norm, parameters.
#pragma once
#include "elem.hpp"
#include "norm.hpp"
#include "philox.hpp"

namespace dwm {

// K parameters, `step` channels apart from channel c on, and behind the last channel that one.  The kinds part in front of the loads, so
// that these go out together (64 images of 96 channels, 55 x 55, parameters in binary16: 27.9 us with a load after the other, 24.6).
template <class T, int K> __device__ __forceinline__ void strided_params(const void* p, int typed, int c, int step, int C, float none, float (&f)[K])
{
    if (!p) {
#pragma unroll
        for (int k = 0; k < K; ++k) f[k] = none;
    } else if (typed) {
        T t[K];
#pragma unroll
        for (int k = 0; k < K; ++k) t[k] = ((const T*)p)[min(c + k * step, C - 1)];
#pragma unroll
        for (int k = 0; k < K; ++k) f[k] = (float)t[k];
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k) f[k] = ((const float*)p)[min(c + k * step, C - 1)];
    }
}

// V parameters from channel c on, which the caller knows to exist.
template <class T, int V> __device__ __forceinline__ void params(const void* p, int typed, long long c, float none, float (&f)[V])
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = none;
    } else if (typed) {
        unpack<T, V>(load_vector<T, V>((const T*)p + c), f);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            float q[4];
            unpack<float, 4>(load_vector<float, 4>((const float*)p + c + j), q);
#pragma unroll
            for (int i = 0; i < 4; ++i) f[j + i] = q[i];
        }
    }
}

template <int CTRL> __device__ __forceinline__ float dpp(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// The sum over groups of 16 (STEP = 16) or 32 lanes that lie side by side, lane by lane: v[i] + v[i ^ STEP].
template <int STEP> __device__ __forceinline__ float add_across(float v)
{
    const uint32_t u = __float_as_uint(v);
    if (STEP == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

// The sum over N consecutive lanes (2 to 64), for all of them.
template <int N> __device__ __forceinline__ float lanes_sum(float v)
{
    v += dpp<0xB1>(v);               // the neighbour of a pair
    if (N >= 4) v += dpp<0x4E>(v);   // the other pair of four
    if (N >= 8) v += dpp<0x141>(v);  // the other four of eight, mirrored: all four have the same sum
    if (N >= 16) v += dpp<0x140>(v);
    if (N >= 32) v = add_across<16>(v);
    if (N >= 64) v = add_across<32>(v);
    return v;
}

// Sums over the lanes of a wave that are N apart, 2 N apart, ...: for all of them, and the same number for all, which takes eight lanes in front of
// four (four first: two lanes eight apart add the pairs that they are in, two lanes four apart others).
template <int N> __device__ __forceinline__ float strided_sum(float v)
{
    if (N <= 8) v += dpp<0x128>(v);  // eight lanes on, round in sixteen
    if (N <= 4) v += dpp<0x124>(v);  // four
    if (N <= 16) v = add_across<16>(v);
    if (N <= 32) v = add_across<32>(v);
    return v;
}

// A product rounded by itself.  A mean is one: fused into what it is taken from, it would be another number there than where it is not, off by half a
// unit of the mean -- of one value in all of a row of 300, 0.005 in y for a deviation of zero.
__device__ __forceinline__ float rounded_product(float a, float b)
{
#pragma clang fp contract(off)
    return a * b;
}

// The statistics of a norm from a first mean m0, the mean s1 of d = z - m0 and its variance: `off` is what is taken off d for y.
// s1 is the rounding of m0, which counts where the mean is larger than the deviations; where it is smaller, m0 is good
// to a fraction of the deviations' roundoff, and s1 holds the roundings of z - m0 instead, which all have one sign where z has few
// bits (rows of bfloat16 with means of a hundredth: a mean off by 1e-6 of itself).
struct NormStats {
    float off, mean, rstd;
};
__device__ __forceinline__ NormStats norm_stats(float m0, float s1, float var, float eps)
{
    NormStats r;
    r.rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);  // (NaN stays)
    r.off = fabsf(m0) * r.rstd > 1.0f ? s1 : 0.0f;
    r.mean = m0 + r.off;
    return r;
}

// A wave's share of a norm: how many elements it holds, their mean, and the sums of d and of d^2, d = z - mean (the first only by
// the mean's rounding).  Shares are joined without a second reading of the elements: with m0 the mean of all, the sum of z - m0
// over a share is n (mean - m0) + q1, which makes s1, and with u = mean - m0 - s1 the sum of (z - m0 - s1)^2 is q2 + 2 u q1 + n u^2: deviations
// all of it, nothing cancels.
struct NormShare {
    float n, mean, q1, q2;
    __device__ __forceinline__ float first(float m0) const { return n * (mean - m0) + q1; }
    __device__ __forceinline__ float second(float m0, float s1) const
    {
        const float u = mean - m0 - s1;
        return q2 + u * (2.0f * q1 + n * u);
    }
};

}  // namespace dwm

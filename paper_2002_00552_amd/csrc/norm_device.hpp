// What the norm kernels share on the device: sums over lanes, the statistics of a norm, parameters.
#pragma once
#include "elem.hpp"
#include "norm.hpp"
#include "philox.hpp"

namespace dwm {

template <class T> __device__ __forceinline__ float param(const void* p, int typed, long long c, float none)
{
    if (!p) return none;
    return typed ? (float)((const T*)p)[c] : ((const float*)p)[c];
}

// V parameters from channel c on, which the caller knows to exist.
template <class T, int V> __device__ __forceinline__ void params(const void* p, int typed, long long c, float none, float (&f)[V])
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = none;
    } else if (typed) {
        unpack<T>(load16((const T*)p + c), f);
    } else {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            float q[4];
            unpack<float>(load16((const float*)p + c + j), q);
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

// The sum over N consecutive lanes (4 to 64), for all of them.
template <int N> __device__ __forceinline__ float lanes_sum(float v)
{
    v += dpp<0xB1>(v);               // the neighbour of a pair
    v += dpp<0x4E>(v);               // the other pair of four
    if (N >= 8) v += dpp<0x141>(v);  // the other four of eight, mirrored: all four have the same sum
    if (N >= 16) v += dpp<0x140>(v);
    if (N >= 32) v = add_across<16>(v);
    if (N >= 64) v = add_across<32>(v);
    return v;
}

// From the first mean m0 (a sum times 1 / C) and the means s1, s2 of d and d^2, d = z - m0: what is taken off d for y (`off`),
// the mean and rstd.  s1 is the rounding of m0, which counts where the mean is larger than the deviations; where it is smaller,
// m0 is good to a fraction of the deviations' roundoff, and s1 holds the roundings of z - m0 instead, which all have
// one sign where z has few bits (rows of bfloat16 with means of a hundredth: a mean off by 1e-6 of itself).
struct NormStats {
    float off, mean, rstd;
};
__device__ __forceinline__ NormStats norm_stats(float m0, float s1, float s2, float eps)
{
    NormStats r;
    const float var = s2 - s1 * s1;
    r.rstd = 1.0f / sqrtf((var < 0.0f ? 0.0f : var) + eps);  // (NaN stays)
    r.off = fabsf(m0) * r.rstd > 1.0f ? s1 : 0.0f;
    r.mean = m0 + r.off;
    return r;
}

}  // namespace dwm

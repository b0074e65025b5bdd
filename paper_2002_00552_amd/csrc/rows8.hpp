// Rows in 8 bits on the device: blocks of 32 channels, an octet of each of four lanes, e4m3 codes under a power of two.
// Activations and their derivatives too, which act.hip and the products share.
#pragma once
#include "branch.hpp"
#include "elem.hpp"

namespace dwm {

// An octet as it lies in memory.
template <class T> struct Octet {
    typename Vector<T, kVec<T>>::type r[8 / kVec<T>];
};

// n (up to 8) elements from p on, zeros behind them; p is a multiple of its element's size only.
template <class T> __device__ __forceinline__ Octet<T> fetch_octet(const T* p, int n)
{
    Octet<T> o;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < 8 / kVec<T>; ++i) o.r[i] = load_vector<T, kVec<T>>(p + i * kVec<T>);
    } else {
        T t[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] = j < n ? p[j] : (T)0.0f;
        __builtin_memcpy(&o, t, sizeof(o));
    }
    return o;
}
template <class T> __device__ __forceinline__ void octet_values(const Octet<T>& o, float (&f)[8])
{
    constexpr int V = kVec<T>;
#pragma unroll
    for (int i = 0; i < 8 / V; ++i) {
        float q[V];
        unpack<T, V>(o.r[i], q);
#pragma unroll
        for (int j = 0; j < V; ++j) f[i * V + j] = q[j];
    }
}
template <class T> __device__ __forceinline__ void load_octet(const T* p, int n, float (&f)[8]) { octet_values<T>(fetch_octet<T>(p, n), f); }

template <class T> __device__ __forceinline__ void store_octet(T* p, int n, const float (&f)[8])
{
    if (n >= 8) {
        constexpr int V = kVec<T>;
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) {
            float q[V];
#pragma unroll
            for (int j = 0; j < V; ++j) q[j] = f[i * V + j];
            store_vector<T, V>(p + i * V, pack<T, V>(q));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = (T)f[j];
    }
}

// An octet of parameters, binary32 or of the tensors' type.
template <class T> __device__ __forceinline__ void param_octet(const void* p, int typed, long long c, int n, float none, float (&f)[8])
{
    if (!p) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = none;
    } else if (typed) {
        load_octet<T>((const T*)p + c, n, f);
    } else {
        load_octet<float>((const float*)p + c, n, f);
    }
}

// The larger of v over the four lanes that hold a block: side by side (a quad of a row kernel's lanes) ...
struct QuadLanes {
    static __device__ __forceinline__ uint32_t most(uint32_t v)
    {
        v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, true));
        return max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, true));
    }
};
// ... or sixteen apart (a product's accumulators).
struct SixteenApart {
    static __device__ __forceinline__ uint32_t most(uint32_t v)
    {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max((uint32_t)r[0], (uint32_t)r[1]);
        const auto q = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return max((uint32_t)q[0], (uint32_t)q[1]);
    }
};

constexpr uint32_t kInfinity = 0x7f800000u;

// The codes of an octet and its block's scale; all four lanes of the block take part, with zeros behind the last channel.
// As unsigned numbers the patterns of magnitudes are in their order, infinities and NaN last; only a block that has some looks at each
// element.  448 is 1.75 * 2^8: the scale is the magnitude's exponent less 8, and one more where its fraction is over 0.75,
// which the addition carries.  v / 2^(s - 127) is exact but for numbers below the smallest code.
template <class Lanes> __device__ __forceinline__ uint2v pack_octet(const float (&f)[8], uint32_t* scale)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(f[j]) & 0x7fffffffu);
    m = Lanes::most(m);
    if (m >= kInfinity) {  // (all four lanes have the same m)
        m = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t a = __float_as_uint(f[j]) & 0x7fffffffu;
            m = max(m, a < kInfinity ? a : 0u);
        }
        m = Lanes::most(m);
    }
    const int s = max((int)((m + 0x1fffffu) >> 23) - 8, 0);
    *scale = (uint32_t)s;
    const float by = __uint_as_float((uint32_t)(254 - s) << 23);
    uint2v codes;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i] * by, f[4 * i + 1] * by, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * i + 2] * by, f[4 * i + 3] * by, w, true);
        codes[i] = (uint32_t)w;
    }
    return codes;
}

__device__ __forceinline__ void unpack_octet(uint2v codes, uint32_t scale, float (&f)[8])
{
    const float by = __uint_as_float(scale ? scale << 23 : 0x400000u);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes[i], true);
        f[4 * i] = lo[0] * by;
        f[4 * i + 1] = lo[1] * by;
        f[4 * i + 2] = hi[0] * by;
        f[4 * i + 3] = hi[1] * by;
    }
}

// Writes an octet's codes, and by the block's first lane its scale, with the zeros behind the last block of a row.  `octet` counts from
// the row's start; octets behind the last block write nothing.
__device__ __forceinline__ void store_packed(const Packed& p, long long row, int octet, int C, uint2v codes, uint32_t scale)
{
    const int blocks = (C + kBlock - 1) / kBlock, block = octet >> 2, width = (blocks + 3) & ~3;
    if (block >= blocks) return;
    *(uint2v*)(p.codes + row * (blocks * (long long)kBlock) + octet * 8) = codes;
    if (octet & 3) return;
    uint8_t* s = p.scales + row * width + block;
    *s = (uint8_t)scale;
    if (block == blocks - 1)
        for (int i = 1; i < width - block; ++i) s[i] = 0;
}

__device__ __forceinline__ void load_packed(const Packed& p, long long row, int octet, int C, uint2v* codes, uint32_t* scale)
{
    const int blocks = (C + kBlock - 1) / kBlock;
    *codes = *(const uint2v*)(p.codes + row * (blocks * (long long)kBlock) + octet * 8);
    *scale = p.scales[row * ((blocks + 3) & ~3) + (octet >> 2)];
}

// phi(-|x|) exp(x^2 / 2), phi the normal distribution function, as a polynomial in t = 1 / (1 + 0.3 |x|) without a constant term: fitted
// with weights that even out the relative error (Lawson's iteration), 2e-7 of itself (5e-7 as evaluated) up to |x| = 14, where
// the exponential is zero in binary32.
__device__ __forceinline__ float normal_tail(float x)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(0.3f, fabsf(x), 1.0f));
    float q = 0.0356745869f;
    q = fmaf(q, t, -0.157202244f);
    q = fmaf(q, t, 0.206351966f);
    q = fmaf(q, t, -0.0536821596f);
    q = fmaf(q, t, 0.128560811f);
    q = fmaf(q, t, 0.0999137461f);
    q = fmaf(q, t, 0.120753914f);
    q = fmaf(q, t, 0.119629301f);
    return q * t;
}

constexpr float kLog2e = 1.44269504f;

__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * x)); }

__device__ __forceinline__ float act_value(int act, float x)
{
    if (act == DWM_ACT_RELU) return x < 0.0f ? 0.0f : x;  // (NaN stays)
    if (act == DWM_ACT_GELU) {
        const float tail = x * (normal_tail(x) * __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x));
        return x > 0.0f ? x - tail : tail;
    }
    return act == DWM_ACT_SILU ? x * sigmoid(x) : x;
}

__device__ __forceinline__ float act_slope(int act, float x)
{
    if (act == DWM_ACT_RELU) return x > 0.0f ? 1.0f : x != x ? x : 0.0f;
    if (act == DWM_ACT_GELU) {
        const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * x * x), tail = normal_tail(x) * e;
        return fmaf(x * 0.39894228f, e, x > 0.0f ? 1.0f - tail : tail);
    }
    if (act == DWM_ACT_SILU) {
        const float s = sigmoid(x);
        return s * fmaf(x, 1.0f - s, 1.0f);
    }
    return 1.0f;
}

// An octet at a time: the kind of activation parts before the loop.
__device__ __forceinline__ void act_octet(int act, float (&f)[8])
{
    if (act == DWM_ACT_NONE) return;
    if (act == DWM_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = act_value(DWM_ACT_RELU, f[j]);
    } else if (act == DWM_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = act_value(DWM_ACT_GELU, f[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = act_value(DWM_ACT_SILU, f[j]);
    }
}

// g times the derivative at p.
__device__ __forceinline__ void slope_octet(int act, const float (&p)[8], float (&g)[8])
{
    if (act == DWM_ACT_NONE) return;
    if (act == DWM_ACT_RELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] *= act_slope(DWM_ACT_RELU, p[j]);
    } else if (act == DWM_ACT_GELU) {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] *= act_slope(DWM_ACT_GELU, p[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] *= act_slope(DWM_ACT_SILU, p[j]);
    }
}

}  // namespace dwm

// Elements of the three storage types, sixteen or eight bytes at a time, and their way to binary32 and back (one rounding, to nearest even).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace dwm {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// N elements of sixteen or eight bytes at an address that is only a multiple of the element's size: gfx950's global loads and stores take
// those, at the full rate where the address happens to be a multiple of their own.
typedef uint32_t uint2v __attribute__((ext_vector_type(2)));
template <class T, int N> struct Vector;
template <> struct Vector<float, 4> { typedef uint4v type; typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Vector<_Float16, 8> { typedef uint4v type; typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Vector<_Float16, 4> { typedef uint2v type; typedef uint32_t loose __attribute__((ext_vector_type(2), aligned(2))); };
template <> struct Vector<__bf16, 8> { typedef uint4v type; typedef uint32_t loose __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Vector<__bf16, 4> { typedef uint2v type; typedef uint32_t loose __attribute__((ext_vector_type(2), aligned(2))); };

template <class T> constexpr int kVec = 16 / (int)sizeof(T);  // elements of sixteen bytes

template <class T, int N> __device__ __forceinline__ typename Vector<T, N>::type load_vector(const T* p)
{
    return *(const typename Vector<T, N>::loose*)p;
}
template <class T, int N> __device__ __forceinline__ void store_vector(T* p, typename Vector<T, N>::type v)
{
    *(typename Vector<T, N>::loose*)p = v;
}

template <class T, int N> __device__ __forceinline__ void unpack(typename Vector<T, N>::type r, float (&f)[N])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < N; ++j) f[j] = __uint_as_float(r[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            const uint32_t w = r[j];
            if constexpr (__is_same(T, __bf16)) {
                f[2 * j] = __uint_as_float(w << 16);
                f[2 * j + 1] = __uint_as_float(w & 0xffff0000u);
            } else {
                const half2v h = __builtin_bit_cast(half2v, w);
                f[2 * j] = (float)h[0];
                f[2 * j + 1] = (float)h[1];
            }
        }
    }
}

template <class T, int N> __device__ __forceinline__ typename Vector<T, N>::type pack(const float (&f)[N])
{
    typename Vector<T, N>::type r;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = __float_as_uint(f[j]);
    } else {
#pragma unroll
        for (int j = 0; j < N / 2; ++j) {
            if constexpr (__is_same(T, __bf16)) {
                const bf16x2v h = __builtin_convertvector((float2v){f[2 * j], f[2 * j + 1]}, bf16x2v);
                r[j] = __builtin_bit_cast(uint32_t, h);
            } else {
                const half2v h = {(_Float16)f[2 * j], (_Float16)f[2 * j + 1]};
                r[j] = __builtin_bit_cast(uint32_t, h);
            }
        }
    }
    return r;
}

}  // namespace dwm

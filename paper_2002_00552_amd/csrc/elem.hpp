// Elements of the three storage types, sixteen bytes at a time, and their way to binary32 and back (one rounding, to nearest even).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace dwm {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

// Sixteen bytes at an address that is only a multiple of the element's size: gfx950's global loads and stores take those, at the
// full rate where the address happens to be a multiple of sixteen.
template <class T> struct Unaligned;
template <> struct Unaligned<float> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(4))); };
template <> struct Unaligned<_Float16> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Unaligned<__bf16> { typedef uint32_t type __attribute__((ext_vector_type(4), aligned(2))); };

template <class T> constexpr int kVec = 16 / (int)sizeof(T);  // elements of sixteen bytes

template <class T> __device__ __forceinline__ uint4v load16(const T* p) { return *(const typename Unaligned<T>::type*)p; }
template <class T> __device__ __forceinline__ void store16(T* p, uint4v v) { *(typename Unaligned<T>::type*)p = v; }

template <class T> __device__ __forceinline__ void unpack(uint4v r, float (&f)[kVec<T>]);
template <> __device__ __forceinline__ void unpack<float>(uint4v r, float (&f)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(r[j]);
}
template <> __device__ __forceinline__ void unpack<_Float16>(uint4v r, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = r[j];
        const half2v h = __builtin_bit_cast(half2v, w);
        f[2 * j] = (float)h[0];
        f[2 * j + 1] = (float)h[1];
    }
}
template <> __device__ __forceinline__ void unpack<__bf16>(uint4v r, float (&f)[8])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f[2 * j] = __uint_as_float(r[j] << 16);
        f[2 * j + 1] = __uint_as_float(r[j] & 0xffff0000u);
    }
}

template <class T> __device__ __forceinline__ uint4v pack(const float (&f)[kVec<T>]);
template <> __device__ __forceinline__ uint4v pack<float>(const float (&f)[4])
{
    uint4v r;
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __float_as_uint(f[j]);
    return r;
}
template <> __device__ __forceinline__ uint4v pack<_Float16>(const float (&f)[8])
{
    uint4v r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const half2v h = {(_Float16)f[2 * j], (_Float16)f[2 * j + 1]};
        r[j] = __builtin_bit_cast(uint32_t, h);
    }
    return r;
}
template <> __device__ __forceinline__ uint4v pack<__bf16>(const float (&f)[8])
{
    uint4v r;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const bf16x2v h = __builtin_convertvector((float2v){f[2 * j], f[2 * j + 1]}, bf16x2v);
        r[j] = __builtin_bit_cast(uint32_t, h);
    }
    return r;
}

}  // namespace dwm

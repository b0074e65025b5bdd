// Random words from a counter: Philox-4x32 with ten rounds (Salmon, Moraes, Dror, Shaw: "Parallel random numbers: as easy as
// 1, 2, 3", SC 2011).  Element e of a tensor, in its dense order, has word e % 4 of the block of counter (e / 4, sequence) under
// the key seed, so a mask needs no memory: whoever knows (seed, sequence) can draw it again.
// Ten rounds and 32 bits a draw cost nothing here: a copy of 2 GiB of bfloat16 takes 695 us with the draws and 693 without.
#pragma once
#include <hip/hip_runtime.h>

#include "norm.hpp"

namespace dwm {

struct Philox {
    uint32_t w[4];
};

__device__ __forceinline__ Philox philox(uint64_t block, uint64_t sequence, uint32_t k0, uint32_t k1)
{
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)sequence, c3 = (uint32_t)(sequence >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const uint64_t a = (uint64_t)0xD2511F53u * c0, b = (uint64_t)0xCD9E8D57u * c2;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return Philox{{c0, c1, c2, c3}};
}

__device__ __forceinline__ uint64_t drop_sequence(const DropArgs& d)
{
    return d.sequence + (d.mode == kDropDraw && d.sequence_dev ? *d.sequence_dev : 0);
}

// Which of the elements e0 .. e0 + N - 1 are kept: element e0 + j at bit 31 - j.  `aligned` (the same for the whole call): e0 is a multiple of four.
// In one word, so that the draws, which need no data, can be made while data is on its way and kept for later.
template <int N> __device__ __forceinline__ uint32_t drop_bits(const DropArgs& d, uint64_t sequence, uint64_t e0, bool aligned)
{
    if (d.mode != kDropDraw) return d.mode == kDropNone ? ~0u : 0u;
    uint32_t bits = 0;
    if (aligned) {
        constexpr int B = (N + 3) / 4;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const Philox r = philox(e0 / 4 + b, sequence, d.seed_lo, d.seed_hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) bits = bits + bits + (r.w[j] >= d.threshold ? 1u : 0u);
        }
        return bits << (32 - 4 * B);
    }
    constexpr int B = (N + 6) / 4;  // as many blocks as N elements can lie in
#pragma unroll
    for (int b = 0; b < B; ++b) {
        const Philox r = philox(e0 / 4 + b, sequence, d.seed_lo, d.seed_hi);
#pragma unroll
        for (int j = 0; j < 4; ++j) bits = bits + bits + (r.w[j] >= d.threshold ? 1u : 0u);
    }
    return bits << (32 - 4 * B) << ((uint32_t)e0 & 3u);
}

// Element j of the vector that `bits` was drawn for: times the scale, rounded to 32 bits by itself, or zero.
__device__ __forceinline__ float drop_scaled(float v, uint32_t bits, int j, float scale)
{
#pragma clang fp contract(off)
    return __uint_as_float(__float_as_uint(v * scale) & (uint32_t)((int32_t)(bits << j) >> 31));
}

// The same as truth values, for where they are used at once: fewer operations than by way of a word (a copy of 256 MB of bfloat16: 88 us, by the
// word 94).
template <int N> __device__ __forceinline__ void drop_keep(const DropArgs& d, uint64_t sequence, uint64_t e0, bool aligned, bool (&keep)[N])
{
    if (aligned && N % 4 == 0 && d.mode == kDropDraw) {
#pragma unroll
        for (int b = 0; b < N / 4; ++b) {
            const Philox r = philox(e0 / 4 + b, sequence, d.seed_lo, d.seed_hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) keep[4 * b + j] = r.w[j] >= d.threshold;
        }
    } else {
        const uint32_t bits = drop_bits<N>(d, sequence, e0, aligned);
#pragma unroll
        for (int j = 0; j < N; ++j) keep[j] = (int32_t)(bits << j) < 0;
    }
}
__device__ __forceinline__ float drop_scaled(float v, bool keep, float scale)
{
#pragma clang fp contract(off)
    return keep ? v * scale : 0.0f;
}
template <int N> __device__ __forceinline__ void drop_vector(const DropArgs& d, uint64_t sequence, uint64_t e0, bool aligned, float (&f)[N])
{
    bool keep[N];
    drop_keep<N>(d, sequence, e0, aligned, keep);
#pragma unroll
    for (int j = 0; j < N; ++j) f[j] = drop_scaled(f[j], keep[j], d.scale);
}

// z = residual + a dropped and scaled branch is a sum of two binary32 numbers.
__device__ __forceinline__ float join_sum(float residual, float branch)
{
#pragma clang fp contract(off)
    return residual + branch;
}

}  // namespace dwm

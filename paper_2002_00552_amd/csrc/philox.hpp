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

// keep[j]: whether element e0 + j is kept.  ALIGNED: e0 is a multiple of four.
template <int N, bool ALIGNED>
__device__ __forceinline__ void drop_draw(const DropArgs& d, uint64_t sequence, uint64_t e0, bool (&keep)[N])
{
    if (ALIGNED) {
#pragma unroll
        for (int b = 0; b < N / 4; ++b) {
            const Philox r = philox(e0 / 4 + b, sequence, d.seed_lo, d.seed_hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) keep[4 * b + j] = r.w[j] >= d.threshold;
        }
    } else {  // as many blocks as N elements can lie in, and from their bits those of the elements
        constexpr int B = (N + 6) / 4;
        uint32_t bits = 0;
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const Philox r = philox(e0 / 4 + b, sequence, d.seed_lo, d.seed_hi);
#pragma unroll
            for (int j = 0; j < 4; ++j) bits |= (r.w[j] >= d.threshold ? 1u : 0u) << (4 * b + j);
        }
        bits >>= (uint32_t)e0 & 3u;
#pragma unroll
        for (int j = 0; j < N; ++j) keep[j] = (bits >> j) & 1u;
    }
}

// A kept element times the scale, rounded to 32 bits by itself: z = residual + this is a sum of two binary32 numbers.
__device__ __forceinline__ float drop_scaled(float v, bool keep, float scale)
{
#pragma clang fp contract(off)
    return keep ? v * scale : 0.0f;
}
__device__ __forceinline__ float join_sum(float residual, float branch)
{
#pragma clang fp contract(off)
    return residual + branch;
}

}  // namespace dwm

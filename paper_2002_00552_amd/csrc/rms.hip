// Root-mean-square norms of rows with the addition of a residual (gfx950).  Memory bounds them: a row is read once and held in registers, an
// octet of neighbouring channels to a thread (and one more, a row's threads further on, in the widest rows), so that four lanes hold a block of
// 32 channels and its scale comes out of two exchanges between neighbours.  A row's threads are a part of a wave, a wave or a
// workgroup; the kernels for any size read a row twice.  Operands out of the caches, 16384 rows of 4096 bfloat16: z and y from x and residual 99 us (5.4 TB/s), the
// gradient from z's checkpoint with dz and dgamma 85 us (5.5 TB/s) and 5 for the last sums; a copy of 1 GiB runs at 5.1 TB/s on the same card.
#include "norm_device.hpp"
#include "rows8.hpp"

namespace dwm {

constexpr int rms_threads(int tpr) { return tpr > 256 ? tpr : 256; }

// The sum over N consecutive lanes in 64 bits, for all of them.
template <int CTRL> __device__ __forceinline__ double dpp64(double v)
{
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, true);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}
template <int N> __device__ __forceinline__ double lanes_sum(double v)
{
    v += dpp64<0xB1>(v);
    if (N >= 4) v += dpp64<0x4E>(v);
    if (N >= 8) v += dpp64<0x141>(v);
    if (N >= 16) v += dpp64<0x140>(v);
#pragma unroll
    for (int step = 16; step < 64; step *= 2)
        if (N > step) {
            const uint64_t u = __builtin_bit_cast(uint64_t, v);
            const uint32_t lo = (uint32_t)u, hi = (uint32_t)(u >> 32);
            const auto a = step == 16 ? __builtin_amdgcn_permlane16_swap(lo, lo, false, false) : __builtin_amdgcn_permlane32_swap(lo, lo, false, false);
            const auto b = step == 16 ? __builtin_amdgcn_permlane16_swap(hi, hi, false, false) : __builtin_amdgcn_permlane32_swap(hi, hi, false, false);
            v = __builtin_bit_cast(double, (uint64_t)b[0] << 32 | a[0]) + __builtin_bit_cast(double, (uint64_t)b[1] << 32 | a[1]);
        }
    return v;
}

// The sum over a row's threads, for all of them; `slots` has two times sixteen places, used in turn.
template <int TPR, class F> __device__ __forceinline__ F row_sum(F v, F* slots, int turn)
{
    v = lanes_sum<(TPR < 64 ? TPR : 64)>(v);
    if constexpr (TPR > 64) {
        constexpr int W = TPR / 64;
        const int wave = threadIdx.x / 64, first = wave / W * W;
        F* s = slots + 16 * (turn & 1);
        s[wave] = v;
        __syncthreads();
        v = 0;
#pragma unroll
        for (int i = 0; i < W; ++i) v += s[first + i];
    }
    return v;
}

// z of an octet as it is stored: the sum rounded to binary32, then to T; zeros behind the last channel.
template <class T> __device__ __forceinline__ void joined(float (&z)[8], const float (&r)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = (float)(T)(z[j] + r[j]);
}

// rstd from the sum of squares: the hardware's reciprocal root of 64 bits (good to some 26 bits) and a step of Newton's; as two numbers of 32 bits.
// The squares are summed in 64 bits too, so that y is off by its own rounding and hardly more: what is rounded to 8 bits goes to the other side of a
// border where a sum in 32 bits has it wrong (a value in some 10^7; memory has time for it).
struct Rstd {
    float hi, lo;
};
__device__ __forceinline__ Rstd rms_rstd(double sum, const RmsArgs& a)
{
    const double m = fma(sum, a.inverse, a.eps);
    double r = __builtin_amdgcn_rsq(m);
    const double better = r * (1.5 - 0.5 * m * r * r);
    r = better > 0.0 && m > 0.0 ? better : r;  // (zero, infinity and NaN as they are)
    const float hi = (float)r;
    return {hi, hi < 3e38f ? (float)(r - (double)hi) : 0.0f};
}

// Whether a number may lie right between two codes, or be the largest that a scale holds: some do once they are rounded to binary32, and then the side that the
// exact value is on decides, not the tie.  Borders have at most four bits behind the first (between two codes of three: four; 448: two; odd multiples of 2^-10, between the
// codes below the smallest binade, three), so the lowest 19 of one value in 2^19 are zeros; numbers of so few bits that are no borders are as near to their code a step of binary32 further.
__device__ __forceinline__ uint32_t off_border(float y) { return __float_as_uint(y) & 0x7ffffu; }

// What a row's octet leaves behind: z, y and both in 8 bits.
template <class T>
__device__ __forceinline__ void rms_write(const RmsArgs& a, long long row, int octet, const float (&z)[8], const float (&gamma)[8], Rstd rstd)
{
    const int c = octet * 8, n = a.C - c;
    if (a.z && n > 0) store_octet<T>((T*)a.z + row * a.stride[kRmsZ] + c, n, z);
    if (a.kept.codes) {
        uint32_t s;
        const uint2v codes = pack_octet<QuadLanes>(z, &s);
        store_packed(a.kept, row, octet, a.C, codes, s);
    }
    if (!a.y && !a.packed_y.codes) return;
    float y[8], t[8], rest[8];  // y = t * gamma + rest with t = z * hi, what that rounding lost and lo in rest: one rounding; z * rstd first, which is at most sqrt(C), where z * gamma might leave binary32
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        t[j] = z[j] * rstd.hi;
        rest[j] = fmaf(z[j], rstd.lo, fmaf(z[j], rstd.hi, -t[j])) * gamma[j];
        y[j] = fmaf(t[j], gamma[j], rest[j]);
    }
    if (a.y && n > 0) store_octet<T>((T*)a.y + row * a.stride[kRmsY] + c, n, y);
    if (a.packed_y.codes) {
        if (n < 8)
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = j < n ? y[j] : 0.0f;  // (an infinite rstd makes NaN of zeros)
        uint32_t least = ~0u;  // (one question for the octet)
#pragma unroll
        for (int j = 0; j < 8; ++j) least = min(least, off_border(y[j]));
        if (least == 0)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float off = fmaf(t[j], gamma[j], -y[j]) + rest[j];
                const bool number = (__float_as_uint(y[j]) & 0x7fffffffu) - 1u < kInfinity - 1u;  // (no zero, infinity or NaN)
                if (j < n && number && off_border(y[j]) == 0 && off != 0.0f) y[j] = __uint_as_float(__float_as_uint(y[j]) + ((off > 0.0f) == (y[j] > 0.0f) ? 1 : -1));
            }
        uint32_t s;
        const uint2v codes = pack_octet<QuadLanes>(y, &s);
        store_packed(a.packed_y, row, octet, a.C, codes, s);
    }
}

template <class T, int TPR, int K> __global__ __launch_bounds__(rms_threads(TPR)) void rms_forward_kernel(RmsArgs a)
{
    constexpr int R = rms_threads(TPR) / TPR;
    __shared__ double slots[32];
    const int lane = threadIdx.x % TPR;
    float gamma[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (lane + k * TPR) * 8;
        param_octet<T>(a.gamma, a.param_typed, c, a.C - c, 1.0f, gamma[k]);
    }
    // With one octet a thread and several rows to a workgroup, a row ahead of the one that is worked on.
    struct Row {
        Octet<T> x[K], r[K];
    } ahead;
    const long long group = threadIdx.x / TPR, step = (long long)gridDim.x * R;
    const auto fetch = [&](long long row) {
        const bool here = row < a.rows;
        if (!here) row = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + k * TPR) * 8, n = here ? a.C - c : 0;
            ahead.x[k] = fetch_octet<T>((const T*)a.x + row * a.stride[kRmsX] + c, n);
            if (a.residual) ahead.r[k] = fetch_octet<T>((const T*)a.residual + row * a.stride[kRmsResidual] + c, n);
        }
    };
    int turn = 0;
    if (K == 1) fetch((long long)blockIdx.x * R + group);
    for (long long first = (long long)blockIdx.x * R; first < a.rows; first += step, ++turn) {
        const long long row = first + group;
        const bool here = row < a.rows;
        if (K > 1) fetch(row);
        float z[K][8], r[K][8];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            octet_values<T>(ahead.x[k], z[k]);
            if (a.residual) octet_values<T>(ahead.r[k], r[k]);
        }
        if (K == 1 && first + step < a.rows) fetch(row + step);
        if (a.residual)
#pragma unroll
            for (int k = 0; k < K; ++k) joined<T>(z[k], r[k]);
        double sum = 0.0;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fma((double)z[k][j], (double)z[k][j], sum);
        const Rstd rstd = rms_rstd(row_sum<TPR>(sum, slots, turn), a);
        if (!here) continue;  // (a whole group of lanes; no barrier of this row is left)
        if (a.rstd && lane == 0) a.rstd[row] = rstd.hi;
#pragma unroll
        for (int k = 0; k < K; ++k) rms_write<T>(a, row, lane + k * TPR, z[k], gamma[k], rstd);
    }
}

// Any number of channels: a workgroup for a row, read twice.
template <class T> __global__ __launch_bounds__(1024) void rms_forward_any_kernel(RmsArgs a)
{
    __shared__ double slots[32];
    const int octets = (int)((a.C + kBlock - 1) / kBlock) * 4;
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
        double sum = 0.0;
        for (int pass = 0; pass < 2; ++pass) {
            Rstd rstd = {0.0f, 0.0f};
            if (pass) {
                rstd = rms_rstd(row_sum<1024>(sum, slots, turn), a);
                if (a.rstd && threadIdx.x == 0) a.rstd[row] = rstd.hi;
            }
            for (int octet = threadIdx.x; octet < octets; octet += 1024) {
                const int c = octet * 8, n = a.C - c;
                float z[8], r[8], gamma[8];
                load_octet<T>((const T*)a.x + row * a.stride[kRmsX] + c, n, z);
                if (a.residual) {
                    load_octet<T>((const T*)a.residual + row * a.stride[kRmsResidual] + c, n, r);
                    joined<T>(z, r);
                }
                if (pass) {
                    param_octet<T>(a.gamma, a.param_typed, c, n, 1.0f, gamma);
                    rms_write<T>(a, row, octet, z, gamma, rstd);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fma((double)z[j], (double)z[j], sum);
                }
            }
        }
    }
}

// An octet of z for the gradient, on its way and then as numbers: as it was stored, or what its checkpoint stands for.
template <class T> struct KeptOctet {
    Octet<T> z;
    uint2v codes;
    uint32_t scale;
};
template <class T> __device__ __forceinline__ KeptOctet<T> fetch_kept(const RmsArgs& a, long long row, int octet, int n)
{
    KeptOctet<T> o = {};
    if (!a.kept.codes)
        o.z = fetch_octet<T>((const T*)a.z + row * a.stride[kRmsZ] + octet * 8, n);
    else if (n > 0)
        load_packed(a.kept, row, octet, a.C, &o.codes, &o.scale);
    return o;
}
template <class T> __device__ __forceinline__ void kept_values(const RmsArgs& a, const KeptOctet<T>& o, int n, float (&z)[8])
{
    if (!a.kept.codes) return octet_values<T>(o.z, z);
    unpack_octet(o.codes, o.scale, z);
    if (n < 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = j < n ? z[j] : 0.0f;
}
template <class T> __device__ __forceinline__ void kept_octet(const RmsArgs& a, long long row, int octet, int n, float (&z)[8])
{
    kept_values<T>(a, fetch_kept<T>(a, row, octet, n), n, z);
}

template <class T> __device__ __forceinline__ Octet<T> fetch_dz(const RmsArgs& a, long long row, int c, int n)
{
    Octet<T> o = {};
    if (a.dz) o = fetch_octet<T>((const T*)a.dz + row * a.stride[kRmsDz] + c, n);
    return o;
}

template <class T>
__device__ __forceinline__ void rms_gradient(const RmsArgs& a, long long row, int c, int n, const float (&dy)[8], const float (&z)[8], const float (&gamma)[8],
                                             float rstd, float along, const Octet<T>& more)
{
    if (n <= 0) return;
    float dz[8] = {0, 0, 0, 0, 0, 0, 0, 0}, dx[8];
    if (a.dz) octet_values<T>(more, dz);
#pragma unroll
    for (int j = 0; j < 8; ++j) dx[j] = dz[j] + rstd * (dy[j] * gamma[j] - z[j] * rstd * along);
    store_octet<T>((T*)a.dx + row * a.stride[kRmsDx] + c, n, dx);
}

// The gradient, and a workgroup's sums of dy * xhat over its rows for dgamma: in registers, over its groups of lanes through LDS.
template <class T, int TPR, int K> __global__ __launch_bounds__(rms_threads(TPR)) void rms_backward_kernel(RmsArgs a)
{
    constexpr int R = rms_threads(TPR) / TPR;
    __shared__ float slots[32];
    __shared__ float sums[R > 1 ? R * TPR * K * 8 : 1];
    const int lane = threadIdx.x % TPR;
    float gamma[K][8], acc[K][8];
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int c = (lane + k * TPR) * 8;
        param_octet<T>(a.gamma, a.param_typed, c, a.C - c, 1.0f, gamma[k]);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[k][j] = 0.0f;
    }
    // With one octet a thread, a row ahead of the one that is worked on (two do not fit the registers; 16384 rows of 4096 bfloat16 from their checkpoints, out of the caches: 105 us without, 85 with).
    struct Row {
        Octet<T> dy[K], dz[K];
        KeptOctet<T> z[K];
        float rstd;
    } ahead, now;
    const long long group = threadIdx.x / TPR, step = (long long)gridDim.x * R;
    const auto fetch = [&](long long row) {
        const bool here = row < a.rows;
        if (!here) row = 0;
        ahead.rstd = here ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int octet = lane + k * TPR, n = here ? a.C - octet * 8 : 0;
            ahead.dy[k] = fetch_octet<T>((const T*)a.dy + row * a.stride[kRmsDy] + octet * 8, n);
            ahead.z[k] = fetch_kept<T>(a, row, octet, n);
            ahead.dz[k] = fetch_dz<T>(a, row, octet * 8, n);
        }
    };
    int turn = 0;
    if (K == 1) fetch((long long)blockIdx.x * R + group);
    for (long long first = (long long)blockIdx.x * R; first < a.rows; first += step, ++turn) {
        const long long row = first + group;
        const bool here = row < a.rows;
        if (K > 1) fetch(row);
        now = ahead;
        if (K == 1 && first + step < a.rows) fetch(row + step);
        float dy[K][8], z[K][8];
        const float rstd = now.rstd;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            octet_values<T>(now.dy[k], dy[k]);
            kept_values<T>(a, now.z[k], here ? a.C - (lane + k * TPR) * 8 : 0, z[k]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float xhat = z[k][j] * rstd;
                if (here) acc[k][j] = fmaf(dy[k][j], xhat, acc[k][j]);
                sum = fmaf(dy[k][j] * gamma[k][j], xhat, sum);
            }
        }
        if (!a.dx) continue;
        const float along = row_sum<TPR>(sum, slots, turn) / (float)a.C;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + k * TPR) * 8;
            rms_gradient<T>(a, row, c, here ? a.C - c : 0, dy[k], z[k], gamma[k], rstd, along, now.dz[k]);
        }
    }
    if (!a.partial) return;
    float* to = a.partial + (long long)blockIdx.x * a.C;
    if constexpr (R == 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int c = (lane + k * TPR) * 8;
            if (c < a.C) store_octet<float>(to + c, a.C - c, acc[k]);
        }
    } else {
        constexpr int W = TPR * K * 8;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < 8; ++j) sums[group * W + (lane + k * TPR) * 8 + j] = acc[k][j];
        __syncthreads();
        for (int c = threadIdx.x; c < W && c < a.C; c += rms_threads(TPR)) {
            float s = 0.0f;
#pragma unroll
            for (int g = 0; g < R; ++g) s += sums[g * W + c];
            to[c] = s;
        }
    }
}

// Any number of channels, dx: a workgroup for a row, read twice.  dgamma has a kernel of its own, before dx may overwrite dy.
template <class T> __global__ __launch_bounds__(1024) void rms_backward_any_kernel(RmsArgs a)
{
    __shared__ float slots[32];
    const int octets = (a.C + 7) / 8;
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, ++turn) {
        const float rstd = a.rstd[row];
        float sum = 0.0f, along = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {
            if (pass) along = row_sum<1024>(sum, slots, turn) / (float)a.C;
            for (int octet = threadIdx.x; octet < octets; octet += 1024) {
                const int c = octet * 8, n = a.C - c;
                float dy[8], z[8], gamma[8];
                load_octet<T>((const T*)a.dy + row * a.stride[kRmsDy] + c, n, dy);
                kept_octet<T>(a, row, octet, n, z);
                param_octet<T>(a.gamma, a.param_typed, c, n, 1.0f, gamma);
                if (pass) {
                    rms_gradient<T>(a, row, c, n, dy, z, gamma, rstd, along, fetch_dz<T>(a, row, c, n));
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fmaf(dy[j] * gamma[j], z[j] * rstd, sum);
                }
            }
        }
    }
}

// A part of the rows for 2048 channels.
template <class T> __global__ __launch_bounds__(256) void rms_gamma_any_kernel(RmsArgs a)
{
    const int octet = blockIdx.x * 256 + threadIdx.x, c = octet * 8, n = a.C - c;
    if (n <= 0) return;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const float rstd = a.rstd[row];
        float dy[8], z[8];
        load_octet<T>((const T*)a.dy + row * a.stride[kRmsDy] + c, n, dy);
        kept_octet<T>(a, row, octet, n, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = fmaf(dy[j], z[j] * rstd, acc[j]);
    }
    store_octet<float>(a.partial + (long long)blockIdx.y * a.C + c, n, acc);
}

constexpr long long kRmsBlocks = 1 << 20;  // of a launch forward, at most

// Forward, a workgroup for each row (or each few short ones), or, from four times the 256 * 1024 threads on that backward kernels have too, so many that go
// on to further rows, one ahead.  us, operands out of the caches, one workgroup a row and staying: 4096 rows of 4096 bfloat16, z and y, 32.9, 28.1; 16384 rows 114, 99; 5000 of
// 8192 71, 62; 32768 of 1024 binary32 96, 102 (twice the bytes under way as it is: not there).
template <class T, int TPR, int K> static dwm_status_t forward_shape(const RmsArgs& a, hipStream_t s)
{
    constexpr int R = rms_threads(TPR) / TPR, kStaying = 256 * 1024 / rms_threads(TPR);
    const long long blocks = (a.rows + R - 1) / R, most = K == 1 && sizeof(T) == 2 && blocks >= 4 * kStaying ? kStaying : kRmsBlocks;
    hipLaunchKernelGGL((rms_forward_kernel<T, TPR, K>), dim3((unsigned)(blocks < most ? blocks : most)), dim3(rms_threads(TPR)), 0, s, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}
template <class T, int TPR, int K> static dwm_status_t backward_shape(const RmsArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL((rms_backward_kernel<T, TPR, K>), dim3(a.splits), dim3(rms_threads(TPR)), 0, s, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

template <class T, int I> static dwm_status_t shaped(const RmsArgs& a, int kernel, bool backward, hipStream_t s)
{
    if constexpr (I < kRmsShapeCount) {
        constexpr RmsShape sh = kRmsShapes[I];
        if (kernel != I + 1) return shaped<T, I + 1>(a, kernel, backward, s);
        return backward ? backward_shape<T, sh.tpr, sh.k>(a, s) : forward_shape<T, sh.tpr, sh.k>(a, s);
    }
    return DWM_ERR_INVALID_ARG;
}

template <class T> static dwm_status_t forward(const RmsArgs& a, int kernel, hipStream_t s)
{
    if (kernel > 0) return shaped<T, 0>(a, kernel, false, s);
    hipLaunchKernelGGL(rms_forward_any_kernel<T>, dim3((unsigned)(a.rows < kRmsBlocks ? a.rows : kRmsBlocks)), dim3(1024), 0, s, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

template <class T> static dwm_status_t backward(const RmsArgs& a, int kernel, hipStream_t s)
{
    if (kernel > 0) return shaped<T, 0>(a, kernel, true, s);
    if (a.partial) {
        hipLaunchKernelGGL(rms_gamma_any_kernel<T>, dim3((a.C + 2047) / 2048, a.splits), dim3(256), 0, s, a);
        if (hipGetLastError() != hipSuccess) return DWM_ERR_HIP;
    }
    if (!a.dx) return DWM_OK;
    hipLaunchKernelGGL(rms_backward_any_kernel<T>, dim3((unsigned)(a.rows < kRmsBlocks ? a.rows : kRmsBlocks)), dim3(1024), 0, s, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

dwm_status_t launch_rms_forward(const RmsArgs& a, dwm_type_t type, int kernel, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    switch (type) {
        case DWM_F32: return forward<float>(a, kernel, s);
        case DWM_F16: return forward<_Float16>(a, kernel, s);
        case DWM_BF16: return forward<__bf16>(a, kernel, s);
        default: return DWM_ERR_INVALID_ARG;
    }
}

dwm_status_t launch_rms_backward(const RmsArgs& a, dwm_type_t type, int kernel, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    switch (type) {
        case DWM_F32: return backward<float>(a, kernel, s);
        case DWM_F16: return backward<_Float16>(a, kernel, s);
        case DWM_BF16: return backward<__bf16>(a, kernel, s);
        default: return DWM_ERR_INVALID_ARG;
    }
}

}  // namespace dwm

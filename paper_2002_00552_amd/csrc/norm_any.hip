// Layer norm over the channels of [outer][C][inner] and its gradients, with or without the join of a residual branch, for any
// sizes (gfx950).  A position (o, i) is a norm of its own:
//     m = (1/C) sum_c z,  v = (1/C) sum_c (z - m)^2,  r = 1 / sqrt(v + eps),  y = (z - m) r gamma_c + beta_c
//     g = dy gamma,  dz = r (g - (1/C) sum_c g - xhat (1/C) sum_c g xhat),  dgamma_c = sum_{o,i} dy xhat,  dbeta_c = sum_{o,i} dy
// with xhat = (z - m) r and, in a join, z = residual + dropout(x) rounded to its type.
//
// Nothing is held from one pass over the channels to the next, so a norm is read three times and its gradient twice; the kernels
// that keep a norm in registers (norm_impl.inc) take every size that they can.  Sums are in binary32.  The second pass takes the
// sums of d and of d^2, d = z - m; the first of them tells how far m was off (norm_device.hpp).
// A workgroup owns L positions next to each other, 256 / L threads each: lanes lie along what is contiguous, the channels of a
// row (L = 1) or the pixels of a map (L = 64 or 8).  A thread meets the same elements in every pass, so z may be the residual's own
// memory, and what a pass wrote is there for the next.
#include "norm_device.hpp"

namespace dwm {

// Calls f for the channels g, g + G, ... below n: for four of them at once, whose loads go out together, and for the last ones one by one.
// One by one and four at once, us, forward and backward: 500 rows of 32768 bfloat16 117 and 134, 46 and 86; 2 images of 2500 channels, 28 x 28, binary32 97
// and 84, 47 and 67.  (Four under conditions instead of one by one at the end: of bfloat16 117 and 151, since a half word loaded under a condition
// waits for the one whose register it shares.)
template <int N> struct Count { static constexpr int n = N; };
template <int G, class F> __device__ __forceinline__ void channels(int g, int n, const F& f)
{
    int c = g;
    for (; c < n - 3 * G; c += 4 * G) f(c, Count<4>());
    for (; c < n; c += G) f(c, Count<1>());
}

// The sum over the 256 / L threads of a position, for all of them.
template <int L>
__device__ __forceinline__ float position_sum(float v, float* lds)
{
    const int tid = threadIdx.x;
    __syncthreads();  // what was read last
    lds[tid] = v;
    __syncthreads();
#pragma unroll
    for (int h = 128; h >= L; h /= 2) {
        if (tid < h) lds[tid] += lds[tid + h];
        __syncthreads();
    }
    return lds[tid % L];
}

template <class T, int L, bool JOIN>
__global__ __launch_bounds__(256) void norm_any_forward_kernel(NormArgs a)
{
    __shared__ float lds[256];
    const int p = threadIdx.x % L, g = threadIdx.x / L;
    constexpr int G = 256 / L;
    const long long positions = a.outer * a.inner;
    const uint64_t sequence = drop_sequence(a.drop);
    const float inv_c = 1.0f / (float)a.C;
    const T *x = (const T*)a.x, *residual = (const T*)a.residual;
    T *z = (T*)a.z, *y = (T*)a.y;
    for (long long t0 = (long long)blockIdx.x * L; t0 < positions; t0 += (long long)gridDim.x * L) {
        const long long t = t0 + p;
        const int n = t < positions ? a.C : 0;  // every thread meets the barriers
        const long long o = t / a.inner, i = t % a.inner;
        const T* xp = x + o * a.stride[kNormX] + i;
        const T* rp = residual + o * a.stride[kNormResidual] + i;
        T* zp = z + o * a.stride[kNormZ] + i;
        float sum = 0.0f;
        channels<G>(g, n, [&](int c0, auto count) {
            constexpr int N = decltype(count)::n;
            T xs[N], rs[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                xs[k] = xp[(c0 + k * G) * a.inner];
                if (JOIN) rs[k] = rp[(c0 + k * G) * a.inner];
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int c = c0 + k * G;
                float v = (float)xs[k];
                if (JOIN) {
                    const uint32_t bits = drop_bits<1>(a.drop, sequence, (uint64_t)((o * a.C + c) * a.inner + i), false);
                    const T r = (T)join_sum((float)rs[k], drop_scaled(v, bits, 0, a.drop.scale));
                    zp[c * a.inner] = r;
                    v = (float)r;
                }
                sum += v;
            }
        });
        const T* vp = JOIN ? zp : xp;
        const float m0 = rounded_product(position_sum<L>(sum, lds), inv_c);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll 4
        for (int c = g; c < n; c += G) {
            const float d = (float)vp[c * a.inner] - m0;
            s1 += d;
            s2 += d * d;
        }
        s1 = position_sum<L>(s1, lds) * inv_c;
        s2 = position_sum<L>(s2, lds) * inv_c;
        const NormStats st = norm_stats(m0, s1, s2 - s1 * s1, a.eps);
        T* yp = y + o * a.stride[kNormY] + i;
        channels<G>(g, n, [&](int c0, auto count) {
            constexpr int N = decltype(count)::n;
            T zs[N];
            float gamma[N], beta[N];
#pragma unroll
            for (int k = 0; k < N; ++k) zs[k] = vp[(c0 + k * G) * a.inner];
            strided_params<T>(a.gamma, a.param_typed, c0, G, a.C, 1.0f, gamma);
            strided_params<T>(a.beta, a.param_typed, c0, G, a.C, 0.0f, beta);
#pragma unroll
            for (int k = 0; k < N; ++k) yp[(c0 + k * G) * a.inner] = (T)(((float)zs[k] - m0 - st.off) * st.rstd * gamma[k] + beta[k]);
        });
        if (g == 0 && n) {
            if (a.mean) a.mean[t] = st.mean;
            if (a.rstd) a.rstd[t] = st.rstd;
        }
    }
}

template <class T, int L>
__global__ __launch_bounds__(256) void norm_any_backward_kernel(NormArgs a)
{
    __shared__ float lds[256];
    const int p = threadIdx.x % L, g = threadIdx.x / L;
    constexpr int G = 256 / L;
    const long long positions = a.outer * a.inner;
    const uint64_t sequence = drop_sequence(a.drop);
    const float inv_c = 1.0f / (float)a.C;
    for (long long t0 = (long long)blockIdx.x * L; t0 < positions; t0 += (long long)gridDim.x * L) {
        const long long t = t0 + p;
        const int n = t < positions ? a.C : 0;
        const long long o = t / a.inner, i = t % a.inner;
        const float mean = n ? a.mean[t] : 0.0f, rstd = n ? a.rstd[t] : 0.0f;
        const T* dyp = (const T*)a.dy + o * a.stride[kNormDy] + i;
        const T* zp = (const T*)a.z + o * a.stride[kNormZ] + i;
        float s1 = 0.0f, s2 = 0.0f;
        channels<G>(g, n, [&](int c0, auto count) {
            constexpr int N = decltype(count)::n;
            T dys[N], zs[N];
            float gamma[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                dys[k] = dyp[(c0 + k * G) * a.inner];
                zs[k] = zp[(c0 + k * G) * a.inner];
            }
            strided_params<T>(a.gamma, a.param_typed, c0, G, a.C, 1.0f, gamma);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float gr = (float)dys[k] * gamma[k];
                s1 += gr;
                s2 += gr * (((float)zs[k] - mean) * rstd);
            }
        });
        s1 = position_sum<L>(s1, lds) * inv_c;
        s2 = position_sum<L>(s2, lds) * inv_c;
        channels<G>(g, n, [&](int c0, auto count) {
            constexpr int N = decltype(count)::n;
            T dys[N], zs[N], dzs[N];
            float gamma[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const long long at = (c0 + k * G) * a.inner;
                dys[k] = dyp[at];
                zs[k] = zp[at];
                if (a.dz) dzs[k] = ((const T*)a.dz)[o * a.stride[kNormDz] + i + at];
            }
            strided_params<T>(a.gamma, a.param_typed, c0, G, a.C, 1.0f, gamma);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int c = c0 + k * G;
                const long long at = c * a.inner;
                const float gr = (float)dys[k] * gamma[k];
                const float xhat = ((float)zs[k] - mean) * rstd;
                float d = rstd * (gr - s1 - xhat * s2);
                if (a.dz) d += (float)dzs[k];
                if (a.dresidual) ((T*)a.dresidual)[o * a.stride[kNormDresidual] + i + at] = (T)d;
                if (a.dx) {
                    const uint32_t bits = drop_bits<1>(a.drop, sequence, (uint64_t)((o * a.C + c) * a.inner + i), false);
                    ((T*)a.dx)[o * a.stride[kNormDx] + i + at] = (T)drop_scaled(d, bits, 0, a.drop.scale);
                }
            }
        });
    }
}

// The parameters' gradients over one split of the positions: L channels of a workgroup, 256 / L threads each.
template <class T, int L>
__global__ __launch_bounds__(256) void norm_any_params_kernel(NormArgs a)
{
    __shared__ float lds[256];
    const int c = blockIdx.x * L + threadIdx.x % L;
    const long long positions = a.outer * a.inner;
    float dgamma = 0.0f, dbeta = 0.0f;
    if (c < a.C)
        for (long long t = (long long)blockIdx.y * (256 / L) + threadIdx.x / L; t < positions; t += (long long)gridDim.y * (256 / L)) {
            const long long o = t / a.inner, i = t % a.inner;
            const float dy = (float)((const T*)a.dy)[o * a.stride[kNormDy] + c * a.inner + i];
            const float z = (float)((const T*)a.z)[o * a.stride[kNormZ] + c * a.inner + i];
            dgamma += dy * ((z - a.mean[t]) * a.rstd[t]);
            dbeta += dy;
        }
    dgamma = position_sum<L>(dgamma, lds);
    dbeta = position_sum<L>(dbeta, lds);
    if (threadIdx.x < L && c < a.C) {
        a.partial[(long long)blockIdx.y * 2 * a.C + c] = dgamma;
        a.partial[((long long)blockIdx.y * 2 + 1) * a.C + c] = dbeta;
    }
}

// The splits' sums added up, in an order that does not vary: 32 channels of a workgroup, 32 threads each.
template <class T>
__global__ __launch_bounds__(1024) void norm_params_final_kernel(NormArgs a)
{
    __shared__ float lds[32][33];
    const int lane = threadIdx.x % 32, group = threadIdx.x / 32, which = blockIdx.y;
    const int c = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    if (c < a.C)
#pragma unroll 8
        for (int s = group; s < a.splits; s += 32) sum += a.partial[((long long)s * 2 + which) * a.C + c];
    lds[group][lane] = sum;
    __syncthreads();
    sum = lanes_sum<32>(lds[lane][group]);  // a channel's 32 threads side by side
    const int mine = blockIdx.x * 32 + group;
    void* out = which ? a.dbeta : a.dgamma;
    if (lane == 0 && mine < a.C && out) {
        if (a.param_typed) ((T*)out)[mine] = (T)sum;
        else ((float*)out)[mine] = sum;
    }
}

template <class T>
static dwm_status_t params_final(const NormArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((norm_params_final_kernel<T>), dim3((a.C + 31) / 32, 2), dim3(1024), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

// Pixels of a workgroup: a wave's 64, or eight where those would be few workgroups.
static int lanes(const NormArgs& a) { return a.inner == 1 ? 1 : a.outer * a.inner >= 64 * 2048 ? 64 : 8; }

template <class T, int L>
static dwm_status_t forward_lanes(const NormArgs& a, bool join, hipStream_t stream)
{
    const long long tiles = (a.outer * a.inner + L - 1) / L;
    const dim3 grid((unsigned)(tiles < (1 << 20) ? tiles : 1 << 20));
    if (join) hipLaunchKernelGGL((norm_any_forward_kernel<T, L, true>), grid, dim3(256), 0, stream, a);
    else hipLaunchKernelGGL((norm_any_forward_kernel<T, L, false>), grid, dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

template <class T>
static dwm_status_t forward(const NormArgs& a, bool join, hipStream_t stream)
{
    const int L = lanes(a);
    return L == 1 ? forward_lanes<T, 1>(a, join, stream) : L == 8 ? forward_lanes<T, 8>(a, join, stream) : forward_lanes<T, 64>(a, join, stream);
}

template <class T>
static dwm_status_t backward(const NormArgs& a, hipStream_t stream)
{
    const long long positions = a.outer * a.inner;
    if (a.dgamma || a.dbeta) {  // first: dx may be dy's own memory
        if (a.inner == 1)
            hipLaunchKernelGGL((norm_any_params_kernel<T, 64>), dim3((a.C + 63) / 64, a.splits), dim3(256), 0, stream, a);
        else
            hipLaunchKernelGGL((norm_any_params_kernel<T, 1>), dim3(a.C, a.splits), dim3(256), 0, stream, a);
        if (hipGetLastError() != hipSuccess) return DWM_ERR_HIP;
        const dwm_status_t st = params_final<T>(a, stream);
        if (st != DWM_OK) return st;
    }
    if ((a.dx || a.dresidual) && positions > 0) {
        const int L = lanes(a);
        const long long tiles = (positions + L - 1) / L;
        const dim3 grid((unsigned)(tiles < (1 << 20) ? tiles : 1 << 20));
        if (L == 1) hipLaunchKernelGGL((norm_any_backward_kernel<T, 1>), grid, dim3(256), 0, stream, a);
        else if (L == 8) hipLaunchKernelGGL((norm_any_backward_kernel<T, 8>), grid, dim3(256), 0, stream, a);
        else hipLaunchKernelGGL((norm_any_backward_kernel<T, 64>), grid, dim3(256), 0, stream, a);
        if (hipGetLastError() != hipSuccess) return DWM_ERR_HIP;
    }
    return DWM_OK;
}

dwm_status_t launch_norm_any_forward(const NormArgs& a, dwm_type_t type, bool join, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    if (a.outer == 0) return DWM_OK;
    switch (type) {
        case DWM_F32: return forward<float>(a, join, s);
        case DWM_F16: return forward<_Float16>(a, join, s);
        case DWM_BF16: return forward<__bf16>(a, join, s);
    }
    return DWM_ERR_INVALID_ARG;
}

dwm_status_t launch_norm_any_backward(const NormArgs& a, dwm_type_t type, void* stream)
{
    switch (type) {
        case DWM_F32: return backward<float>(a, (hipStream_t)stream);
        case DWM_F16: return backward<_Float16>(a, (hipStream_t)stream);
        case DWM_BF16: return backward<__bf16>(a, (hipStream_t)stream);
    }
    return DWM_ERR_INVALID_ARG;
}

dwm_status_t launch_norm_params_final(const NormArgs& a, dwm_type_t type, void* stream)
{
    switch (type) {
        case DWM_F32: return params_final<float>(a, (hipStream_t)stream);
        case DWM_F16: return params_final<_Float16>(a, (hipStream_t)stream);
        case DWM_BF16: return params_final<__bf16>(a, (hipStream_t)stream);
    }
    return DWM_ERR_INVALID_ARG;
}

}  // namespace dwm

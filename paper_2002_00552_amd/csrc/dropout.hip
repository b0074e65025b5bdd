// Dropout (gfx950): y = keep ? x / (1 - p) : 0, the mask drawn from a counter (philox.hpp) in the forward pass and again in the
// backward one, where dy takes the place of x.  Memory alone bounds it: a thread owns sixteen bytes, whose one or two blocks of
// draws are made while they are on their way; one vector a thread and as many workgroups as that takes, which is what a
// copy does best with here (2 GiB: 6.2 TB/s, with two vectors a thread 5.7, with eight 4.2).
#include "elem.hpp"
#include "philox.hpp"

namespace dwm {

template <class T>
__global__ __launch_bounds__(256) void dropout_kernel(DropArgs d, long long first, long long n, const T* x, T* y)
{
    constexpr int V = kVec<T>;
    const long long e0 = first + ((long long)blockIdx.x * 256 + threadIdx.x) * V;
    if (e0 >= n) return;
    const uint64_t sequence = drop_sequence(d);
    if (e0 + V <= n) {
        const uint4v r = load_vector<T, V>(x + e0);
        bool keep[V];
        drop_keep<V>(d, sequence, (uint64_t)e0, true, keep);  // while the load is on its way
        float f[V];
        unpack<T, V>(r, f);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = drop_scaled(f[j], keep[j], d.scale);
        store_vector<T, V>(y + e0, pack<T, V>(f));
    } else {
        const uint32_t bits = drop_bits<V>(d, sequence, (uint64_t)e0, true);
        for (int j = 0; j < V; ++j)
            if (e0 + j < n) y[e0 + j] = (T)drop_scaled((float)x[e0 + j], bits, j, d.scale);
    }
}

template <class T>
static dwm_status_t launch(const DropArgs& d, long long n, const void* x, void* y, hipStream_t stream)
{
    const long long per = 256 * kVec<T>;
    const long long most = per << 23;  // a launch has fewer than 2^32 threads
    for (long long first = 0; first < n; first += most) {
        const long long here = n - first < most ? n - first : most;
        hipLaunchKernelGGL(dropout_kernel<T>, dim3((unsigned)((here + per - 1) / per)), dim3(256), 0, stream, d, first, n,
                           (const T*)x, (T*)y);
        if (hipGetLastError() != hipSuccess) return DWM_ERR_HIP;
    }
    return DWM_OK;
}

dwm_status_t launch_dropout(const DropArgs& d, dwm_type_t type, long long n, const void* x, void* y, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    switch (type) {
        case DWM_F32: return launch<float>(d, n, x, y, s);
        case DWM_F16: return launch<_Float16>(d, n, x, y, s);
        case DWM_BF16: return launch<__bf16>(d, n, x, y, s);
        default: return DWM_ERR_INVALID_ARG;
    }
}

}  // namespace dwm

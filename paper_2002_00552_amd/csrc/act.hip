// Activations with a bias, their checkpoints in 8 bits and their gradients from them, rows into 8 bits and back; the last sums of
// the parameters' gradients (gfx950).  Memory bounds all but the gelus in 16 bits, where the vector units come near it: an octet of
// neighbouring channels to a thread, one row at a time and as many waves as a CU holds (four rows at a time, with their loads together and half the waves: 148 us
// for 136, 199 for 159).  A workgroup's 256 threads lie along one row or along several short ones.  16384 rows of 8192 bfloat16 with a bias and
// checkpoints, out of the caches: gelu 136 us (5.0 TB/s), its gradient 150 (4.5) and 8 for the last sums; relu 117 and 136; to 8 bits and back 77 and 78 us (5.3 TB/s).
#include "rows8.hpp"

namespace dwm {

// Lanes of a row: a power of two from 4 to 256, in as many column tiles as it takes.
static int row_lanes(int C)
{
    int lanes = 4;
    while (lanes < 256 && lanes * kOctet < C) lanes *= 2;
    return lanes;
}
static int shift_of(int lanes) { return __builtin_ctz((unsigned)lanes); }

// x there: p = x + bias into 8 bits (kept) and through the activation (y); x not there: y is what kept stands for.
template <class T> __global__ __launch_bounds__(256) void act_forward_kernel(ActArgs a, int shift)
{
    const int octet = blockIdx.x * 256 + (threadIdx.x & ((1 << shift) - 1)), c = octet * 8, n = a.C - c;
    if ((octet & ~3) * 8 >= a.C) return;  // (behind the last block: all four lanes)
    const long long step = (long long)gridDim.y << (8 - shift);
    float bias[8];
    param_octet<T>(a.bias, a.param_typed, c, n, 0.0f, bias);
    for (long long row = ((long long)blockIdx.y << (8 - shift)) + (threadIdx.x >> shift); row < a.rows; row += step) {
        float p[8];
        if (a.x) {
            load_octet<T>((const T*)a.x + row * a.stride[kActX] + c, n, p);
            if (a.bias)
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] += bias[j];
            if (a.kept.codes) {
                uint32_t s;
                const uint2v codes = pack_octet<QuadLanes>(p, &s);
                store_packed(a.kept, row, octet, a.C, codes, s);
            }
            if (!a.y) continue;
            act_octet(a.act, p);
        } else {
            uint2v codes;
            uint32_t s;
            load_packed(a.kept, row, octet, a.C, &codes, &s);
            unpack_octet(codes, s, p);
        }
        if (n > 0) store_octet<T>((T*)a.y + row * a.stride[kActY] + c, n, p);
    }
}

// dx = dy * act'(p), p from its checkpoint or from x and bias; and the workgroup's sums of dx over its rows.
template <class T> __global__ __launch_bounds__(256) void act_backward_kernel(ActArgs a, int shift)
{
    __shared__ float sums[256 * 8];
    const int lane = threadIdx.x & ((1 << shift) - 1), octet = blockIdx.x * 256 + lane, c = octet * 8, n = a.C - c;
    const int group = threadIdx.x >> shift, groups = 256 >> shift;
    float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    if (n > 0) {
        float bias[8];
        param_octet<T>(a.bias, a.param_typed, c, n, 0.0f, bias);
        for (long long row = (long long)blockIdx.y * groups + group; row < a.rows; row += (long long)gridDim.y * groups) {
            float g[8], p[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            load_octet<T>((const T*)a.dy + row * a.stride[kActDy] + c, n, g);
            if (a.kept.codes) {
                uint2v codes;
                uint32_t s;
                load_packed(a.kept, row, octet, a.C, &codes, &s);
                unpack_octet(codes, s, p);
            } else if (a.x) {
                load_octet<T>((const T*)a.x + row * a.stride[kActX] + c, n, p);
                if (a.bias)
#pragma unroll
                    for (int j = 0; j < 8; ++j) p[j] += bias[j];
            }
            slope_octet(a.act, p, g);
            if (a.dx) store_octet<T>((T*)a.dx + row * a.stride[kActDx] + c, n, g);
#pragma unroll
            for (int j = 0; j < 8; ++j) acc[j] += g[j];
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[(group * 8 + j) * (256 / groups) + lane] = acc[j];
    __syncthreads();
    if (group || n <= 0) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        acc[j] = 0.0f;
        for (int g = 0; g < groups; ++g) acc[j] += sums[(g * 8 + j) * (256 / groups) + lane];
    }
    store_octet<float>(a.partial + (long long)blockIdx.y * a.C + c, n, acc);
}

// Sixteen channels of a workgroup and 64 threads along the splits for each: all of a thread's loads go out together, as long as it has
// no more than sixteen.  The order of the sums is the same in every run.
template <class P> __global__ __launch_bounds__(1024) void columns_kernel(const float* partial, int splits, int C, P* out)
{
    __shared__ float sums[64][17];
    const int lane = threadIdx.x % 16, part = threadIdx.x / 16, c = blockIdx.x * 16 + lane;
    float v = 0.0f;
    if (c < C)
#pragma unroll 16
        for (int s = part; s < splits; s += 64) v += partial[(long long)s * C + c];
    sums[part][lane] = v;
    __syncthreads();
    if (part < 16) {
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) v += sums[part + 16 * i][lane];
        sums[part][lane] = v;  // (read by this thread alone before)
    }
    __syncthreads();
    if (part || c >= C) return;
    v = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; ++i) v += sums[i][lane];
    out[c] = (P)v;
}

// Workgroups along the rows, at most: fewer than 2^32 threads in all.
static long long most_blocks(int groups) { return groups > 128 ? (1 << 23) / groups : 65535; }

template <class T> static dwm_status_t forward(const ActArgs& a, hipStream_t s)
{
    const int lanes = row_lanes(a.C), rows = 256 / lanes, groups = (a.C + 2047) / 2048;
    const long long blocks = (a.rows + rows - 1) / rows, most = most_blocks(groups);
    hipLaunchKernelGGL(act_forward_kernel<T>, dim3(groups, (unsigned)(blocks < most ? blocks : most)), dim3(256), 0, s, a, shift_of(lanes));
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}
template <class T> static dwm_status_t backward(const ActArgs& a, hipStream_t s)
{
    hipLaunchKernelGGL(act_backward_kernel<T>, dim3((a.C + 2047) / 2048, a.splits), dim3(256), 0, s, a, shift_of(row_lanes(a.C)));
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

dwm_status_t launch_act_forward(const ActArgs& a, dwm_type_t type, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    switch (type) {
        case DWM_F32: return forward<float>(a, s);
        case DWM_F16: return forward<_Float16>(a, s);
        case DWM_BF16: return forward<__bf16>(a, s);
        default: return DWM_ERR_INVALID_ARG;
    }
}

dwm_status_t launch_act_backward(const ActArgs& a, dwm_type_t type, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    switch (type) {
        case DWM_F32: return backward<float>(a, s);
        case DWM_F16: return backward<_Float16>(a, s);
        case DWM_BF16: return backward<__bf16>(a, s);
        default: return DWM_ERR_INVALID_ARG;
    }
}

// An octet to a thread; rows of one or two of a product's operands that lie anywhere.
__global__ __launch_bounds__(256) void aligned_rows_kernel(AlignedRows first, AlignedRows second)
{
    const AlignedRows& r = blockIdx.y ? second : first;
    const int octets = (int)(r.to_stride / 8);
    const long long total = r.rows * octets;
    for (long long at = (long long)blockIdx.x * 256 + threadIdx.x; at < total; at += (long long)gridDim.x * 256) {
        const long long row = at / octets;
        const int c = (int)(at - row * octets) * 8;
        *(uint4v*)((_Float16*)r.to + row * r.to_stride + c) = fetch_octet<_Float16>((const _Float16*)r.from + row * r.stride + c, r.width - c).r[0];  // (bits, not numbers)
    }
}

dwm_status_t launch_aligned_rows(const AlignedRows* r, int count, void* stream)
{
    long long blocks = 1;
    for (int i = 0; i < count; ++i) {
        const long long own = (r[i].rows * (r[i].to_stride / 8) + 255) / 256;
        if (own > blocks) blocks = own;
    }
    hipLaunchKernelGGL(aligned_rows_kernel, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20), (unsigned)count), dim3(256), 0, (hipStream_t)stream, r[0], r[count - 1]);
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

dwm_status_t launch_columns(const float* partial, int splits, int C, void* out, dwm_type_t type, void* stream)
{
    const hipStream_t s = (hipStream_t)stream;
    const dim3 grid((C + 15) / 16), block(1024);
    switch (type) {
        case DWM_F32: hipLaunchKernelGGL(columns_kernel<float>, grid, block, 0, s, partial, splits, C, (float*)out); break;
        case DWM_F16: hipLaunchKernelGGL(columns_kernel<_Float16>, grid, block, 0, s, partial, splits, C, (_Float16*)out); break;
        case DWM_BF16: hipLaunchKernelGGL(columns_kernel<__bf16>, grid, block, 0, s, partial, splits, C, (__bf16*)out); break;
        default: return DWM_ERR_INVALID_ARG;
    }
    return hipGetLastError() == hipSuccess ? DWM_OK : DWM_ERR_HIP;
}

}  // namespace dwm

// The pointwise branch over rows (norms, activations, rows in 8 bits, matrix products): what the host side and the kernels share.
// Plain C++.
#pragma once
#include <cstddef>
#include <cstdint>

#include "../../include/dwm.h"

namespace dwm {

// Rows in 8 bits: codes null where there are none.
struct Packed {
    uint8_t *codes, *scales;
};
constexpr int kBlock = 32, kOctet = 8;  // channels of a scale, and of a thread
inline long long packed_width(long long C) { return (C + kBlock - 1) / kBlock * kBlock; }       // bytes of a row of codes
inline long long packed_scales(long long C) { return (C + 4 * kBlock - 1) / (4 * kBlock) * 4; }  // and of scales

// The largest tensor, in elements: kernels count in 64 bits, and a byte offset stays far from their end.
constexpr long long kMostElements = 1LL << 40;
constexpr int kMostChannels = 1 << 20;

// Root-mean-square norms.
enum RmsTensor { kRmsX, kRmsResidual, kRmsZ, kRmsY, kRmsDy, kRmsDz, kRmsDx, kRmsTensors };
struct RmsArgs {
    const void *x, *residual, *gamma, *dy, *dz;
    void *z, *y, *dx;
    Packed packed_y, kept;
    float *rstd, *partial;  // [rows], [splits][C]
    long long stride[kRmsTensors];
    long long rows;
    int C, param_typed, splits;
    double eps, inverse;  // 1 / C
};
// Threads of a row, octets of a thread; variant i + 1 is entry i, built forward and backward.  The planner takes those of one octet and, past 8192 channels, the last; the others are for
// dwm_rms_set_variant alone.
struct RmsShape {
    int tpr, k;
    static constexpr bool forward = true, backward = true;
};
constexpr RmsShape kRmsShapes[] = {
    {4, 1}, {8, 1}, {16, 1}, {32, 1}, {64, 1}, {64, 2}, {128, 1}, {128, 2}, {256, 1}, {256, 2}, {512, 1}, {512, 2}, {1024, 1}, {1024, 2},
};
constexpr int kRmsShapeCount = sizeof(kRmsShapes) / sizeof(kRmsShapes[0]);

// Activations and their checkpoints.
enum ActTensor { kActX, kActY, kActDy, kActDx, kActTensors };
struct ActArgs {
    const void *x, *bias, *dy;
    void *y, *dx;
    Packed kept;
    float* partial;  // [splits][C]
    long long stride[kActTensors];
    long long rows;
    int C, param_typed, splits, act;
};

// Matrix products.
enum MatmulTensor { kMatA, kMatB, kMatResidual, kMatOut, kMatTensors };
struct MatmulArgs {
    const void *a, *b;
    const uint8_t *a_scales, *b_scales;
    const void *bias, *residual;
    void* out;
    Packed packed_y, kept;
    float* partial;  // [splits][M][width of N]
    long long stride[kMatTensors];
    int M, N, K, splits, act;
    int param_typed, wide_out;  // bias has the operands' 16-bit type, out and residual have 32 bits
    int bf16_out;               // packed operands: the type of out (else binary16)
};
// Tiles of the result, few rows; the first two and the last (never a plan's own kernel) for operands of any alignment.
enum MatmulKernel { kMatAny, kMatAny64, kMat64, kMat128, kMat256, kMatFew, kMatFewLoose };
constexpr int kMatFewRows = 32;
struct MatmulShape {
    int kernel, splits;
};
inline long long matmul_partial_width(int N) { return packed_width(N); }

// `rows` rows of `width` 16-bit elements from anywhere to rows of `to_stride` (a multiple of 8, at a multiple of 16 bytes), zeros behind each.
struct AlignedRows {
    const void* from;
    long long stride;
    void* to;
    long long to_stride, rows;
    int width;
};

dwm_status_t launch_rms_forward(const RmsArgs& a, dwm_type_t type, int kernel, void* stream);
dwm_status_t launch_rms_backward(const RmsArgs& a, dwm_type_t type, int kernel, void* stream);
dwm_status_t launch_act_forward(const ActArgs& a, dwm_type_t type, void* stream);
dwm_status_t launch_act_backward(const ActArgs& a, dwm_type_t type, void* stream);
// out[c] = sum over the splits of partial[split][c], in the order of the splits.
dwm_status_t launch_columns(const float* partial, int splits, int C, void* out, dwm_type_t type, void* stream);
dwm_status_t launch_aligned_rows(const AlignedRows* r, int count, void* stream);  // one or two
// flags: DWM_A_ACROSS, DWM_B_ACROSS.
dwm_status_t launch_matmul_f16(const MatmulArgs& a, int flags, int kernel, void* stream);
dwm_status_t launch_matmul_bf16(const MatmulArgs& a, int flags, int kernel, void* stream);
dwm_status_t launch_matmul_packed(const MatmulArgs& a, int flags, int kernel, void* stream);

}  // namespace dwm

struct dwm_rms_plan {
    long long rows;
    int C;
    dwm_type_t type, param_type;
    double eps;
    long long stride[dwm::kRmsTensors];
    int forward, backward, splits;
    void* ws;
};

struct dwm_act_plan {
    long long rows;
    int C;
    dwm_type_t type, param_type;
    dwm_act_t act;
    long long stride[dwm::kActTensors];
    int splits;
    void* ws;
};

struct dwm_matmul_plan {
    int M, N, K, flags;
    dwm_type_t operands, type, param_type;
    dwm_act_t act;
    long long stride[dwm::kMatTensors];
    int asked_kernel;        // by dwm_matmul_set_variant; negative: the planner's choice
    dwm::MatmulShape shape;  // where the operands are aligned
    dwm::MatmulShape any;    // and where they are not
    bool copies;             // operands whose rows are no multiple of eight elements are laid out anew first, and `shape` runs
    void* ws;
};

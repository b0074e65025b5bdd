// Layer norms, dropouts and joins of residual branches: what the host side and the kernels share.  Plain C++.
#pragma once
#include <cstddef>
#include <cstdint>

#include "../../include/dwm.h"

namespace dwm {

// What a kernel needs of a dwm_dropout_t.
struct DropArgs {
    int mode;            // kDropNone, kDropDraw, kDropAll
    uint32_t threshold;  // an element is kept where its word is not below this
    float scale;         // 1 / (1 - p)
    uint32_t seed_lo, seed_hi;
    uint64_t sequence;
    const unsigned long long* sequence_dev;  // added to sequence if not null
};
enum { kDropNone = 0, kDropDraw = 1, kDropAll = 2 };

// Tensors [outer][C][inner]: element (o, c, i) lies at o * stride + c * inner + i.
enum NormTensor { kNormX, kNormResidual, kNormZ, kNormY, kNormDy, kNormDz, kNormDx, kNormDresidual, kNormTensors };

// One call.  The norm's input is z: the plain norm's x goes by that name in the backward kernels, and its dx by dresidual.
struct NormArgs {
    const void *x, *residual, *dy, *dz, *gamma, *beta;
    void *z, *y, *dx, *dresidual, *dgamma, *dbeta;
    float *mean, *rstd;  // [outer][inner]
    float* partial;      // [splits][2][C]: sums of dy * xhat and of dy over a part of the positions
    long long stride[kNormTensors];
    long long outer, inner;
    int C;
    int param_typed;  // parameters have the tensors' type, otherwise binary32
    int splits;       // workgroups of a backward kernel for the gradient of z
    int aside;        // in front of them, others for the parameters' gradients (their number, set at the launch); `partial` is null then
    float eps;
    DropArgs drop;
};

// The shapes that the register-resident kernels (norm_impl.inc) are built in, from the narrowest to the widest.  Rows: threads of a row, vectors of
// sixteen bytes of a thread, and in which directions the shape is built.  Maps: lanes along the pixels, groups along the channels,
// channels of a thread.
struct NormRows {
    int tpr, k;
    bool forward, backward;
};
struct NormMaps {
    int pl, cg, k;
    bool one;            // with one pixel a lane too
    int join, backward;  // the largest element size of a join's forward kernel and of a backward one (0: none)
};
constexpr NormRows kNormRows[] = {
    {8, 1, true, true},    {16, 1, true, true},   {32, 1, true, true},   {64, 1, true, true},   {64, 2, true, false},  {128, 1, true, true},   {128, 2, true, false},
    {256, 1, true, true},  {256, 2, true, false}, {512, 1, true, true},  {512, 2, true, true},  {1024, 2, true, true}, {1024, 4, true, true},
};
constexpr NormMaps kNormMaps[] = {
    {64, 4, 4, true, 4, 4}, {64, 4, 8, false, 4, 4}, {16, 16, 4, true, 4, 4}, {8, 32, 4, true, 4, 4},  {16, 16, 8, false, 4, 2}, {8, 32, 6, false, 4, 0},  {8, 32, 8, false, 0, 0},
    {8, 64, 4, true, 4, 4}, {4, 128, 4, true, 4, 4}, {8, 64, 6, false, 4, 2}, {8, 64, 8, false, 2, 2}, {4, 256, 4, true, 4, 4},  {8, 128, 8, false, 2, 2}, {4, 256, 8, true, 4, 4},
};
constexpr int kNormRowsShapes = sizeof(kNormRows) / sizeof(kNormRows[0]), kNormMapsShapes = sizeof(kNormMaps) / sizeof(kNormMaps[0]);

// Threads of a backward workgroup over rows, and how many workgroups at most: each writes its sums of the parameters' gradients.  One of 1024 on
// each CU where a wave or more hold a row in one vector a thread, without an odd end; two of 512 elsewhere, for the registers and the
// sums over many short rows (a join in bfloat16, us, 512 and 1024 threads: 16384 rows of 4096 144, 129; 65536 of 2048 277, 248; of 1500
// 257, 292; 2048 of 64 8.2, 10.2; 16384 of 8192, two vectors a thread, 252, 439).
constexpr int norm_rows_threads(NormRows r, bool tail) { return r.tpr > 512 || (r.tpr >= 128 && r.k == 1 && !tail) ? 1024 : 512; }
constexpr int norm_rows_blocks(int threads) { return 256 * 1024 / threads; }
constexpr int kNormRowsWidest = 16384;  // channels that a backward kernel holds: the sums of dgamma and dbeta fill 128 KB of LDS
constexpr int kNormMapsPixels = 4;      // of a lane

#ifdef __HIPCC__
#define DWM_HD __host__ __device__
#else
#define DWM_HD
#endif

// Vector `index` of `length` elements in a line (a row's channels, an image's pixels), vec to a vector: where it starts, and the first of its elements that
// are its own, vec if there is no such vector.  Where the length is no multiple of vec the last one starts early, in the line.
struct NormVector {
    int start, first;
};
DWM_HD inline NormVector norm_vector(int index, int length, int vec)
{
    const int at = index * vec;
    if (at >= length) return {0, vec};
    const int start = at + vec <= length ? at : length - vec;
    return {start, at - start};
}

// The tiles of workgroup `block` of n: tile, tile + step, ... below end.  Workgroups go to the eight XCDs in turn, so each XCD is given a run of the tiles:
// lines that two tiles of an image share, at every channel where its rows are no multiple of 128 bytes, are read and written through
// one L2 (32 images of 256 channels, 28 x 28, binary16, forward: 11.0 us without this, 9.9 with it).
struct NormTiles {
    long long tile, end, step;
};
DWM_HD inline NormTiles norm_tiles(long long tiles, int block, int n)
{
    const int xcd = block % 8, mine = (n - xcd + 7) / 8;                         // workgroups of this XCD
    const long long before = (long long)xcd * (n / 8) + (xcd < n % 8 ? xcd : n % 8);  // and of those in front of it
    const bool each = tiles == n;
    return {(each ? before : tiles * before / n) + block / 8, each ? before + mine : tiles * (before + mine) / n, mine};
}

// A plan's kernel: 0 (norm_any.hip), or a shape from here on of rows, of maps with four pixels a lane, with one.
constexpr int kNormAny = 0, kNormRowsFirst = 1, kNormMapsVec = 100, kNormMapsOne = 200;

struct NormShape {
    int kernel;
    int blocks;  // workgroups; backward: splits of the parameters' gradients too
    bool aside;  // backward: the parameters' gradients by workgroups of their own in the same launch
};

// The planner's choice (variant < 0), or the kernel asked for; kernel = -1: it does not apply.
enum NormStage { kNormForward, kNormJoinForward, kNormBackward, kNormStages };
NormShape norm_choose(long long outer, int C, long long inner, dwm_type_t type, NormStage stage, int variant);

dwm_status_t launch_norm_any_forward(const NormArgs& a, dwm_type_t type, bool join, void* stream);
dwm_status_t launch_norm_any_backward(const NormArgs& a, dwm_type_t type, void* stream);
dwm_status_t launch_norm_params_final(const NormArgs& a, dwm_type_t type, void* stream);
dwm_status_t launch_norm_f32(const NormArgs& a, const NormShape& shape, bool backward, bool join, void* stream);
dwm_status_t launch_norm_f16(const NormArgs& a, const NormShape& shape, bool backward, bool join, void* stream);
dwm_status_t launch_norm_bf16(const NormArgs& a, const NormShape& shape, bool backward, bool join, void* stream);
dwm_status_t launch_dropout(const DropArgs& d, dwm_type_t type, long long n, const void* x, void* y, void* stream);

}  // namespace dwm

struct dwm_norm_plan {
    long long outer, inner;
    int C;
    dwm_type_t type, param_type;
    float eps;
    long long stride[dwm::kNormTensors];
    dwm::NormShape shape[dwm::kNormStages];
    void* ws;
};

// The pointwise branch over rows: plans, checks of arguments and entry points (host only, plain C++).
#include "branch.hpp"

#include <cstring>
#include <new>

namespace dwm {
namespace {

size_t size_of(dwm_type_t type) { return type == DWM_F32 ? 4 : 2; }
bool known(dwm_type_t type) { return type == DWM_F32 || type == DWM_F16 || type == DWM_BF16; }
bool known(dwm_act_t act) { return act >= DWM_ACT_NONE && act <= DWM_ACT_SILU; }
bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

bool rows_fit(long long rows, long long C) { return C <= kMostChannels && (C == 0 || rows <= kMostElements / C); }

// Packed rows that a call is given: there in whole, and where they have to lie.
bool packed_ok(const dwm_packed_t* p) { return !p || (p->codes && p->scales && aligned(p->codes, 16) && aligned(p->scales, 4)); }
Packed packed_of(const dwm_packed_t* p) { return p ? Packed{(uint8_t*)p->codes, (uint8_t*)p->scales} : Packed{nullptr, nullptr}; }

template <int N> int named(const char* const (&names)[N], const char* name)
{
    for (int i = 0; name && i < N; ++i)
        if (!std::strcmp(name, names[i])) return i;
    return -1;
}

bool rms_fits(int variant, int C)
{
    if (variant < 1 || variant > kRmsShapeCount) return variant == 0;
    const RmsShape& s = kRmsShapes[variant - 1];
    return s.tpr * s.k * kOctet >= C;
}

// The narrowest shape that holds a row with one octet a thread, or, past 8192 channels, two (16384 rows of 4096 bfloat16, z and y: 256 threads with two octets 116 us,
// 512 with one 109; backward 114 and 108).
int rms_choice(int C)
{
    for (int octets = 1; octets <= 2; ++octets)
        for (int v = 1; v <= kRmsShapeCount; ++v)
            if (rms_fits(v, C) && kRmsShapes[v - 1].k == octets) return v;
    return 0;
}

int rms_splits(long long rows, int C, int kernel)
{
    if (kernel == 0) {
        const long long groups = (C + 2047) / 2048, most = groups > 1024 ? 1 : 1024 / groups, some = (rows + 31) / 32;
        return (int)(some < 1 ? 1 : some < most ? some : most);
    }
    const int tpr = kRmsShapes[kernel - 1].tpr, threads = tpr > 256 ? tpr : 256;
    const long long blocks = (rows + threads / tpr - 1) / (threads / tpr), most = 256 * 1024 / threads;
    return (int)(blocks < 1 ? 1 : blocks < most ? blocks : most);
}

// Parts of the rows, a workgroup each for 2048 channels: up to 2048 workgroups, of four rows a thread at least where there are that many (16384 rows of 8192 bfloat16, gelu, with
// the last sums: 1024 workgroups 164 us, 2048 159).
int act_splits(long long rows, int C)
{
    const long long groups = (C + 2047) / 2048, most = groups > 2048 ? 1 : 2048 / groups;
    long long lanes = 1;
    while (lanes < 256 && lanes * kOctet < C) lanes *= 2;
    const long long each = (rows + 256 / lanes - 1) / (256 / lanes), per = each * groups >= 2048 ? 4 : each * groups >= 1024 ? 2 : 1, some = (each + per - 1) / per;
    return (int)(some < 1 ? 1 : some < most ? some : most);
}

// What a tile's kernel takes, in us: a step of 128 bytes of K for a workgroup that has a CU to itself, for one of several on every CU (each CU's share), how
// many a CU holds, and what a workgroup takes before its first and after its last step.  From 45 shapes of 1 to 16384 rows, 64 to 16384 columns and 256
// to 16384 terms in bfloat16 and 8 bits, operands out of the caches, each with one to eight parts: the choice by these is 3% behind the best on the average, a
// fifth at most.
struct MatmulRate {
    int side;
    double alone, shared;
    int held;
    double ends;
};
const MatmulRate kMatmulRates[] = {
    {128, 1.9, 1.3, 2, 3.5},   // any alignment (4001 x 4003 x 4005: 351 us, with 64 x 64 tiles 365; 2000 x 2001 x 2003: 63, 54)
    {64, 0.7, 0.35, 4, 1.5},   // any alignment (1000 x 777 x 1021: 16 us, with 128 x 128 tiles 34; both across 22, 64)
    {64, 0.32, 0.17, 2, 1.5},  // 512 x 512 x 16384: 60 us, in eight parts 22, with 128 x 128 tiles 156, 30; 1024 x 1024 x 1024: 8, 15
    {128, 0.68, 0.47, 2, 3.5}, // 2048 x 4096 x 1024: 20 us, with 64 x 64 tiles 31, with 256 x 256 29
    {256, 1.2, 1.5, 1, 8.0},   // 2048 x 8192 x 2048: 58 us, with 128 x 128 tiles 70
};

double matmul_cost(const dwm_matmul_plan& p, int kernel, int splits)
{
    const double elements = (double)p.N * p.K, launch = 3.5;
    if (kernel >= kMatFew)  // b once, and a again and again from the L2 (N = 12288, K = 4096 bfloat16, M = 1, 16, 32: 22, 32, 43 us, by tiles 24 to 26)
        return launch + elements * 1e-6 * ((p.operands == DWM_PACKED ? 0.2 : 0.33) + 0.011 * p.M);
    const MatmulRate& r = kMatmulRates[kernel];
    const long long step = p.operands == DWM_PACKED ? 128 : 64, steps = (p.K + step - 1) / step, part = (steps + splits - 1) / splits;
    const double more = kernel == kMatAny ? 0.4 : kernel == kMatAny64 ? 0.25 : kernel < kMat256 ? 0.15 : 0;  // (twice as many LDS reads, and strides of whole rows)
    const double across = 1 + more * (!!(p.flags & DWM_A_ACROSS) + !!(p.flags & DWM_B_ACROSS));
    const double groups = (double)((p.M + r.side - 1) / r.side) * ((p.N + r.side - 1) / r.side) * splits, rounds = groups / (256.0 * r.held);
    const double each = groups <= 256 ? 1 : rounds >= 1 ? r.held : groups / 256, step_time = across * (each * r.shared > r.alone ? each * r.shared : r.alone);
    double time = launch + (rounds <= 1 ? 1 : rounds < 4 ? (double)(long long)(rounds + 0.999) : rounds + 0.5) * (part * step_time + r.ends * (each > 2 ? 2 : each > 1 ? 1.4 : 1));
    if (splits > 1) time += 5.5 + (double)p.M * p.N * (8.0 * splits + 2) / 6.5e6;  // the parts' sums there and back, and a launch
    return time;
}

bool matmul_applies(const dwm_matmul_plan& p, int kernel)
{
    if (kernel == kMatFew) return p.M <= kMatFewRows && p.flags == 0;
    return kernel <= kMatAny64 ? kernel >= 0 && p.operands != DWM_PACKED : kernel < kMatFew;
}

// Whether a launch can hold a workgroup for each tile and part: fewer than 2^32 threads (results of 2^36 elements on in tiles of 64 x 64; one part in larger ones always).
bool matmul_launches(const dwm_matmul_plan& p, int kernel, int splits)
{
    if (kernel >= kMatFew) return true;
    const long long side = kMatmulRates[kernel].side;
    return (p.M + side - 1) / side * ((p.N + side - 1) / side) * splits * (side == 256 ? 512 : 256) < 1LL << 32;
}

// The cheapest of some kernels, with as many parts of K as are asked for or the best number of them, each of four steps at least; kernel -1 where none can be launched.
MatmulShape matmul_shape(const dwm_matmul_plan& p, int first, int last, int splits)
{
    MatmulShape best = {-1, 1};
    double least = -1;
    const long long step = p.operands == DWM_PACKED ? 128 : 64, steps = (p.K + step - 1) / step;
    for (int kernel = first; kernel <= last; ++kernel)
        for (int s = 1; s <= 16; s *= 2) {
            if (s > 1 && (kernel >= kMatFew || splits > 0 || s * 4 > steps)) continue;
            const int parts = splits > 0 && kernel < kMatFew ? splits : s;
            if (!matmul_launches(p, kernel, parts)) continue;
            const double cost = matmul_cost(p, kernel, parts);
            if (least < 0 || cost < least) {
                least = cost;
                best = {kernel, parts};
            }
        }
    return best;
}

// An operand of 16 bits: its rows, their length, and whether that keeps it from being read sixteen bytes at a time wherever it lies.
struct OperandRows {
    long long rows, length;
    bool odd() const { return length % 8 != 0; }
    long long stride() const { return (length + 7) / 8 * 8; }  // of a copy
    size_t bytes() const { return odd() ? (size_t)(rows * stride() * 2 + 255) / 256 * 256 : 0; }
};
OperandRows operand_rows(const dwm_matmul_plan& p, bool second)
{
    const bool across = p.flags & (second ? DWM_B_ACROSS : DWM_A_ACROSS);
    const long long own = second ? p.N : p.M;
    return across ? OperandRows{p.K, own} : OperandRows{own, p.K};
}

// Laying odd operands out anew: a launch, and their bytes there and back.
double copies_cost(const dwm_matmul_plan& p)
{
    double time = 4;
    for (int second = 0; second < 2; ++second) {
        const OperandRows r = operand_rows(p, second);
        if (r.odd()) time += (double)r.rows * r.length * 4 / 4.0e6;
    }
    return time;
}
size_t parts_bytes(const dwm_matmul_plan& p)
{
    const int splits = p.shape.splits > p.any.splits ? p.shape.splits : p.any.splits;
    return splits > 1 ? ((size_t)splits * p.M * matmul_partial_width(p.N) * sizeof(float) + 255) / 256 * 256 : 0;
}

// kernel, splits: negative for the planner's choice.  False, and the plan as it was, for what cannot be launched.
bool matmul_plan(dwm_matmul_plan& plan, int kernel, int splits)
{
    dwm_matmul_plan p = plan;
    const bool few = matmul_applies(p, kMatFew) && splits <= 1;
    p.shape = kernel >= 0 ? matmul_shape(p, kernel, kernel, splits) : matmul_shape(p, kMat64, few ? kMatFew : kMat256, splits);
    if (p.shape.kernel < 0) return false;
    if (p.operands == DWM_PACKED || p.shape.kernel <= kMatAny64) {
        p.any = p.shape;
    } else if (kernel == kMatFew || (kernel < 0 && few && matmul_cost(p, kMatFewLoose, 1) < matmul_cost(p, kMatAny64, matmul_shape(p, kMatAny64, kMatAny64, splits).splits))) {
        p.any = {kMatFewLoose, 1};
    } else {
        p.any = matmul_shape(p, kMatAny, kMatAny64, splits);
        if (p.any.kernel < 0) return false;
    }
    // Rows of odd lengths: the kernels for any alignment, or, where it costs less (or a kernel for aligned operands was asked for), copies and those for aligned ones
    // (bfloat16, us, without and with: 4001 x 4003 x 4005 350, 142; 1000 x 777 x 1021 16.3, 13.6, both across 22.7, 13.9; 300 x 300 x 500 8.3, 12.4).
    const OperandRows a = operand_rows(p, false), b = operand_rows(p, true);
    p.copies = p.operands != DWM_PACKED && (a.odd() || b.odd()) && p.K > 0 && p.shape.kernel >= kMat64 && p.shape.kernel <= kMat256 && a.stride() <= 1 << 22 && b.stride() <= 1 << 22 &&
               (kernel >= 0 || matmul_cost(p, p.shape.kernel, p.shape.splits) + copies_cost(p) < matmul_cost(p, p.any.kernel, p.any.splits));
    if (p.operands != DWM_PACKED && (a.odd() || b.odd()) && p.K > 0 && !p.copies) p.shape = p.any;  // (no address or stride makes these whole vectors)
    plan = p;
    return true;
}

// Whether the kernels that copy sixteen bytes at a time straight into LDS can read an operand; a tile's 256 rows have to lie within 2^32 bytes.
bool operand_aligned(const void* p, long long stride, long long length)
{
    return aligned(p, 16) && stride % 8 == 0 && length % 8 == 0 && stride <= 1 << 22;
}

dwm_status_t run_matmul(const dwm_matmul_plan& p, MatmulArgs& a, const MatmulShape& shape, const long long* strides, const void* bias,
                        const void* residual, void* out, const dwm_packed_t* packed_y, const dwm_packed_t* kept, void* stream)
{
    if (shape.splits > 1 && !p.ws) return DWM_ERR_WORKSPACE;
    std::memcpy(a.stride, p.stride, sizeof(a.stride));
    a.stride[kMatA] = strides[0];
    a.stride[kMatB] = strides[1];
    a.bias = bias;
    a.residual = residual;
    a.out = out;
    a.packed_y = packed_of(packed_y);
    a.kept = packed_of(kept);
    a.partial = (float*)p.ws;
    a.M = p.M;
    a.N = p.N;
    a.K = p.K;
    a.splits = shape.splits;
    a.act = p.act;
    a.param_typed = p.param_type != DWM_F32;
    a.wide_out = p.type == DWM_F32;
    a.bf16_out = p.type == DWM_BF16;
    switch (p.operands) {
        case DWM_F16: return launch_matmul_f16(a, p.flags, shape.kernel, stream);
        case DWM_BF16: return launch_matmul_bf16(a, p.flags, shape.kernel, stream);
        case DWM_PACKED: return launch_matmul_packed(a, p.flags, shape.kernel, stream);
        default: return DWM_ERR_INVALID_ARG;
    }
}

// What both matmul calls ask of everything but the operands.
dwm_status_t matmul_ok(const dwm_matmul_plan& p, const void* bias, const void* residual, const void* out, const dwm_packed_t* packed_y,
                       const dwm_packed_t* kept)
{
    if (!(out || packed_y || kept || p.M == 0 || p.N == 0) || !aligned(bias, size_of(p.param_type)) || !aligned(residual, size_of(p.type)) ||
        !aligned(out, size_of(p.type)) || !packed_ok(packed_y) || !packed_ok(kept))
        return DWM_ERR_INVALID_ARG;
    return (packed_y || kept) && !rows_fit(p.M, p.N) ? DWM_ERR_UNSUPPORTED : DWM_OK;
}

const char* const kRmsNames[kRmsTensors] = {"x", "residual", "z", "y", "dy", "dz", "dx"};
const char* const kActNames[kActTensors] = {"x", "y", "dy", "dx"};
const char* const kMatNames[kMatTensors] = {"a", "b", "residual", "out"};

}  // namespace
}  // namespace dwm

using namespace dwm;

extern "C" {

size_t dwm_packed_codes_bytes(long long rows, int C)
{
    return rows < 0 || C < 1 || !rows_fit(rows, C) ? 0 : (size_t)(rows * packed_width(C));
}

size_t dwm_packed_scales_bytes(long long rows, int C)
{
    return rows < 0 || C < 1 || !rows_fit(rows, C) ? 0 : (size_t)(rows * packed_scales(C));
}

static dwm_status_t pack_args(ActArgs* a, dwm_type_t type, long long rows, int C, const void* tensor, long long stride,
                              const dwm_packed_t* packed)
{
    if (!known(type) || rows < 0 || C < 1 || stride < C || (rows > 0 && (!tensor || !packed)) || !packed_ok(packed) || !aligned(tensor, size_of(type)))
        return DWM_ERR_INVALID_ARG;
    if (!rows_fit(rows, C) || (rows > 0 && stride > kMostElements / rows)) return DWM_ERR_UNSUPPORTED;
    *a = ActArgs{};
    a->rows = rows;
    a->C = C;
    a->kept = packed_of(packed);
    for (long long& s : a->stride) s = stride;
    return DWM_OK;
}

dwm_status_t dwm_pack(dwm_type_t type, long long rows, int C, const void* x_dev, long long stride, const dwm_packed_t* packed, void* stream)
{
    ActArgs a;
    const dwm_status_t st = pack_args(&a, type, rows, C, x_dev, stride, packed);
    if (st != DWM_OK || rows == 0) return st;
    a.x = x_dev;
    return launch_act_forward(a, type, stream);
}

dwm_status_t dwm_unpack(dwm_type_t type, long long rows, int C, const dwm_packed_t* packed, void* y_dev, long long stride, void* stream)
{
    ActArgs a;
    const dwm_status_t st = pack_args(&a, type, rows, C, y_dev, stride, packed);
    if (st != DWM_OK || rows == 0) return st;
    a.y = y_dev;
    return launch_act_forward(a, type, stream);
}

dwm_status_t dwm_rms_plan_create(dwm_rms_plan_t** out, long long rows, int C, dwm_type_t type, dwm_type_t param_type, double eps)
{
    if (!out || rows < 0 || C < 1 || !known(type) || !(param_type == DWM_F32 || param_type == type) || !(eps >= 0.0) || !(eps <= 3e38))
        return DWM_ERR_INVALID_ARG;
    if (!rows_fit(rows, C)) return DWM_ERR_UNSUPPORTED;
    dwm_rms_plan* p = new (std::nothrow) dwm_rms_plan;
    if (!p) return DWM_ERR_ALLOC;
    std::memset(p, 0, sizeof(*p));
    p->rows = rows;
    p->C = C;
    p->type = type;
    p->param_type = param_type;
    p->eps = eps;
    for (long long& s : p->stride) s = C;
    p->forward = p->backward = rms_choice(C);
    p->splits = rms_splits(rows, C, p->backward);
    *out = p;
    return DWM_OK;
}

dwm_status_t dwm_rms_plan_destroy(dwm_rms_plan_t* plan)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    delete plan;
    return DWM_OK;
}

dwm_status_t dwm_rms_plan_info(const dwm_rms_plan_t* plan, dwm_rms_info_t* info)
{
    if (!plan || !info) return DWM_ERR_INVALID_ARG;
    *info = dwm_rms_info_t{plan->rows, plan->C, plan->forward, plan->backward, plan->splits};
    return DWM_OK;
}

dwm_status_t dwm_rms_set_stride(dwm_rms_plan_t* plan, const char* tensor, long long stride)
{
    const int which = named(kRmsNames, tensor);
    if (!plan || which < 0 || stride < plan->C) return DWM_ERR_INVALID_ARG;
    if (plan->rows > 0 && stride > kMostElements / plan->rows) return DWM_ERR_UNSUPPORTED;
    plan->stride[which] = stride;
    return DWM_OK;
}

dwm_status_t dwm_rms_set_variant(dwm_rms_plan_t* plan, const char* stage, int variant)
{
    if (!plan || !stage) return DWM_ERR_INVALID_ARG;
    const bool backward = !std::strcmp(stage, "backward");
    if (!backward && std::strcmp(stage, "forward")) return DWM_ERR_INVALID_ARG;
    if (backward && plan->ws) return DWM_ERR_WORKSPACE;
    const int v = variant < 0 ? rms_choice(plan->C) : variant;
    if (!rms_fits(v, plan->C)) return DWM_ERR_INVALID_ARG;
    (backward ? plan->backward : plan->forward) = v;
    plan->splits = rms_splits(plan->rows, plan->C, plan->backward);
    return DWM_OK;
}

size_t dwm_rms_workspace_bytes(const dwm_rms_plan_t* plan) { return plan ? (size_t)plan->splits * plan->C * sizeof(float) : 0; }

dwm_status_t dwm_rms_set_workspace(dwm_rms_plan_t* plan, void* ws_dev, size_t bytes)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    if (!ws_dev || !aligned(ws_dev, 256) || bytes < dwm_rms_workspace_bytes(plan)) return DWM_ERR_WORKSPACE;
    plan->ws = ws_dev;
    return DWM_OK;
}

static RmsArgs rms_args(const dwm_rms_plan& p)
{
    RmsArgs a{};
    std::memcpy(a.stride, p.stride, sizeof(a.stride));
    a.rows = p.rows;
    a.C = p.C;
    a.param_typed = p.param_type == p.type && p.type != DWM_F32;
    a.splits = p.splits;
    a.eps = p.eps;
    a.inverse = 1.0 / p.C;
    return a;
}

dwm_status_t dwm_rms_forward(const dwm_rms_plan_t* plan, const void* x_dev, const void* residual_dev, const void* gamma_dev, void* z_dev,
                             void* y_dev, const dwm_packed_t* y_packed, const dwm_packed_t* kept, float* rstd_dev, void* stream)
{
    if (!plan || (z_dev && !residual_dev) || !packed_ok(y_packed) || !packed_ok(kept)) return DWM_ERR_INVALID_ARG;
    if (plan->rows > 0 && (!x_dev || !(z_dev || y_dev || y_packed || kept || rstd_dev))) return DWM_ERR_INVALID_ARG;
    const size_t size = size_of(plan->type);
    if (!aligned(x_dev, size) || !aligned(residual_dev, size) || !aligned(z_dev, size) || !aligned(y_dev, size) ||
        !aligned(gamma_dev, size_of(plan->param_type)) || !aligned(rstd_dev, 4))
        return DWM_ERR_INVALID_ARG;
    if (plan->rows == 0) return DWM_OK;
    RmsArgs a = rms_args(*plan);
    a.x = x_dev;
    a.residual = residual_dev;
    a.gamma = gamma_dev;
    a.z = z_dev;
    a.y = y_dev;
    a.packed_y = packed_of(y_packed);
    a.kept = packed_of(kept);
    a.rstd = rstd_dev;
    return launch_rms_forward(a, plan->type, plan->forward, stream);
}

dwm_status_t dwm_rms_backward(const dwm_rms_plan_t* plan, const void* dy_dev, const void* dz_dev, const void* z_dev, const dwm_packed_t* kept,
                              const void* gamma_dev, const float* rstd_dev, void* dx_dev, void* dgamma_dev, void* stream)
{
    if (!plan || !packed_ok(kept) || (z_dev && kept) || (!dx_dev && !dgamma_dev)) return DWM_ERR_INVALID_ARG;
    if (plan->rows > 0 && (!dy_dev || !rstd_dev || !(z_dev || kept))) return DWM_ERR_INVALID_ARG;
    const size_t size = size_of(plan->type), param = size_of(plan->param_type);
    if (!aligned(dy_dev, size) || !aligned(dz_dev, size) || !aligned(z_dev, size) || !aligned(dx_dev, size) || !aligned(gamma_dev, param) ||
        !aligned(dgamma_dev, param) || !aligned(rstd_dev, 4))
        return DWM_ERR_INVALID_ARG;
    if (dgamma_dev && !plan->ws) return DWM_ERR_WORKSPACE;
    if (plan->rows == 0) return dgamma_dev ? launch_columns(nullptr, 0, plan->C, dgamma_dev, plan->param_type, stream) : DWM_OK;
    RmsArgs a = rms_args(*plan);
    a.dy = dy_dev;
    a.dz = dz_dev;
    a.z = const_cast<void*>(z_dev);
    a.kept = packed_of(kept);
    a.gamma = gamma_dev;
    a.rstd = const_cast<float*>(rstd_dev);
    a.dx = dx_dev;
    a.partial = dgamma_dev ? (float*)plan->ws : nullptr;
    const dwm_status_t st = launch_rms_backward(a, plan->type, plan->backward, stream);
    return st != DWM_OK || !dgamma_dev ? st : launch_columns(a.partial, plan->splits, plan->C, dgamma_dev, plan->param_type, stream);
}

dwm_status_t dwm_act_plan_create(dwm_act_plan_t** out, dwm_act_t act, long long rows, int C, dwm_type_t type, dwm_type_t param_type)
{
    if (!out || !known(act) || rows < 0 || C < 1 || !known(type) || !(param_type == DWM_F32 || param_type == type)) return DWM_ERR_INVALID_ARG;
    if (!rows_fit(rows, C)) return DWM_ERR_UNSUPPORTED;
    dwm_act_plan* p = new (std::nothrow) dwm_act_plan;
    if (!p) return DWM_ERR_ALLOC;
    std::memset(p, 0, sizeof(*p));
    p->rows = rows;
    p->C = C;
    p->type = type;
    p->param_type = param_type;
    p->act = act;
    for (long long& s : p->stride) s = C;
    p->splits = act_splits(rows, C);
    *out = p;
    return DWM_OK;
}

dwm_status_t dwm_act_plan_destroy(dwm_act_plan_t* plan)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    delete plan;
    return DWM_OK;
}

dwm_status_t dwm_act_set_stride(dwm_act_plan_t* plan, const char* tensor, long long stride)
{
    const int which = named(kActNames, tensor);
    if (!plan || which < 0 || stride < plan->C) return DWM_ERR_INVALID_ARG;
    if (plan->rows > 0 && stride > kMostElements / plan->rows) return DWM_ERR_UNSUPPORTED;
    plan->stride[which] = stride;
    return DWM_OK;
}

size_t dwm_act_workspace_bytes(const dwm_act_plan_t* plan) { return plan ? (size_t)plan->splits * plan->C * sizeof(float) : 0; }

dwm_status_t dwm_act_set_workspace(dwm_act_plan_t* plan, void* ws_dev, size_t bytes)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    if (!ws_dev || !aligned(ws_dev, 256) || bytes < dwm_act_workspace_bytes(plan)) return DWM_ERR_WORKSPACE;
    plan->ws = ws_dev;
    return DWM_OK;
}

static ActArgs act_args(const dwm_act_plan& p)
{
    ActArgs a{};
    std::memcpy(a.stride, p.stride, sizeof(a.stride));
    a.rows = p.rows;
    a.C = p.C;
    a.param_typed = p.param_type == p.type && p.type != DWM_F32;
    a.splits = p.splits;
    a.act = p.act;
    return a;
}

dwm_status_t dwm_act_forward(const dwm_act_plan_t* plan, const void* x_dev, const void* bias_dev, void* y_dev, const dwm_packed_t* kept, void* stream)
{
    if (!plan || !packed_ok(kept) || (plan->rows > 0 && (!x_dev || !(y_dev || kept)))) return DWM_ERR_INVALID_ARG;
    const size_t size = size_of(plan->type);
    if (!aligned(x_dev, size) || !aligned(y_dev, size) || !aligned(bias_dev, size_of(plan->param_type))) return DWM_ERR_INVALID_ARG;
    if (plan->rows == 0) return DWM_OK;
    ActArgs a = act_args(*plan);
    a.x = x_dev;
    a.bias = bias_dev;
    a.y = y_dev;
    a.kept = packed_of(kept);
    return launch_act_forward(a, plan->type, stream);
}

dwm_status_t dwm_act_backward(const dwm_act_plan_t* plan, const void* dy_dev, const void* x_dev, const void* bias_dev, const dwm_packed_t* kept,
                              void* dx_dev, void* dbias_dev, void* stream)
{
    if (!plan || !packed_ok(kept) || (kept && (x_dev || bias_dev)) || (bias_dev && !x_dev) || (!dx_dev && !dbias_dev)) return DWM_ERR_INVALID_ARG;
    if (plan->rows > 0 && (!dy_dev || !(x_dev || kept || plan->act == DWM_ACT_NONE))) return DWM_ERR_INVALID_ARG;
    const size_t size = size_of(plan->type), param = size_of(plan->param_type);
    if (!aligned(dy_dev, size) || !aligned(x_dev, size) || !aligned(dx_dev, size) || !aligned(bias_dev, param) || !aligned(dbias_dev, param))
        return DWM_ERR_INVALID_ARG;
    if (dbias_dev && !plan->ws) return DWM_ERR_WORKSPACE;
    if (plan->rows == 0) return dbias_dev ? launch_columns(nullptr, 0, plan->C, dbias_dev, plan->param_type, stream) : DWM_OK;
    ActArgs a = act_args(*plan);
    a.dy = dy_dev;
    if (plan->act != DWM_ACT_NONE) {  // (a derivative of one needs no p)
        a.x = x_dev;
        a.bias = bias_dev;
        a.kept = packed_of(kept);
    }
    a.dx = dx_dev;
    a.partial = dbias_dev ? (float*)plan->ws : nullptr;
    const dwm_status_t st = launch_act_backward(a, plan->type, stream);
    return st != DWM_OK || !dbias_dev ? st : launch_columns(a.partial, plan->splits, plan->C, dbias_dev, plan->param_type, stream);
}

dwm_status_t dwm_matmul_plan_create(dwm_matmul_plan_t** out, int M, int N, int K, dwm_type_t operands, dwm_type_t type, dwm_type_t param_type,
                                    dwm_act_t act, int flags)
{
    const int most = 1 << 24;
    if (!out || M < 0 || N < 0 || K < 0 || !known(act) || (flags & ~(DWM_A_ACROSS | DWM_B_ACROSS)) || !known(type) ||
        !(known(operands) || operands == DWM_PACKED) || !(param_type == DWM_F32 || param_type == (operands == DWM_PACKED ? type : operands)))
        return DWM_ERR_INVALID_ARG;
    if (operands == DWM_F32 || (operands == DWM_PACKED ? type == DWM_F32 || flags : type != DWM_F32 && type != operands)) return DWM_ERR_UNSUPPORTED;
    if (M > most || N > most || K > most || (long long)M * N > kMostElements >> 3) return DWM_ERR_UNSUPPORTED;
    if (operands == DWM_PACKED && (!rows_fit(M, K) || !rows_fit(N, K))) return DWM_ERR_UNSUPPORTED;  // (rows that dwm_pack does not make)
    dwm_matmul_plan* p = new (std::nothrow) dwm_matmul_plan;
    if (!p) return DWM_ERR_ALLOC;
    std::memset(p, 0, sizeof(*p));
    p->M = M;
    p->N = N;
    p->K = K;
    p->flags = flags;
    p->operands = operands;
    p->type = type;
    p->param_type = param_type;
    p->act = act;
    p->stride[kMatA] = flags & DWM_A_ACROSS ? M : K;
    p->stride[kMatB] = flags & DWM_B_ACROSS ? N : K;
    p->stride[kMatResidual] = p->stride[kMatOut] = N;
    p->asked_kernel = -1;
    matmul_plan(*p, -1, -1);
    *out = p;
    return DWM_OK;
}

dwm_status_t dwm_matmul_plan_destroy(dwm_matmul_plan_t* plan)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    delete plan;
    return DWM_OK;
}

dwm_status_t dwm_matmul_plan_info(const dwm_matmul_plan_t* plan, dwm_matmul_info_t* info)
{
    if (!plan || !info) return DWM_ERR_INVALID_ARG;
    *info = dwm_matmul_info_t{plan->M, plan->N, plan->K, plan->shape.kernel == kMatFewLoose ? (int)kMatFew : plan->shape.kernel, plan->shape.splits};
    return DWM_OK;
}

dwm_status_t dwm_matmul_set_stride(dwm_matmul_plan_t* plan, const char* tensor, long long stride)
{
    const int which = named(kMatNames, tensor);
    if (!plan || which < 0 || (plan->operands == DWM_PACKED && which <= kMatB)) return DWM_ERR_INVALID_ARG;
    const bool across = plan->flags & (which == kMatA ? DWM_A_ACROSS : which == kMatB ? DWM_B_ACROSS : 0);
    const long long own = which == kMatA ? plan->M : which == kMatB ? plan->N : plan->M;  // rows of a tensor whose rows run along K or N
    const long long rows = across ? plan->K : own, width = across ? own : which <= kMatB ? plan->K : plan->N;
    if (stride < width) return DWM_ERR_INVALID_ARG;
    if (rows > 0 && stride > kMostElements / rows) return DWM_ERR_UNSUPPORTED;
    plan->stride[which] = stride;
    return DWM_OK;
}

dwm_status_t dwm_matmul_set_variant(dwm_matmul_plan_t* plan, const char* stage, int variant)
{
    if (!plan || !stage) return DWM_ERR_INVALID_ARG;
    const bool kernel = !std::strcmp(stage, "kernel");
    if (!kernel && std::strcmp(stage, "splits")) return DWM_ERR_INVALID_ARG;
    if (plan->ws) return DWM_ERR_WORKSPACE;
    if (kernel) {
        if (variant >= 0 && !matmul_applies(*plan, variant)) return DWM_ERR_INVALID_ARG;
        const int asked = variant < 0 ? -1 : variant;
        if (!matmul_plan(*plan, asked, -1)) return DWM_ERR_INVALID_ARG;
        plan->asked_kernel = asked;
    } else {
        if (variant == 0 || variant > 64 || (variant > 1 && plan->asked_kernel == kMatFew)) return DWM_ERR_INVALID_ARG;
        if (!matmul_plan(*plan, plan->asked_kernel, variant)) return DWM_ERR_INVALID_ARG;
    }
    return DWM_OK;
}

size_t dwm_matmul_workspace_bytes(const dwm_matmul_plan_t* plan)
{
    return plan ? parts_bytes(*plan) + (plan->copies ? operand_rows(*plan, false).bytes() + operand_rows(*plan, true).bytes() : 0) : 0;
}

dwm_status_t dwm_matmul_set_workspace(dwm_matmul_plan_t* plan, void* ws_dev, size_t bytes)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    if (!ws_dev || !aligned(ws_dev, 256) || bytes < dwm_matmul_workspace_bytes(plan)) return DWM_ERR_WORKSPACE;
    plan->ws = ws_dev;
    return DWM_OK;
}

dwm_status_t dwm_matmul(const dwm_matmul_plan_t* plan, const void* a_dev, const void* b_dev, const void* bias_dev, const void* residual_dev,
                        void* out_dev, const dwm_packed_t* y_packed, const dwm_packed_t* kept, void* stream)
{
    if (!plan || plan->operands == DWM_PACKED) return DWM_ERR_INVALID_ARG;
    const bool some = plan->M > 0 && plan->N > 0;
    if ((some && plan->K > 0 && (!a_dev || !b_dev)) || !aligned(a_dev, 2) || !aligned(b_dev, 2)) return DWM_ERR_INVALID_ARG;
    const dwm_status_t ok = matmul_ok(*plan, bias_dev, residual_dev, out_dev, y_packed, kept);
    if (ok != DWM_OK) return ok;
    if (!some) return DWM_OK;
    MatmulArgs a{};
    a.a = a_dev;
    a.b = b_dev;
    long long strides[2] = {plan->stride[kMatA], plan->stride[kMatB]};
    const void* operands[2] = {a_dev, b_dev};
    if (plan->copies) {  // where the operand that needs no copy can be read as it lies
        bool good = true;
        for (int second = 0; second < 2; ++second) {
            const OperandRows r = operand_rows(*plan, second);
            good = good && (r.odd() || operand_aligned(operands[second], strides[second], r.length));
        }
        if (good) {
            if (!plan->ws) return DWM_ERR_WORKSPACE;
            char* to = (char*)plan->ws + parts_bytes(*plan);
            AlignedRows rows[2];
            int count = 0;
            for (int second = 0; second < 2; ++second) {
                const OperandRows r = operand_rows(*plan, second);
                if (!r.odd()) continue;
                rows[count++] = {operands[second], strides[second], to, r.stride(), r.rows, (int)r.length};
                operands[second] = to;
                strides[second] = r.stride();
                to += r.bytes();
            }
            const dwm_status_t st = launch_aligned_rows(rows, count, stream);
            if (st != DWM_OK) return st;
            a.a = operands[0];
            a.b = operands[1];
            return run_matmul(*plan, a, plan->shape, strides, bias_dev, residual_dev, out_dev, y_packed, kept, stream);
        }
    }
    const bool fast = plan->K == 0 || (operand_aligned(a_dev, strides[0], operand_rows(*plan, false).length) && operand_aligned(b_dev, strides[1], operand_rows(*plan, true).length));
    return run_matmul(*plan, a, fast ? plan->shape : plan->any, strides, bias_dev, residual_dev, out_dev, y_packed, kept, stream);
}

dwm_status_t dwm_matmul_packed(const dwm_matmul_plan_t* plan, const dwm_packed_t* a, const dwm_packed_t* b, const void* bias_dev,
                               const void* residual_dev, void* out_dev, const dwm_packed_t* y_packed, const dwm_packed_t* kept, void* stream)
{
    if (!plan || plan->operands != DWM_PACKED || !packed_ok(a) || !packed_ok(b)) return DWM_ERR_INVALID_ARG;
    const bool some = plan->M > 0 && plan->N > 0;
    if (some && plan->K > 0 && (!a || !b)) return DWM_ERR_INVALID_ARG;
    const dwm_status_t ok = matmul_ok(*plan, bias_dev, residual_dev, out_dev, y_packed, kept);
    if (ok != DWM_OK) return ok;
    if (!some) return DWM_OK;
    MatmulArgs args{};
    if (a && b) {
        args.a = a->codes;
        args.a_scales = (const uint8_t*)a->scales;
        args.b = b->codes;
        args.b_scales = (const uint8_t*)b->scales;
    }
    return run_matmul(*plan, args, plan->shape, plan->stride, bias_dev, residual_dev, out_dev, y_packed, kept, stream);
}

}  // extern "C"

// Layer norms, dropouts and joins of residual branches: plans, checks of arguments and entry points (host only, plain C++).
#include "norm.hpp"

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>

namespace dwm {

static int workgroups(long long v, int most) { return v < 1 ? 1 : v < most ? (int)v : most; }

// norm_any.hip: splits of the positions for the parameters' gradients, enough for the chip, none without some work.
static NormShape any_shape(long long positions, int C, bool rows)
{
    const long long groups = rows ? (C + 63) / 64 : C, threads = rows ? 4 : 256;
    long long splits = (positions + 16 * threads - 1) / (16 * threads);
    if (splits * groups > 4096) splits = 4096 / groups;
    return {kNormAny, workgroups(splits, 256), false};
}

// Whether a shape can hold the norms of a plan.
static bool rows_fit(int shape, int C, int vec, bool backward)
{
    if (shape < 0 || shape >= kNormRowsShapes) return false;
    const NormRows& r = kNormRows[shape];
    const int holds = r.tpr * r.k * vec;
    return holds >= C && C >= vec && (backward ? r.backward && holds <= kNormRowsWidest : r.forward);
}
static bool maps_fit(int shape, int C, int size, bool one, NormStage stage)
{
    if (shape < 0 || shape >= kNormMapsShapes) return false;
    const NormMaps& m = kNormMaps[shape];
    return m.cg * m.k >= C && (!one || m.one) && (stage != kNormJoinForward || size <= m.join) && (stage != kNormBackward || size <= m.backward);
}
static long long maps_tiles(int shape, long long vectors) { return (vectors + kNormMaps[shape].pl - 1) / kNormMaps[shape].pl; }

// Rows, forward: the narrowest shape; below 2048 rows those with one vector a thread, a shorter way from the first load to the last store
// (2048 rows of 4096 bfloat16: 9.4 us with two vectors, 9.9 with one; 256 rows of 2048: 3.8 and 3.6).  Backward: one vector a
// thread wherever there is a shape for it (4096 rows of 1500 bfloat16: 21.7 us with two, 17.5 with one; 65536 of 1024: 83 and 81; 16384 of 2048: 44
// both).
// Forward, 16385 to 32768 channels of 16 bits: the shape that holds them spills registers, and is taken for a row on each CU (two of a bfloat16 norm's, four
// of a binary16 one's: it spills least); with more rows the kernel for any size, which reads them again, is ahead.  us, in registers and any size, rows of 24576,
// parameters in binary32: joins of 256 rows 40, 52, of 320 71, 61, of 2000 292, 178; norms in bfloat16 of 512 rows 35, 36, of 1024 62, 46; in binary16
// of 1024 44, 47, of 4000 170, 156.
static long long spilling_rows(dwm_type_t type, NormStage stage) { return stage == kNormJoinForward ? 256 : type == DWM_BF16 ? 512 : 1024; }
static int rows_choice(long long outer, int C, dwm_type_t type, NormStage stage)
{
    const bool backward = stage == kNormBackward;
    const int vec = type == DWM_F32 ? 4 : 8;
    if (C > kNormRowsWidest && outer > spilling_rows(type, stage)) return -1;
    for (int pass = backward || outer < 2048 ? 0 : 1; pass < 2; ++pass)
        for (int i = 0; i < kNormRowsShapes; ++i)
            if (rows_fit(i, C, vec, backward) && (pass == 1 || kNormRows[i].k == 1)) return i;
    return -1;
}

// Maps: four channels a thread, so that a tile is small and many are under way, or, where wider tiles (six or eight channels a thread, whose lanes lie
// along more pixels) are still enough for the chip, those.  us, four and wide, forward: 64 images of 1024 channels, 14 x 14, binary32: 35.5,
// 31.8; of 7 x 7: 13.3, 15.7; 8 images of 512, 20 x 20, binary16: 6.1, 7.0; 64 of 300: 15.3, 13.2; 64 of 96, 55 x 55, bfloat16: 26.6, 23.2; 8 of them:
// 6.3, 6.8.  Tiles of 1024 threads have to be twice as many (300 images of 700, 5 x 5, binary32: 20.7, 22.6).  Over 129 to 256 channels and over 17 to
// 32 they always pay (32 images of 192, 28 x 28, bfloat16: 9.7, 8.1; 64 of 32, 112 x 112, binary32: 48, 44).
// Backward in binary32 wide tiles do not pay (64 images of 256, 28 x 28: 39.4, 45.9), with 16 bits from twice the size on (64 of 96, 55 x 55: 40.2,
// 35.4; 64 of 300, 20 x 20, a join: 35.4, 33.1; of 128, 28 x 28: 17.9, 18.8).
// A join holds the residual and the draws too.  With 16 bits wide tiles pay as for a norm (64 images of 300, 20 x 20: 25.1, 23.6; of 512, 14 x 14: 23.2, 22.0;
// of 1024: 46.4, 38.7), but not with eight channels over 193 to 256 (16 of 256, 14 x 14: 7.6, 8.7; 64 of them, 28 x 28: 29.9, 31.7: not built); in binary32 with six,
// or eight up to 128, from three times the size on (10 of 259, 88 x 82: 74.2, 70.9; 64 of 300, 20 x 20: 34.2, 35.3; 64 of 96, 55 x 55: 78.8, 73.8;
// of 128, 28 x 28: 24.9, 28.1), else not (64 of 1024, 14 x 14: 67.4, 74.7: not built).
static int maps_choice(int C, int size, long long vectors, bool one, NormStage stage)
{
    const bool backward = stage == kNormBackward, join = stage == kNormJoinForward;
    int four = -1, wide = -1;
    for (int i = kNormMapsShapes - 1; i >= 0; --i)
        if (maps_fit(i, C, size, one, stage)) (kNormMaps[i].k == 4 ? four : wide) = i;
    if (four < 0 || wide < 0) return four < 0 ? wide : four;
    const NormMaps &m = kNormMaps[wide], &n = kNormMaps[four];
    if (m.cg == 4) return C > 16 ? wide : four;
    if (m.cg * m.k > n.cg * n.k) return four;  // (made for more channels)
    const long long threads = maps_tiles(wide, vectors) * m.pl * m.cg, enough = 256 * 768;
    return (m.cg == 32 && C > 128 && !join) || threads >= (backward || m.cg == 128 ? 2 : join && size == 4 ? 3 : 1) * enough ? wide : four;
}

// How many workgroups: forward, enough to fill the chip several times over; backward over maps, two for each of the 256 CUs, since each writes its
// sums of the parameters' gradients (32 images of 256 channels, 28 x 28, binary32: 256 workgroups 29.9 us, 512 24.4, 1024 25.2).
// The parameters' gradients are made aside up to 1024 rows or 4096 pixels and 8 MB (777 rows of 1021 binary32: 7.6 us against 10.3; 1024 rows of 4096
// bfloat16 17.2 and 18.8; 2048 rows of 1021 14.9 and 13.9; 16 maps of 256 channels, 14 x 14: 7.8 and 10.7, 32 maps 11.4 and 11.9).
constexpr int kForwardBlocks = 4096, kMapsBackwardBlocks = 512;

NormShape norm_choose(long long outer, int C, long long inner, dwm_type_t type, NormStage stage, int variant)
{
    const bool backward = stage == kNormBackward;
    const long long positions = outer * inner;
    const NormShape any = any_shape(positions, C, inner == 1), none{-1, 0, false};
    if (variant == kNormAny || (variant < 0 && positions == 0)) return any;
    const int size = type == DWM_F32 ? 4 : 2;
    const bool small = positions * C * size <= 8 << 20;
    // (rows shorter than a vector are taken as maps of one pixel)
    if (inner == 1 && (variant < 0 ? C >= 16 / size : variant < kNormMapsVec)) {
        const int vec = 16 / size, shape = variant < 0 ? rows_choice(outer, C, type, stage) : variant - kNormRowsFirst;
        if (!rows_fit(shape, C, vec, backward)) return variant < 0 ? any : none;
        const int tpr = kNormRows[shape].tpr, threads = backward ? norm_rows_threads(kNormRows[shape], C % vec != 0) : tpr > 256 ? tpr : 256;
        const long long blocks = (outer + threads / tpr - 1) / (threads / tpr);
        return {kNormRowsFirst + shape, workgroups(blocks, backward ? norm_rows_blocks(threads) : kForwardBlocks), small && outer <= 1024};
    }
    // One pixel a lane where there are fewer than four, and up to 2^20 elements, where four leave CUs without work (one image of 256 channels, 28 x 28,
    // bfloat16, forward: 4.2 us against 7.2; 8 images 5.5 both; 64 of 14 x 14 9.6 against 7.7).
    const bool one = variant < 0 ? inner < kNormMapsPixels || positions * C <= 1 << 20 : variant >= kNormMapsOne;
    const long long vectors = one ? positions : outer * ((inner + kNormMapsPixels - 1) / kNormMapsPixels), limit = (1LL << 31) - 64;  // (indexes in 32 bits)
    const int shape = variant < 0 ? maps_choice(C, size, vectors, one, stage) : variant - (one ? kNormMapsOne : kNormMapsVec);
    if (!maps_fit(shape, C, size, one, stage) || !(one || inner >= kNormMapsPixels) || vectors >= limit || inner >= limit)
        return variant < 0 ? any : none;
    return {(one ? kNormMapsOne : kNormMapsVec) + shape, workgroups(maps_tiles(shape, vectors), backward ? kMapsBackwardBlocks : kForwardBlocks), small && positions <= 4096};
}

static const char* const kTensorNames[kNormTensors] = {"x", "residual", "z", "y", "dy", "dz", "dx", "dresidual"};

static size_t size_of(dwm_type_t type) { return type == DWM_F32 ? 4 : 2; }
static bool known(dwm_type_t type) { return type == DWM_F32 || type == DWM_F16 || type == DWM_BF16; }
static bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// The largest tensor, in elements: kernels count in 64 bits, and a byte offset stays far from their end.
constexpr long long kMostElements = 1LL << 40;

static bool drop_args(const dwm_dropout_t* drop, DropArgs* out)
{
    *out = DropArgs{};
    out->scale = 1.0f;
    if (!drop) return true;
    if (!(drop->p >= 0.0 && drop->p <= 1.0) || !aligned(drop->sequence_dev, 8)) return false;
    const double limit = std::nearbyint(drop->p * 4294967296.0);
    out->mode = drop->p == 0.0 ? kDropNone : limit >= 4294967296.0 ? kDropAll : kDropDraw;
    out->threshold = out->mode == kDropDraw ? (uint32_t)limit : 0;
    out->scale = out->mode == kDropAll ? 0.0f : (float)(1.0 / (1.0 - drop->p));
    out->seed_lo = (uint32_t)drop->seed;
    out->seed_hi = (uint32_t)(drop->seed >> 32);
    out->sequence = drop->sequence;
    out->sequence_dev = drop->sequence_dev;
    return true;
}

static NormArgs args_of(const dwm_norm_plan& p)
{
    NormArgs a{};
    std::memcpy(a.stride, p.stride, sizeof(a.stride));
    a.outer = p.outer;
    a.inner = p.inner;
    a.C = p.C;
    a.param_typed = p.param_type == p.type && p.type != DWM_F32;
    a.splits = p.shape[kNormBackward].blocks;
    a.eps = p.eps;
    a.partial = (float*)p.ws;
    a.drop.scale = 1.0f;
    return a;
}

// Whether tensors that a call cannot do without are there; without a single element none is needed.
static bool given(const dwm_norm_plan& p, std::initializer_list<const void*> tensors)
{
    for (const void* t : tensors)
        if (!t && p.outer > 0) return false;
    return true;
}
// Whether what is given lies at multiples of its element's size.
static bool tensors_ok(const dwm_norm_plan& p, std::initializer_list<const void*> tensors)
{
    for (const void* t : tensors)
        if (!aligned(t, size_of(p.type))) return false;
    return true;
}
static bool params_ok(const dwm_norm_plan& p, std::initializer_list<const void*> params)
{
    for (const void* t : params)
        if (!aligned(t, size_of(p.param_type))) return false;
    return true;
}
static bool stats_ok(const void* mean, const void* rstd) { return aligned(mean, 4) && aligned(rstd, 4); }

static dwm_status_t run_kernel(const dwm_norm_plan& p, const NormArgs& a, const NormShape& shape, bool backward, bool join, void* stream)
{
    switch (p.type) {
        case DWM_F32: return launch_norm_f32(a, shape, backward, join, stream);
        case DWM_F16: return launch_norm_f16(a, shape, backward, join, stream);
        case DWM_BF16: return launch_norm_bf16(a, shape, backward, join, stream);
    }
    return DWM_ERR_INVALID_ARG;
}

static dwm_status_t run_forward(const dwm_norm_plan& p, const NormArgs& a, bool join, void* stream)
{
    if (p.outer == 0) return DWM_OK;
    const NormShape& shape = p.shape[join ? kNormJoinForward : kNormForward];
    return shape.kernel == kNormAny ? launch_norm_any_forward(a, p.type, join, stream) : run_kernel(p, a, shape, false, join, stream);
}

static dwm_status_t run_backward(const dwm_norm_plan& p, const NormArgs& a, bool join, void* stream)
{
    const bool params = a.dgamma || a.dbeta;
    if (params && !p.ws) return DWM_ERR_WORKSPACE;
    if (p.shape[kNormBackward].kernel == kNormAny) return launch_norm_any_backward(a, p.type, stream);
    NormArgs b = a;
    if (!params || p.shape[kNormBackward].aside) b.partial = nullptr;
    if (params && p.shape[kNormBackward].aside) {
        b.aside = 1;
        if (!a.dx && !a.dresidual) {  // nothing else to make
            b.splits = 0;
        } else if (a.dy == a.dx || a.dy == a.dresidual) {  // dy would be overwritten while it is read: the parameters' gradients first
            b.splits = 0;
            const dwm_status_t st = run_kernel(p, b, p.shape[kNormBackward], true, join, stream);
            if (st != DWM_OK) return st;
            b.splits = a.splits;
            b.aside = 0;
        }
    }
    const dwm_status_t st = run_kernel(p, b, p.shape[kNormBackward], true, join, stream);
    return st != DWM_OK || !b.partial ? st : launch_norm_params_final(a, p.type, stream);
}

}  // namespace dwm

extern "C" {

dwm_status_t dwm_norm_plan_create(dwm_norm_plan_t** out, long long outer, int C, long long inner, dwm_type_t type,
                                  dwm_type_t param_type, double eps)
{
    using namespace dwm;
    if (!out || outer < 0 || C < 1 || inner < 1 || !known(type) || !(param_type == DWM_F32 || param_type == type) ||
        !(eps >= 0.0) || !(eps <= 3e38))
        return DWM_ERR_INVALID_ARG;
    if (C > (1 << 20) || inner > kMostElements / C || outer > kMostElements / (C * inner)) return DWM_ERR_UNSUPPORTED;
    dwm_norm_plan* p = new (std::nothrow) dwm_norm_plan;
    if (!p) return DWM_ERR_ALLOC;
    std::memset(p, 0, sizeof(*p));
    p->outer = outer;
    p->C = C;
    p->inner = inner;
    p->type = type;
    p->param_type = param_type;
    p->eps = (float)eps;
    for (long long& s : p->stride) s = C * inner;
    for (int s = 0; s < kNormStages; ++s) p->shape[s] = norm_choose(outer, C, inner, type, (NormStage)s, -1);
    *out = p;
    return DWM_OK;
}

dwm_status_t dwm_norm_plan_destroy(dwm_norm_plan_t* plan)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    delete plan;
    return DWM_OK;
}

dwm_status_t dwm_norm_set_stride(dwm_norm_plan_t* plan, const char* tensor, long long stride)
{
    using namespace dwm;
    if (!plan || !tensor || stride < plan->C * plan->inner) return DWM_ERR_INVALID_ARG;
    int which = 0;
    while (which < kNormTensors && std::strcmp(tensor, kTensorNames[which])) ++which;
    if (which == kNormTensors) return DWM_ERR_INVALID_ARG;
    if (plan->outer > 0 && stride > kMostElements / plan->outer) return DWM_ERR_UNSUPPORTED;
    plan->stride[which] = stride;
    return DWM_OK;
}

dwm_status_t dwm_norm_set_variant(dwm_norm_plan_t* plan, const char* stage, int variant)
{
    using namespace dwm;
    if (!plan || !stage) return DWM_ERR_INVALID_ARG;
    const bool backward = !std::strcmp(stage, "backward");
    if (!backward && std::strcmp(stage, "forward")) return DWM_ERR_INVALID_ARG;
    if (backward && plan->ws) return DWM_ERR_WORKSPACE;
    const int from = backward ? kNormBackward : kNormForward, to = backward ? kNormStages : kNormBackward;
    NormShape asked[kNormStages];
    for (int s = from; s < to; ++s) {
        asked[s] = norm_choose(plan->outer, plan->C, plan->inner, plan->type, (NormStage)s, variant);
        if (s == kNormJoinForward && asked[s].kernel < 0)  // (a shape of the plain norm alone)
            asked[s] = norm_choose(plan->outer, plan->C, plan->inner, plan->type, kNormJoinForward, -1);
        if (asked[s].kernel < 0) return DWM_ERR_INVALID_ARG;
    }
    std::memcpy(plan->shape + from, asked + from, (to - from) * sizeof(NormShape));
    return DWM_OK;
}

dwm_status_t dwm_norm_plan_info(const dwm_norm_plan_t* plan, dwm_norm_info_t* info)
{
    if (!plan || !info) return DWM_ERR_INVALID_ARG;
    info->outer = plan->outer;
    info->C = plan->C;
    info->inner = plan->inner;
    info->forward_kernel = plan->shape[dwm::kNormForward].kernel;
    info->join_forward_kernel = plan->shape[dwm::kNormJoinForward].kernel;
    info->backward_kernel = plan->shape[dwm::kNormBackward].kernel;
    info->splits = plan->shape[dwm::kNormBackward].blocks;
    return DWM_OK;
}

size_t dwm_norm_workspace_bytes(const dwm_norm_plan_t* plan)
{
    return plan ? (size_t)plan->shape[dwm::kNormBackward].blocks * 2 * plan->C * sizeof(float) : 0;
}

dwm_status_t dwm_norm_set_workspace(dwm_norm_plan_t* plan, void* ws_dev, size_t bytes)
{
    if (!plan) return DWM_ERR_INVALID_ARG;
    if (!ws_dev || !dwm::aligned(ws_dev, 256) || bytes < dwm_norm_workspace_bytes(plan)) return DWM_ERR_WORKSPACE;
    plan->ws = ws_dev;
    return DWM_OK;
}

dwm_status_t dwm_norm_forward(const dwm_norm_plan_t* plan, const void* x_dev, const void* gamma_dev, const void* beta_dev,
                              void* y_dev, float* mean_dev, float* rstd_dev, void* stream)
{
    using namespace dwm;
    if (!plan || !given(*plan, {x_dev, y_dev})) return DWM_ERR_INVALID_ARG;
    if (!tensors_ok(*plan, {x_dev, y_dev}) || !params_ok(*plan, {gamma_dev, beta_dev}) || !stats_ok(mean_dev, rstd_dev))
        return DWM_ERR_INVALID_ARG;
    NormArgs a = args_of(*plan);
    a.x = x_dev;
    a.gamma = gamma_dev;
    a.beta = beta_dev;
    a.y = y_dev;
    a.mean = mean_dev;
    a.rstd = rstd_dev;
    return run_forward(*plan, a, false, stream);
}

dwm_status_t dwm_norm_backward(const dwm_norm_plan_t* plan, const void* dy_dev, const void* x_dev, const void* gamma_dev,
                               const float* mean_dev, const float* rstd_dev, void* dx_dev, void* dgamma_dev, void* dbeta_dev,
                               void* stream)
{
    using namespace dwm;
    if (!plan || !given(*plan, {dy_dev, x_dev, mean_dev, rstd_dev}) || (plan->outer > 0 && !dx_dev && !dgamma_dev && !dbeta_dev))
        return DWM_ERR_INVALID_ARG;
    if (!tensors_ok(*plan, {dy_dev, x_dev, dx_dev}) || !params_ok(*plan, {gamma_dev, dgamma_dev, dbeta_dev}) ||
        !stats_ok(mean_dev, rstd_dev))
        return DWM_ERR_INVALID_ARG;
    NormArgs a = args_of(*plan);
    a.dy = dy_dev;
    a.z = const_cast<void*>(x_dev);
    a.stride[kNormZ] = plan->stride[kNormX];
    a.gamma = gamma_dev;
    a.mean = const_cast<float*>(mean_dev);
    a.rstd = const_cast<float*>(rstd_dev);
    a.dresidual = dx_dev;
    a.stride[kNormDresidual] = plan->stride[kNormDx];
    a.dgamma = dgamma_dev;
    a.dbeta = dbeta_dev;
    return run_backward(*plan, a, false, stream);
}

dwm_status_t dwm_norm_join_forward(const dwm_norm_plan_t* plan, const dwm_dropout_t* drop, const void* x_dev,
                                   const void* residual_dev, const void* gamma_dev, const void* beta_dev, void* z_dev,
                                   void* y_dev, float* mean_dev, float* rstd_dev, void* stream)
{
    using namespace dwm;
    if (!plan || !given(*plan, {x_dev, residual_dev, z_dev, y_dev})) return DWM_ERR_INVALID_ARG;
    if (!tensors_ok(*plan, {x_dev, residual_dev, z_dev, y_dev}) || !params_ok(*plan, {gamma_dev, beta_dev}) ||
        !stats_ok(mean_dev, rstd_dev))
        return DWM_ERR_INVALID_ARG;
    NormArgs a = args_of(*plan);
    if (!drop_args(drop, &a.drop)) return DWM_ERR_INVALID_ARG;
    a.x = x_dev;
    a.residual = residual_dev;
    a.gamma = gamma_dev;
    a.beta = beta_dev;
    a.z = z_dev;
    a.y = y_dev;
    a.mean = mean_dev;
    a.rstd = rstd_dev;
    return run_forward(*plan, a, true, stream);
}

dwm_status_t dwm_norm_join_backward(const dwm_norm_plan_t* plan, const dwm_dropout_t* drop, const void* dy_dev,
                                    const void* dz_dev, const void* z_dev, const void* gamma_dev, const float* mean_dev,
                                    const float* rstd_dev, void* dx_dev, void* dresidual_dev, void* dgamma_dev, void* dbeta_dev,
                                    void* stream)
{
    using namespace dwm;
    if (!plan || !given(*plan, {dy_dev, z_dev, mean_dev, rstd_dev}) ||
        (plan->outer > 0 && !dx_dev && !dresidual_dev && !dgamma_dev && !dbeta_dev))
        return DWM_ERR_INVALID_ARG;
    if (!tensors_ok(*plan, {dy_dev, dz_dev, z_dev, dx_dev, dresidual_dev}) ||
        !params_ok(*plan, {gamma_dev, dgamma_dev, dbeta_dev}) || !stats_ok(mean_dev, rstd_dev))
        return DWM_ERR_INVALID_ARG;
    NormArgs a = args_of(*plan);
    if (!drop_args(drop, &a.drop)) return DWM_ERR_INVALID_ARG;
    a.dy = dy_dev;
    a.dz = dz_dev;
    a.z = const_cast<void*>(z_dev);
    a.gamma = gamma_dev;
    a.mean = const_cast<float*>(mean_dev);
    a.rstd = const_cast<float*>(rstd_dev);
    a.dx = dx_dev;
    a.dresidual = dresidual_dev;
    a.dgamma = dgamma_dev;
    a.dbeta = dbeta_dev;
    return run_backward(*plan, a, true, stream);
}

dwm_status_t dwm_dropout_forward(const dwm_dropout_t* drop, dwm_type_t type, long long n, const void* x_dev, void* y_dev,
                                 void* stream)
{
    using namespace dwm;
    DropArgs d;
    if (!drop || !known(type) || n < 0 || (n > 0 && (!x_dev || !y_dev)) || !drop_args(drop, &d)) return DWM_ERR_INVALID_ARG;
    if (!aligned(x_dev, size_of(type)) || !aligned(y_dev, size_of(type))) return DWM_ERR_INVALID_ARG;
    if (n > kMostElements) return DWM_ERR_UNSUPPORTED;
    return n == 0 ? DWM_OK : launch_dropout(d, type, n, x_dev, y_dev, stream);
}

dwm_status_t dwm_dropout_backward(const dwm_dropout_t* drop, dwm_type_t type, long long n, const void* dy_dev, void* dx_dev,
                                  void* stream)
{
    return dwm_dropout_forward(drop, type, n, dy_dev, dx_dev, stream);  // the same mask and scale, on the gradient
}

}  // extern "C"

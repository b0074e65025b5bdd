// Layer norms, dropouts and joins of residual branches: plans, checks of arguments and entry points (host only, plain C++).
#include "norm.hpp"

#include <cmath>
#include <cstring>
#include <initializer_list>
#include <new>

namespace dwm {

static NormShape any_shape(long long positions, int C, bool rows)
{
    const long long groups = rows ? (C + 63) / 64 : C, threads = rows ? 4 : 256;
    long long splits = (positions + 16 * threads - 1) / (16 * threads);
    if (splits * groups > 4096) splits = 4096 / groups;
    return {kNormAny, (int)(splits < 1 ? 1 : splits > 256 ? 256 : splits)};
}

static long long at_most(long long v, long long most) { return v < most ? v : most; }

NormShape norm_choose(long long outer, int C, long long inner, dwm_type_t type, bool backward, int variant)
{
    const long long positions = outer * inner;
    const int vec = type == DWM_F32 ? 4 : 8;
    const NormShape any = any_shape(positions, C, inner == 1), none{-1, 0};
    if (variant == kNormAny || (variant < 0 && positions == 0)) return any;
    if (inner == 1) {
        int shape = variant - kNormRowsFirst;
        if (variant < 0)
            for (shape = 0; shape < kNormRowsShapes && kNormRows[shape].tpr * kNormRows[shape].k * vec < C;) ++shape;
        const bool ok = shape >= 0 && shape < kNormRowsShapes && kNormRows[shape].tpr * kNormRows[shape].k * vec >= C && C >= vec;
        if (!ok) return variant < 0 ? any : none;
        const int tpr = kNormRows[shape].tpr, smallest = backward ? kNormRowsBackwardThreads : 256;
        const int rows = (tpr > smallest ? tpr : smallest) / tpr;
        const long long blocks = (outer + rows - 1) / rows;
        return {kNormRowsFirst + shape, (int)at_most(blocks, backward ? 512 : 2048)};
    }
    bool one = variant < 0 ? inner < vec : variant >= kNormMapsOne;
    int shape = variant - (one ? kNormMapsOne : kNormMapsVec);
    if (variant < 0)
        for (shape = 0; shape < kNormMapsShapes && kNormMaps[shape].cg * kNormMaps[shape].k < C;) ++shape;
    const long long vectors = one ? positions : outer * ((inner + vec - 1) / vec), limit = (1LL << 31) - 1;
    const bool ok = shape >= 0 && shape < kNormMapsShapes && kNormMaps[shape].cg * kNormMaps[shape].k >= C && (one || inner >= vec) &&
                    vectors < limit && inner < limit;
    if (!ok) return variant < 0 ? any : none;
    const long long tiles = (vectors + kNormMaps[shape].pl - 1) / kNormMaps[shape].pl;
    return {(one ? kNormMapsOne : kNormMapsVec) + shape, (int)at_most(tiles, backward ? 512 : 4096)};
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

static NormArgs args_of(const dwm_norm_plan& p, const NormShape& shape)
{
    NormArgs a{};
    std::memcpy(a.stride, p.stride, sizeof(a.stride));
    a.outer = p.outer;
    a.inner = p.inner;
    a.C = p.C;
    a.param_typed = p.param_type == p.type && p.type != DWM_F32;
    a.splits = shape.blocks;
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
    return p.forward.kernel == kNormAny ? launch_norm_any_forward(a, p.type, join, stream) : run_kernel(p, a, p.forward, false, join, stream);
}

static dwm_status_t run_backward(const dwm_norm_plan& p, const NormArgs& a, void* stream)
{
    const bool params = a.dgamma || a.dbeta;
    if (params && !p.ws) return DWM_ERR_WORKSPACE;
    if (p.backward.kernel == kNormAny) return launch_norm_any_backward(a, p.type, stream);
    const dwm_status_t st = run_kernel(p, a, p.backward, true, false, stream);
    return st != DWM_OK || !params ? st : launch_norm_params_final(a, p.type, stream);
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
    p->forward = norm_choose(outer, C, inner, type, false, -1);
    p->backward = norm_choose(outer, C, inner, type, true, -1);
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
    const NormShape s = norm_choose(plan->outer, plan->C, plan->inner, plan->type, backward, variant);
    if (s.kernel < 0) return DWM_ERR_INVALID_ARG;
    (backward ? plan->backward : plan->forward) = s;
    return DWM_OK;
}

dwm_status_t dwm_norm_plan_info(const dwm_norm_plan_t* plan, dwm_norm_info_t* info)
{
    if (!plan || !info) return DWM_ERR_INVALID_ARG;
    info->outer = plan->outer;
    info->C = plan->C;
    info->inner = plan->inner;
    info->forward_kernel = plan->forward.kernel;
    info->backward_kernel = plan->backward.kernel;
    info->splits = plan->backward.blocks;
    return DWM_OK;
}

size_t dwm_norm_workspace_bytes(const dwm_norm_plan_t* plan)
{
    return plan ? (size_t)plan->backward.blocks * 2 * plan->C * sizeof(float) : 0;
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
    NormArgs a = args_of(*plan, plan->forward);
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
    NormArgs a = args_of(*plan, plan->backward);
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
    return run_backward(*plan, a, stream);
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
    NormArgs a = args_of(*plan, plan->forward);
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
    NormArgs a = args_of(*plan, plan->backward);
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
    return run_backward(*plan, a, stream);
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

// Shape fuzz of the plans and entry points over rows (branch.cpp) with the launchers stubbed: what a kernel takes for granted about
// its arguments is checked where it would be launched.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../../paper_2002_00552_amd/csrc/branch.hpp"

static long long launches = 0;

static void require(bool ok, const char* what)
{
    if (ok) return;
    std::printf("ERROR: %s\n", what);
    std::exit(1);
}

namespace dwm {

dwm_status_t launch_rms_forward(const RmsArgs& a, dwm_type_t, int kernel, void*)
{
    ++launches;
    require(a.rows > 0 && a.C > 0 && a.x, "rms forward without rows");
    require(kernel == 0 || (kernel <= kRmsShapeCount && kRmsShapes[kernel - 1].forward && kRmsShapes[kernel - 1].tpr * kRmsShapes[kernel - 1].k * kOctet >= a.C), "rms forward shape");
    return DWM_OK;
}
dwm_status_t launch_rms_backward(const RmsArgs& a, dwm_type_t, int kernel, void*)
{
    ++launches;
    require(kernel == 0 || (kernel <= kRmsShapeCount && kRmsShapes[kernel - 1].backward && kRmsShapes[kernel - 1].tpr * kRmsShapes[kernel - 1].k * kOctet >= a.C), "rms backward shape");
    require(a.splits >= 1 && (a.dx || a.partial) && (a.z || a.kept.codes), "rms backward arguments");
    if (kernel == 0) require((long long)((a.C + 2047) / 2048) * a.splits * 256 < 1LL << 32 && a.splits < 65536, "rms backward grid");
    return DWM_OK;
}
dwm_status_t launch_act_forward(const ActArgs& a, dwm_type_t, void*)
{
    ++launches;
    require(a.rows > 0 && (a.x ? a.y || a.kept.codes : a.y && a.kept.codes), "act forward arguments");
    return DWM_OK;
}
dwm_status_t launch_act_backward(const ActArgs& a, dwm_type_t, void*)
{
    ++launches;
    require(a.rows > 0 && a.dy && (a.dx || a.partial), "act backward arguments");
    require(a.splits >= 1 && a.splits < 65536 && (long long)((a.C + 2047) / 2048) * a.splits * 256 < 1LL << 32, "act backward grid");
    return DWM_OK;
}
dwm_status_t launch_columns(const float* partial, int splits, int C, void* out, dwm_type_t, void*)
{
    ++launches;
    require(out && C > 0 && (splits == 0 || partial), "columns");
    return DWM_OK;
}

static uintptr_t copies_from = 0, copies_to = 0;  // the workspace that copies have to stay in

dwm_status_t launch_aligned_rows(const AlignedRows* r, int count, void*)
{
    ++launches;
    require(count == 1 || count == 2, "operands to copy");
    for (int i = 0; i < count; ++i) {
        const uintptr_t to = (uintptr_t)r[i].to, end = to + r[i].rows * r[i].to_stride * 2;
        require(r[i].from && r[i].rows > 0 && r[i].width > 0 && r[i].stride >= r[i].width, "rows to copy");
        require(r[i].to_stride >= r[i].width && r[i].to_stride < r[i].width + 8 && r[i].to_stride % 8 == 0, "rows of a copy");
        require(to % 256 == 0 && to >= copies_from && end <= copies_to, "copies outside the workspace");
        if (i) require(to >= (uintptr_t)r[0].to + r[0].rows * r[0].to_stride * 2, "copies over each other");
    }
    return DWM_OK;
}

static dwm_status_t matmul(const MatmulArgs& a, int flags, int kernel, bool packed)
{
    ++launches;
    require(a.M > 0 && a.N > 0 && a.splits >= 1 && a.splits <= 64 && (a.splits == 1 || a.partial), "product arguments");
    if (packed) require(kernel >= kMat64 && kernel <= kMatFew, "packed operands and a kernel for any alignment");
    if (kernel >= kMatFew) require(a.M <= kMatFewRows && !flags && a.splits == 1, "few rows");
    if (!packed && a.K > 0 && kernel >= kMat64 && kernel <= kMatFew) {
        const long long la = flags & DWM_A_ACROSS ? a.M : a.K, lb = flags & DWM_B_ACROSS ? a.N : a.K;  // (rows of odd lengths come as copies, whole vectors apart)
        require((la + 7) / 8 * 8 <= a.stride[kMatA] && (lb + 7) / 8 * 8 <= a.stride[kMatB] && a.stride[kMatA] % 8 == 0 && a.stride[kMatB] % 8 == 0 && (uintptr_t)a.a % 16 == 0 && (uintptr_t)a.b % 16 == 0,
                "sixteen bytes at a time");
        require((la % 8 == 0 || (uintptr_t)a.a > 1 << 20) && (lb % 8 == 0 || (uintptr_t)a.b > 1 << 20), "rows of odd lengths that are no copies");
        require(a.stride[kMatA] * 2 * 256 < 1LL << 32 && a.stride[kMatB] * 2 * 256 < 1LL << 32, "offsets of 32 bits");
    }
    return DWM_OK;
}
dwm_status_t launch_matmul_f16(const MatmulArgs& a, int flags, int kernel, void*) { return matmul(a, flags, kernel, false); }
dwm_status_t launch_matmul_bf16(const MatmulArgs& a, int flags, int kernel, void*) { return matmul(a, flags, kernel, false); }
dwm_status_t launch_matmul_packed(const MatmulArgs& a, int flags, int kernel, void*) { return matmul(a, flags, kernel, true); }

}  // namespace dwm

static std::mt19937_64 rng(7);
static long long upto(long long n) { return (long long)(rng() % (uint64_t)(n + 1)); }
static long long size(int bits) { return upto((1LL << upto(bits))); }
static void* const kWs = (void*)(uintptr_t)4096;
static void* place() { return (void*)(uintptr_t)(4096 + 2 * upto(16) * (upto(2) ? 8 : 1)); }

int main(int argc, char** argv)
{
    const int rounds = argc > 1 ? std::atoi(argv[1]) : 2000;
    long long made = 0;
    for (int i = 0; i < rounds; ++i) {
        const dwm_type_t type = (dwm_type_t)upto(3), param = upto(1) ? DWM_F32 : type;
        const long long rows = size(30);
        const int C = (int)size(20);
        dwm_packed_t p = {kWs, kWs};
        dwm_rms_plan_t* rms = nullptr;
        if (dwm_rms_plan_create(&rms, rows, C, type, param, 1e-5) == DWM_OK) {
            ++made;
            if (upto(1)) dwm_rms_set_variant(rms, upto(1) ? "forward" : "backward", (int)upto(16) - 1);
            dwm_rms_set_stride(rms, "x", C + upto(8));
            dwm_rms_forward(rms, kWs, kWs, nullptr, kWs, kWs, &p, &p, (float*)kWs, nullptr);
            if (upto(3)) require(dwm_rms_set_workspace(rms, kWs, dwm_rms_workspace_bytes(rms)) == DWM_OK, "rms workspace");
            dwm_rms_backward(rms, kWs, nullptr, upto(1) ? kWs : nullptr, upto(1) ? &p : nullptr, nullptr, (const float*)kWs, kWs, upto(1) ? kWs : nullptr, nullptr);
            dwm_rms_plan_destroy(rms);
        }
        dwm_act_plan_t* act = nullptr;
        if (dwm_act_plan_create(&act, (dwm_act_t)upto(4), rows, C, type, param) == DWM_OK) {
            ++made;
            dwm_act_forward(act, kWs, nullptr, kWs, &p, nullptr);
            if (upto(3)) require(dwm_act_set_workspace(act, kWs, dwm_act_workspace_bytes(act)) == DWM_OK, "act workspace");
            dwm_act_backward(act, kWs, nullptr, nullptr, &p, kWs, upto(1) ? kWs : nullptr, nullptr);
            dwm_act_plan_destroy(act);
        }
        dwm_pack(type, rows, C, kWs, C, &p, nullptr);
        const dwm_type_t operands = (dwm_type_t)upto(3);
        const int M = (int)size(25), N = (int)size(25), K = (int)size(25), e = upto(1) ? 8 : 1, flags = operands == DWM_PACKED ? 0 : (int)upto(3);
        dwm_matmul_plan_t* mm = nullptr;
        if (dwm_matmul_plan_create(&mm, M / e * e, N / e * e, K / e * e, operands, operands == DWM_PACKED ? DWM_BF16 : upto(1) ? DWM_F32 : operands, DWM_F32, (dwm_act_t)upto(3), flags) == DWM_OK) {
            ++made;
            if (upto(1)) dwm_matmul_set_variant(mm, "kernel", (int)upto(7) - 1);
            if (upto(1)) dwm_matmul_set_variant(mm, "splits", (int)upto(70) - 1);
            if (operands != DWM_PACKED) {
                dwm_matmul_set_stride(mm, "a", (flags & DWM_A_ACROSS ? M : K) / e * e + 8 * upto(3));
                dwm_matmul_set_stride(mm, "b", (flags & DWM_B_ACROSS ? N : K) / e * e + upto(8));
            }
            dwm_matmul_info_t info;
            require(dwm_matmul_plan_info(mm, &info) == DWM_OK && info.splits >= 1, "product info");
            const size_t bytes = dwm_matmul_workspace_bytes(mm);
            void* const space = (void*)((uintptr_t)1 << 40);
            dwm::copies_from = (uintptr_t)space;
            dwm::copies_to = dwm::copies_from + bytes;
            if (bytes && upto(3)) require(dwm_matmul_set_workspace(mm, space, bytes) == DWM_OK, "product workspace");
            if (operands == DWM_PACKED)
                dwm_matmul_packed(mm, &p, &p, nullptr, kWs, kWs, &p, &p, nullptr);
            else
                dwm_matmul(mm, place(), place(), nullptr, kWs, kWs, nullptr, nullptr, nullptr);
            dwm_matmul_plan_destroy(mm);
        }
    }
    std::printf("branch fuzz: %d rounds, %lld plans, %lld launches\n", rounds, made, launches);
    return 0;
}

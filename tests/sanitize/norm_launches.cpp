// Host-only check of which launches a backward call of a layer norm makes (norm.cpp), built by tests/test_norm_launches.py with the launchers stubbed:
// workgroups for the gradient of the norm's input only where one of its outputs is asked for, or where the parameters' gradients come from them.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2002_00552_amd/csrc/norm.hpp"

namespace dwm {
struct Launch {
    int what;  // 1: kernels for any size, 2: a shape, 3: the last sums
    NormArgs a;
};
static std::vector<Launch> taken;
static dwm_status_t shape(const NormArgs& a) { return taken.push_back({2, a}), DWM_OK; }
dwm_status_t launch_norm_any_forward(const NormArgs&, dwm_type_t, bool, void*) { return DWM_OK; }
dwm_status_t launch_norm_any_backward(const NormArgs& a, dwm_type_t, void*) { return taken.push_back({1, a}), DWM_OK; }
dwm_status_t launch_norm_params_final(const NormArgs& a, dwm_type_t, void*) { return taken.push_back({3, a}), DWM_OK; }
dwm_status_t launch_norm_f32(const NormArgs& a, const NormShape&, bool, bool, void*) { return shape(a); }
dwm_status_t launch_norm_f16(const NormArgs& a, const NormShape&, bool, bool, void*) { return shape(a); }
dwm_status_t launch_norm_bf16(const NormArgs& a, const NormShape&, bool, bool, void*) { return shape(a); }
dwm_status_t launch_dropout(const DropArgs&, dwm_type_t, long long, const void*, void*, void*) { return DWM_OK; }
}  // namespace dwm
using namespace dwm;

#define CHECK(c)                                                                        \
    do {                                                                                \
        if (!(c)) {                                                                     \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #c); \
            std::exit(2);                                                               \
        }                                                                               \
    } while (0)

int main()
{
    void* const p = (void*)(uintptr_t)4096;
    void* const q = (void*)(uintptr_t)8192;
    float* const f = (float*)(uintptr_t)12288;
    const long long sizes[][3] = {{1, 384, 1}, {700, 1021, 1}, {200000, 64, 1}, {2, 96, 49}, {16, 256, 196}, {64, 128, 784}, {2, 40000, 1}, {2, 3000, 9}};
    int aside = 0, sums = 0, any = 0;
    for (const auto& s : sizes) {
        dwm_norm_plan_t* plan = nullptr;
        CHECK(dwm_norm_plan_create(&plan, s[0], (int)s[1], s[2], DWM_BF16, DWM_F32, 1e-5) == DWM_OK);
        CHECK(dwm_norm_set_workspace(plan, p, dwm_norm_workspace_bytes(plan)) == DWM_OK);
        for (int params = 0; params < 4; ++params)
            for (int tensors = 0; tensors < 4; ++tensors)
                for (int join = 0; join < 2; ++join) {
                    float *dgamma = params & 1 ? f : nullptr, *dbeta = params & 2 ? f : nullptr;
                    void *dx = tensors & 1 ? q : nullptr, *dresidual = tensors & 2 ? q : nullptr;
                    if ((!join && dresidual) || (!params && !tensors)) continue;
                    taken.clear();
                    CHECK((join ? dwm_norm_join_backward(plan, nullptr, p, p, p, p, f, f, dx, dresidual, dgamma, dbeta, nullptr)
                                : dwm_norm_backward(plan, p, p, p, f, f, dx, dgamma, dbeta, nullptr)) == DWM_OK);
                    CHECK(!taken.empty());
                    for (const Launch& l : taken) {
                        if (l.what == 1) ++any;
                        if (l.what == 3) {
                            ++sums;
                            CHECK(params && l.a.partial);
                        }
                        if (l.what != 2) continue;
                        CHECK(l.a.splits >= 0 && (l.a.splits > 0 || l.a.aside));
                        if (l.a.aside) {
                            ++aside;
                            CHECK(params && !l.a.partial);
                        }
                        CHECK(l.a.splits == 0 || tensors || l.a.partial);  // workgroups for the gradient of z have something to write
                        CHECK(l.a.splits > 0 || !tensors);
                    }
                    // in dy's own memory the parameters' gradients come first, in a launch of their own or in front of it
                    if (!params || !tensors || join) continue;
                    taken.clear();
                    CHECK(dwm_norm_backward(plan, p, p, p, f, f, p, dgamma, dbeta, nullptr) == DWM_OK);
                    for (const Launch& l : taken) CHECK(l.what != 2 || !(l.a.aside && l.a.splits));
                }
        CHECK(dwm_norm_plan_destroy(plan) == DWM_OK);
    }
    CHECK(aside && sums && any);
    std::printf("norm launches: %d aside, %d sums, %d any\n", aside, sums, any);
    return 0;
}

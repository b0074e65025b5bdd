// What a plan of a matrix product says of itself against what its call launches, with the launchers stubbed: the kernel, the parts of K, and whether a workspace is needed.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>

#include "../../paper_2002_00552_amd/csrc/branch.hpp"

static void require(bool ok, const char* what, const dwm_matmul_info_t& i, int flags, int operands)
{
    if (ok) return;
    std::printf("ERROR: %s: %d x %d x %d, kernel %d, %d parts, flags %d, operands %d\n", what, i.M, i.N, i.K, i.kernel, i.splits, flags, operands);
    std::exit(1);
}

namespace dwm {

dwm_status_t launch_rms_forward(const RmsArgs&, dwm_type_t, int, void*) { return DWM_OK; }
dwm_status_t launch_rms_backward(const RmsArgs&, dwm_type_t, int, void*) { return DWM_OK; }
dwm_status_t launch_act_forward(const ActArgs&, dwm_type_t, void*) { return DWM_OK; }
dwm_status_t launch_act_backward(const ActArgs&, dwm_type_t, void*) { return DWM_OK; }
dwm_status_t launch_columns(const float*, int, int, void*, dwm_type_t, void*) { return DWM_OK; }
dwm_status_t launch_aligned_rows(const AlignedRows*, int, void*) { return DWM_OK; }

static MatmulShape launched;
static bool too_many;  // threads: a launch has fewer than 2^32
static dwm_status_t matmul(const MatmulArgs& a, int kernel)
{
    launched = {kernel, a.splits};
    const long long side = kernel == kMatAny64 || kernel == kMat64 ? 64 : kernel == kMat256 ? 256 : 128, threads = side == 256 ? 512 : 256;
    too_many = kernel < kMatFew && (a.M + side - 1) / side * ((a.N + side - 1) / side) * a.splits * threads >= 1LL << 32;
    return DWM_OK;
}
dwm_status_t launch_matmul_f16(const MatmulArgs& a, int, int kernel, void*) { return matmul(a, kernel); }
dwm_status_t launch_matmul_bf16(const MatmulArgs& a, int, int kernel, void*) { return matmul(a, kernel); }
dwm_status_t launch_matmul_packed(const MatmulArgs& a, int, int kernel, void*) { return matmul(a, kernel); }

}  // namespace dwm

static std::mt19937_64 rng(11);
static long long upto(long long n) { return (long long)(rng() % (uint64_t)(n + 1)); }
static int size(int bits) { return (int)upto((1LL << upto(bits))); }
static void* const kSpace = (void*)((uintptr_t)1 << 40);

static dwm_status_t call(dwm_matmul_plan_t* plan, dwm_type_t operands, void* a, void* b)
{
    dwm_packed_t p = {kSpace, kSpace};
    if (operands == DWM_PACKED) return dwm_matmul_packed(plan, &p, &p, nullptr, nullptr, kSpace, nullptr, nullptr, nullptr);
    return dwm_matmul(plan, a, b, nullptr, nullptr, kSpace, nullptr, nullptr, nullptr);
}

int main(int argc, char** argv)
{
    const int rounds = argc > 1 ? std::atoi(argv[1]) : 20000;
    void *const good = (void*)(uintptr_t)4096, *const loose = (void*)(uintptr_t)4098;
    long long run = 0;
    for (int i = 0; i < rounds; ++i) {
        const dwm_type_t operands = (dwm_type_t)(1 + upto(2));
        const int e = upto(1) ? 8 : 1, flags = operands == DWM_PACKED ? 0 : (int)upto(3), M = size(15) / e * e, N = size(15) / e * e, K = size(15) / e * e;
        dwm_matmul_plan_t* plan = nullptr;
        if (dwm_matmul_plan_create(&plan, M, N, K, operands, operands == DWM_PACKED ? DWM_F16 : operands, DWM_F32, DWM_ACT_NONE, flags) != DWM_OK) return 1;
        if (!upto(3)) dwm_matmul_set_variant(plan, "kernel", (int)upto(6) - 1);
        if (!upto(3)) dwm_matmul_set_variant(plan, "splits", (int)upto(9) - 1);
        dwm_matmul_info_t info;
        if (dwm_matmul_plan_info(plan, &info) != DWM_OK) return 1;
        if (M > 0 && N > 0) {
            ++run;
            // Whole vectors at multiples of sixteen, every pair of addresses that are not, without a workspace: refused by some where there is one to be set, by none where there is none.
            const size_t bytes = dwm_matmul_workspace_bytes(plan);
            bool refused = false;
            for (int which = 0; which < 4; ++which) {
                const dwm_status_t st = call(plan, operands, which & 1 ? loose : good, which & 2 ? loose : good);
                require(st == DWM_OK || st == DWM_ERR_WORKSPACE, "status", info, flags, operands);
                refused |= st == DWM_ERR_WORKSPACE;
            }
            require(refused == (bytes > 0), bytes ? "a workspace that nothing needs" : "a workspace that is not asked for", info, flags, operands);
            if (bytes) dwm_matmul_set_workspace(plan, kSpace, bytes);
            require(call(plan, operands, good, good) == DWM_OK, "a call", info, flags, operands);
            const int kernel = dwm::launched.kernel == dwm::kMatFewLoose ? (int)dwm::kMatFew : dwm::launched.kernel;
            require(kernel == info.kernel && dwm::launched.splits == info.splits, "another kernel than the plan says", info, flags, operands);
        }
        dwm_matmul_plan_destroy(plan);
    }
    // The largest results, operands aligned and not, as planned and as asked for: what a plan takes can be launched.
    for (int i = 0; i < rounds; ++i) {
        const int few = (int)upto(1), flags = (int)upto(3), e = upto(1) ? 8 : 1, M = (int)(few ? size(24) : (1 << 24) - size(23)) / e * e, N = (int)((1LL << 37) / (M > 0 ? M : 1) > 1 << 24 ? size(24) : (1LL << 37) / (M > 0 ? M : 1) - size(10));
        const dwm_type_t operands = flags ? DWM_BF16 : (dwm_type_t)(1 + upto(2));
        dwm_matmul_plan_t* plan = nullptr;
        if (M <= 0 || N <= 0 || dwm_matmul_plan_create(&plan, M, N / e * e, size(16), operands, operands == DWM_PACKED ? DWM_F16 : operands, DWM_F32, DWM_ACT_NONE, flags) != DWM_OK) continue;
        if (!upto(2)) dwm_matmul_set_variant(plan, "kernel", (int)upto(6) - 1);
        if (!upto(2)) dwm_matmul_set_variant(plan, "splits", (int)upto(65) - 1);
        const size_t bytes = dwm_matmul_workspace_bytes(plan);
        if (bytes) dwm_matmul_set_workspace(plan, kSpace, bytes);
        dwm_matmul_info_t info;
        if (dwm_matmul_plan_info(plan, &info) != DWM_OK) return 1;
        if (info.M > 0 && info.N > 0)
            for (int which = 0; which < 4; ++which) {
                require(call(plan, operands, which & 1 ? loose : good, which & 2 ? loose : good) == DWM_OK, "a large call", info, flags, operands);
                require(!dwm::too_many, "more threads than a launch has", info, flags, operands);
                ++run;
            }
        dwm_matmul_plan_destroy(plan);
    }
    std::printf("branch launches: %d rounds, %lld calls\n", rounds, run);
    return 0;
}

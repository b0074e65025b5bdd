// Host-only fuzz of the layer norms' plans, checks of arguments and index rules (norm.cpp, norm.hpp), built with
// -fsanitize=address,undefined by tests/test_norm_planning.py: for random sizes, types and variants the launches that the entry points make
// are taken down by stubs, and what the kernels would read and write is replayed from the same rules -- every channel of a row and every pixel and
// channel of a map once, every tile once, partial sums inside the workspace.  Nothing here touches a GPU.
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "../../paper_2002_00552_amd/csrc/norm.hpp"

namespace dwm {
struct Launch {
    int what;  // 1: any, forward; 2: any, backward; 3: a shape; 4: the sums of the partial sums; 5: dropout
    NormArgs a;
    NormShape shape;
    dwm_type_t type;
    bool backward;
};
static std::vector<Launch> taken;
dwm_status_t launch_norm_any_forward(const NormArgs& a, dwm_type_t t, bool, void*) { return taken.push_back({1, a, {}, t, false}), DWM_OK; }
dwm_status_t launch_norm_any_backward(const NormArgs& a, dwm_type_t t, void*) { return taken.push_back({2, a, {}, t, true}), DWM_OK; }
dwm_status_t launch_norm_params_final(const NormArgs& a, dwm_type_t t, void*) { return taken.push_back({4, a, {}, t, true}), DWM_OK; }
dwm_status_t launch_norm_f32(const NormArgs& a, const NormShape& s, bool b, bool, void*) { return taken.push_back({3, a, s, DWM_F32, b}), DWM_OK; }
dwm_status_t launch_norm_f16(const NormArgs& a, const NormShape& s, bool b, bool, void*) { return taken.push_back({3, a, s, DWM_F16, b}), DWM_OK; }
dwm_status_t launch_norm_bf16(const NormArgs& a, const NormShape& s, bool b, bool, void*) { return taken.push_back({3, a, s, DWM_BF16, b}), DWM_OK; }
dwm_status_t launch_dropout(const DropArgs& d, dwm_type_t t, long long, const void*, void*, void*)
{
    Launch l{5, {}, {}, t, false};
    l.a.drop = d;
    return taken.push_back(l), DWM_OK;
}
}  // namespace dwm
using namespace dwm;

static uint64_t g_state = 0x9E3779B97F4A7C15ull;
static uint32_t rnd()
{
    g_state ^= g_state << 13;
    g_state ^= g_state >> 7;
    g_state ^= g_state << 17;
    return (uint32_t)(g_state >> 32);
}
static int pick(int lo, int hi) { return lo + (int)(rnd() % (uint32_t)(hi - lo + 1)); }
#define CHECK(c)                                                              \
    do {                                                                      \
        if (!(c)) {                                                           \
            std::fprintf(stderr, "%s:%d: check failed: %s\n", __FILE__, __LINE__, #c); \
            std::exit(2);                                                     \
        }                                                                     \
    } while (0)

// A line of `length` elements in vectors of vec: each element is some vector's own once, no vector leaves the line.
static void line(int length, int vec, int vectors)
{
    std::vector<char> own(length, 0);
    for (int i = 0; i < vectors; ++i) {
        const NormVector v = norm_vector(i, length, vec);
        CHECK(v.first >= 0 && v.first <= vec);
        if (v.first == vec) continue;
        CHECK(v.start >= 0 && v.start + vec <= length);
        for (int j = v.first; j < vec; ++j) CHECK(!own[v.start + j]++);
    }
    for (char c : own) CHECK(c);
}

// Every tile has one workgroup, also where those in front make parameters' gradients (a multiple of eight of them).
static void tiles(long long n, int blocks)
{
    CHECK(blocks >= 1 && (blocks <= n || (n == 0 && blocks == 1)));
    std::vector<char> done(n, 0);
    for (int b = 0; b < blocks; ++b) {
        const NormTiles t = norm_tiles(n, b, blocks);
        CHECK(t.step >= 1 && t.end <= n);
        for (long long i = t.tile; i < t.end; i += t.step) CHECK(!done[i]++);
    }
    for (char c : done) CHECK(c);
}

static void replay(const Launch& l, size_t workspace)
{
    const NormArgs& a = l.a;
    const int size = l.type == DWM_F32 ? 4 : 2, vec = 16 / size;
    CHECK(a.C >= 1 && a.inner >= 1 && a.outer >= 0);
    for (long long s : a.stride) CHECK(s >= a.C * a.inner);
    if (a.partial && l.backward) CHECK((size_t)a.splits * 2 * a.C * 4 <= workspace);
    if (l.what != 3) return;
    const int k = l.shape.kernel;
    if (k < kNormMapsVec) {
        const NormRows& r = kNormRows[k - kNormRowsFirst];
        CHECK(a.inner == 1 && a.C >= vec && r.tpr * r.k * vec >= a.C);
        CHECK(l.backward ? r.backward && r.tpr * r.k * vec <= kNormRowsWidest : r.forward);
        line(a.C, vec, r.tpr * r.k);
        const int threads = l.backward ? norm_rows_threads(r, a.C % vec != 0) : r.tpr > 256 ? r.tpr : 256;
        CHECK(threads % r.tpr == 0 && threads <= 1024);
        // workgroups step over the rows: none begins behind the last one, so none leaves its partial sums unwritten -- and an empty one would write zeros
        CHECK(l.shape.blocks >= 1 && (long long)(l.shape.blocks - 1) * (threads / r.tpr) <= (a.outer ? a.outer - 1 : 0));
    } else {
        const bool one = k >= kNormMapsOne;
        const NormMaps& m = kNormMaps[k - (one ? kNormMapsOne : kNormMapsVec)];
        const int v = one ? 1 : kNormMapsPixels;
        CHECK(m.cg * m.k >= a.C && (!one || m.one) && (!l.backward || size <= m.backward) && a.inner >= v);
        CHECK(m.pl * m.cg <= 1024 && m.pl * m.cg % 64 == 0 && 64 % m.pl == 0);
        const long long per = (a.inner + v - 1) / v, all = a.outer * per;
        CHECK(all < (1LL << 31) - 8);
        if (a.inner < 100000) line((int)a.inner, v, (int)per);
        const long long n = (all + m.pl - 1) / m.pl;
        if (n < 200000) tiles(n, l.shape.blocks);
    }
}

int main(int argc, char** argv)
{
    const int rounds = argc > 1 ? std::atoi(argv[1]) : 1000;
    long long plans = 0, refused = 0;
    void* const p = (void*)(uintptr_t)4096;
    void* const q = (void*)(uintptr_t)8192;
    float* const f = (float*)(uintptr_t)12288;
    for (int r = 0; r < rounds; ++r) {
        const bool rows = rnd() % 2;
        long long outer = rnd() % 20 ? 1LL << pick(0, 16) : 0, inner = rows ? 1 : 1LL << pick(0, 14);
        outer += outer ? rnd() % outer : 0;
        inner += rows ? 0 : rnd() % inner;
        int C = 1 << pick(0, rows ? 15 : 11);
        C += rnd() % C;
        if (rnd() % 50 == 0) outer = (1LL << 40) / (C * inner) + pick(-1, 1);  // at the limit
        const dwm_type_t type = (dwm_type_t)pick(0, 2), params = rnd() % 2 ? DWM_F32 : type;
        dwm_norm_plan_t* plan = nullptr;
        const dwm_status_t st = dwm_norm_plan_create(&plan, outer, C, inner, type, params, 1e-5);
        CHECK(st == DWM_OK || st == DWM_ERR_UNSUPPORTED);
        if (st != DWM_OK) {
            CHECK(!plan && outer > (1LL << 40) / (C * inner));
            ++refused;
            continue;
        }
        ++plans;
        const int variant = rnd() % 3 ? -1 : pick(-1, 215);
        for (const char* stage : {"forward", "backward"}) {
            const dwm_status_t v = dwm_norm_set_variant(plan, stage, variant);
            CHECK(v == DWM_OK || (variant > 0 && v == DWM_ERR_INVALID_ARG));
        }
        dwm_norm_info_t info;
        CHECK(dwm_norm_plan_info(plan, &info) == DWM_OK && info.splits >= 1);
        const size_t need = dwm_norm_workspace_bytes(plan);
        CHECK(need == (size_t)info.splits * 2 * C * 4);
        taken.clear();
        CHECK(dwm_norm_backward(plan, p, p, p, f, f, q, f, f, nullptr) == DWM_ERR_WORKSPACE && taken.empty());
        CHECK(dwm_norm_set_workspace(plan, p, need) == DWM_OK);
        dwm_dropout_t drop = {rnd() / 4294967296.0, rnd(), rnd(), nullptr};
        CHECK(dwm_norm_forward(plan, p, p, p, p, f, f, nullptr) == DWM_OK);
        CHECK(dwm_norm_join_forward(plan, &drop, p, p, p, p, p, p, f, f, nullptr) == DWM_OK);
        CHECK(dwm_norm_backward(plan, p, p, p, f, f, q, f, f, nullptr) == DWM_OK);
        CHECK(dwm_norm_backward(plan, p, p, p, f, f, p, f, f, nullptr) == DWM_OK);  // in dy's memory
        CHECK(dwm_norm_join_backward(plan, &drop, p, p, p, p, f, f, q, q, f, f, nullptr) == DWM_OK);
        CHECK(dwm_norm_join_backward(plan, nullptr, p, nullptr, p, p, f, f, nullptr, q, nullptr, nullptr, nullptr) == DWM_OK);
        if (outer > 0) CHECK(taken.size() >= 6);
        for (const Launch& l : taken) {
            replay(l, need);
            if (l.a.drop.mode == kDropDraw) CHECK(std::abs((double)l.a.drop.threshold - drop.p * 4294967296.0) <= 0.5);
            // dy's own memory as output beside workgroups that read it: never in one launch
            if (l.what == 3 && l.backward && l.a.aside && l.a.splits) CHECK(l.a.dx != l.a.dy && l.a.dresidual != l.a.dy);
        }
        CHECK(dwm_norm_plan_destroy(plan) == DWM_OK);
    }
    std::printf("norm fuzz: %lld plans, %lld refused\n", plans, refused);
    return 0;
}

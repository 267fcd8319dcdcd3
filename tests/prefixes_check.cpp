// Host checks of shared prefixes and evictions: no word of a group leads outside the call, runs of pages cover every page
// once, and the entry points refuse what they document before any launch (the launchers here only count).
#include <cstdio>
#include <vector>

#include "hga_abi_shared.cpp"

alignas(16) static unsigned char buf[64];
static int g_launches = 0, g_plain = 0, g_bad = 0;

namespace hga {
namespace abi {
hga_status fail(hga_status st, const char*, ...) { return st; }
hga_status hip_fail(hipError_t, const char*) { return HGA_EHIP; }
bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
hga_status check_plan(const hga_plan* plan) { return plan ? HGA_OK : HGA_EINVAL; }
hga_status check_tensor(const void* p, const char*) { return !p ? HGA_EINVAL : aligned(p, 16) ? HGA_OK : HGA_EALIGN; }
hga_status check_index(const void* p, const char*) { return !p ? HGA_EINVAL : aligned(p, 4) ? HGA_OK : HGA_EALIGN; }
hga_status check_workspace(const void* w, int64_t n) {
    return n < 0 || (n > 0 && !w) ? HGA_EINVAL : n > 0 && !aligned(w, 16) ? HGA_EALIGN : HGA_OK;
}
hga_status launched(hipError_t e, const char*) { return e == hipSuccess ? HGA_OK : HGA_EHIP; }
}  // namespace abi
hipError_t launch_attend_tokens(const hga_plan&, const PoolView&, const TokensView&, const void*, int64_t, const int32_t*,
                                int, void*, float*, void*, int64_t, hipStream_t) {
    ++g_plain;
    return hipSuccess;
}
int64_t attend_tokens_bytes(const hga_plan&, int, int, int, int) { return 16; }
// (a shared_hint of 3: too little)
bool attend_shared_pays(const hga_plan&, int, int, int, int, int shared) { return shared != 3; }
int64_t attend_shared_bytes(const hga_plan&, int, int, int, int, int, int, bool must) { return must ? 32 : 64; }
hipError_t launch_attend_shared(const hga_plan&, const PoolView&, const TokensView& tok, const PrefixView&, int shared, int own,
                                const void*, int64_t, void*, float*, void*, int64_t, hipStream_t) {
    if (shared < 1 || shared > tok.max_pages || own < 1 || own > tok.max_pages) ++g_bad, std::printf("hints %d %d\n", shared, own);
    ++g_launches;
    return hipSuccess;
}
int64_t weigh_pages_bytes(const hga_plan&, int, int, int, int) { return 0; }
hipError_t launch_weigh_pages(const hga_plan&, const PoolView&, const TokensView&, const void*, int64_t, const float*,
                              const int32_t*, int, const float*, float*, void*, int64_t, hipStream_t) {
    ++g_launches;
    return hipSuccess;
}
int64_t choose_evictions_bytes(int, int max_pages) { return max_pages > 100 ? 64 : 0; }
hipError_t launch_choose_evictions(const hga_plan&, const int32_t*, int, int, int, const int32_t*, const float*, const int32_t*,
                                   int32_t*, int, void*, int64_t, hipStream_t) {
    ++g_launches;
    return hipSuccess;
}
}  // namespace hga
extern "C" hipError_t hipHostGetDevicePointer(void** d, void* h, unsigned) {
    *d = h;
    return hipSuccess;
}
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

static void expect(bool ok, int line) {
    if (!ok) std::printf("line %d\n", line), ++g_bad;
}
#define EXPECT(x) expect((x), __LINE__)

static void bounds() {
    const int odd[] = {INT_MIN, INT_MIN + 1, -2, -1, 0, 1, 2, 3, 7, 8, 9, 1 << 30, INT_MAX - 1, INT_MAX};
    for (int a : odd)
        for (int b : odd)
            for (int n : {0, 1, 7, 8}) {
                int32_t order[1] = {a}, begin[2] = {a, b}, pages[1] = {b};
                const hga::PrefixView px{order, begin, pages, 1};
                const int t = px.token(0, n), first = px.first(0, n), end = px.end(0, n), shared = px.shared(0, n);
                EXPECT(t == -1 || (t == a && t >= 0 && t < n));
                EXPECT(first >= 0 && first <= end && end <= n && shared >= 0 && shared <= n);
                if (a >= 0 && a <= b && b <= n) EXPECT(first == a && end == b);
            }
    for (int n = 0; n < 70; ++n)
        for (int run : {1, 2, 3, 8, 64, 100})
            for (int most : {1, 2, 5, 70}) {
                const int runs = hga::runs_of(n, run, most);
                EXPECT(runs >= (n > 0) && runs <= most);
                int at = 0;
                for (int j = 0; j < most + 2; ++j) {
                    const hga::PageRun r = hga::page_run(j, n, run, most);
                    if (j >= runs) {
                        EXPECT(r.a == r.b);
                        continue;
                    }
                    EXPECT(r.a == at && r.b > r.a);
                    at = r.b;
                }
                EXPECT(at == n);
            }
}

static void refusals() {
    hga_plan plan{};
    plan.p.n_q_heads = 4, plan.p.n_kv_heads = 2, plan.p.head_dim = 64, plan.p.keep_first = 1, plan.p.force_prev = 1;
    plan.p.topk_chunks = 3, plan.p.dtype = HGA_BF16;
    const auto at = [](int off) { return static_cast<void*>(buf + off); };
    const auto f = [&](int off) { return reinterpret_cast<float*>(buf + off); };
    const auto i = [&](int off) { return reinterpret_cast<int32_t*>(buf + off); };
    hga_pool pool{};
    pool.pages = buf, pool.page_sum = f(0), pool.n_layers = 2, pool.n_pages = 5;
    hga_tokens tok{};
    tok.tok_seq = tok.tok_pos = tok.page_table = i(0), tok.n_tokens = 3, tok.n_seqs = 2, tok.max_pages = 9;
    const hga_prefixes good{i(0), i(0), i(0), 1, 4, 5};
    hga_prefixes px = good;
    const auto attend = [&](int layer = 0, const void* q = buf, int64_t qs = 256, void* o = buf, float* lse = nullptr,
                            void* w = buf, int64_t wb = 64) {
        return hga_attend_shared(&plan, &pool, layer, &tok, &px, q, qs, o, lse, w, wb, nullptr);
    };
    const auto weigh = [&](const float* lse = reinterpret_cast<float*>(buf), const int32_t* l = nullptr, int n = 0,
                           const float* prev = nullptr, float* w = reinterpret_cast<float*>(buf), void* ws = nullptr,
                           int64_t wb = 0) {
        return hga_weigh_pages(&plan, &pool, 0, &tok, buf, 256, lse, l, n, prev, w, ws, wb, nullptr);
    };
    const auto choose = [&](int seqs = 2, int pages = 9, int ids = 5, const void* len = buf, const void* w = buf,
                            const void* budget = buf, void* out = buf, int n = 3, void* ws = nullptr, int64_t wb = 0) {
        return hga_choose_evictions(&plan, i(0), seqs, pages, ids, static_cast<const int32_t*>(len),
                                    static_cast<const float*>(w), static_cast<const int32_t*>(budget),
                                    static_cast<int32_t*>(out), n, ws, wb, nullptr);
    };
    EXPECT(attend() == HGA_OK && g_launches == 1 && weigh() == HGA_OK && choose() == HGA_OK && g_launches == 3);
    EXPECT(weigh(f(0), i(0), 4, f(0)) == HGA_OK && g_launches == 4);
    // without room for two partial results nothing is shared
    EXPECT(attend(0, buf, 256, buf, nullptr, buf, 16) == HGA_OK && attend(0, buf, 256, buf, nullptr, nullptr, 0) == HGA_OK);
    EXPECT(g_plain == 2 && g_launches == 4);
    px.shared_hint = 3;
    EXPECT(attend() == HGA_OK && g_plain == 3 && g_launches == 4);
    EXPECT(hga_attend_shared_workspace(&plan, 3, 2, 9, 1, 3, 0) == 16 && hga_attend_shared_workspace(&plan, 3, 2, 9, 1, 4, 0) == 64);
    for (int hint : {0, 1, 9, 10, INT_MAX}) {
        px.shared_hint = px.own_hint = hint;
        EXPECT(attend() == HGA_OK);
    }
    px.n_groups = 0, px.group_begin = px.group_pages = nullptr;
    EXPECT(attend() == HGA_OK);
    px = good;
    g_launches = g_plain = 0;
    EXPECT(hga_attend_shared(nullptr, &pool, 0, &tok, &px, buf, 256, buf, nullptr, buf, 64, nullptr) == HGA_EINVAL);
    EXPECT(hga_attend_shared(&plan, nullptr, 0, &tok, &px, buf, 256, buf, nullptr, buf, 64, nullptr) == HGA_EINVAL);
    EXPECT(hga_attend_shared(&plan, &pool, 0, nullptr, &px, buf, 256, buf, nullptr, buf, 64, nullptr) == HGA_EINVAL);
    EXPECT(hga_attend_shared(&plan, &pool, 0, &tok, nullptr, buf, 256, buf, nullptr, buf, 64, nullptr) == HGA_EINVAL);
    EXPECT(hga_attend_shared_workspace(nullptr, 1, 1, 1, 1, 0, 0) == HGA_EINVAL && hga_weigh_pages_workspace(nullptr, 1, 1, 1, 0) == HGA_EINVAL);
    EXPECT(hga_choose_evictions_workspace(nullptr, 1, 1) == HGA_EINVAL && hga_choose_evictions_workspace(&plan, -1, 1) == HGA_EINVAL);
    EXPECT(hga_attend_shared_workspace(&plan, 1, 1, 1, -1, 0, 0) == HGA_EINVAL && hga_attend_shared_workspace(&plan, 1, 1, 1, 1, -1, 0) == HGA_EINVAL);
    EXPECT(hga_attend_shared_workspace(&plan, 1, 1, 1, 1, 0, -1) == HGA_EINVAL);
    EXPECT(hga_attend_shared_workspace(&plan, 1, 1, 1, (1 << 20) + 1, 0, 0) == HGA_EUNSUPPORTED);
    EXPECT(hga_attend_shared_workspace(&plan, (1 << 28) + 1, 1, 1, 1, 0, 0) == HGA_EUNSUPPORTED);
    EXPECT(hga_weigh_pages_workspace(&plan, 1, 1, 1, -1) == HGA_EINVAL && hga_weigh_pages_workspace(&plan, 1, 1, (1 << 18) + 1, 0) == HGA_EUNSUPPORTED);
    EXPECT(attend(-1) == HGA_EINVAL && attend(2) == HGA_EINVAL && attend(0, nullptr) == HGA_EINVAL && attend(0, at(8)) == HGA_EALIGN);
    EXPECT(attend(0, buf, 255) == HGA_EINVAL && attend(0, buf, 260) == HGA_EALIGN && attend(0, buf, 256, nullptr) == HGA_EINVAL);
    EXPECT(attend(0, buf, 256, at(4)) == HGA_EALIGN && attend(0, buf, 256, buf, f(1)) == HGA_EALIGN);
    EXPECT(attend(0, buf, 256, buf, nullptr, at(4), 32) == HGA_EALIGN && attend(0, buf, 256, buf, nullptr, nullptr, 32) == HGA_EINVAL);
    EXPECT(attend(0, buf, 256, buf, nullptr, buf, -1) == HGA_EINVAL);
    for (int n = 0; n < 7; ++n) {
        px = good;
        if (n == 0) px.order = nullptr;
        if (n == 1) px.order = i(2);
        if (n == 2) px.group_begin = nullptr;
        if (n == 3) px.group_pages = i(1);
        if (n == 4) px.n_groups = -1;
        if (n == 5) px.shared_hint = -1;
        if (n == 6) px.own_hint = -1;
        EXPECT(attend() < 0);
    }
    px = good;
    px.n_groups = (1 << 20) + 1;
    EXPECT(attend() == HGA_EUNSUPPORTED);
    px = good;
    EXPECT(weigh(nullptr) == HGA_EINVAL && weigh(f(2)) == HGA_EALIGN && weigh(f(0), i(0), 0) == HGA_EINVAL && weigh(f(0), nullptr, 3) == HGA_EINVAL);
    EXPECT(weigh(f(0), i(0), -1) == HGA_EINVAL && weigh(f(0), i(0), (1 << 20) + 1) == HGA_EUNSUPPORTED && weigh(f(0), i(1), 2) == HGA_EALIGN);
    EXPECT(weigh(f(0), nullptr, 0, f(2)) == HGA_EALIGN && weigh(f(0), nullptr, 0, nullptr, nullptr) == HGA_EINVAL);
    EXPECT(weigh(f(0), nullptr, 0, nullptr, f(0), at(4), 16) == HGA_EALIGN && weigh(f(0), nullptr, 0, nullptr, f(0), nullptr, 16) == HGA_EINVAL);
    EXPECT(hga_choose_evictions(nullptr, i(0), 2, 9, 5, i(0), f(0), i(0), i(0), 3, nullptr, 0, nullptr) == HGA_EINVAL);
    EXPECT(choose(-1) == HGA_EINVAL && choose(2, -1) == HGA_EINVAL && choose(2, 9, -1) == HGA_EINVAL && choose(2, (1 << 18) + 1) == HGA_EUNSUPPORTED);
    EXPECT(choose((1 << 30) + 1) == HGA_EUNSUPPORTED);
    EXPECT(choose(2, 9, 5, nullptr) == HGA_EINVAL && choose(2, 9, 5, buf, nullptr) == HGA_EINVAL && choose(2, 9, 5, buf, buf, nullptr) == HGA_EINVAL);
    EXPECT(choose(2, 9, 5, buf, buf, buf, nullptr) == HGA_EINVAL && choose(2, 9, 5, buf, buf, buf, at(2)) == HGA_EALIGN);
    EXPECT(choose(2, 9, 5, buf, buf, buf, buf, -1) == HGA_EINVAL);
    EXPECT(choose(2, 101) == HGA_EINVAL && choose(2, 101, 5, buf, buf, buf, buf, 3, buf, 48) == HGA_EINVAL && g_launches == 0);
    // nothing to do: nothing launched, pointers not looked at
    EXPECT(choose(0) == HGA_OK && choose(2, 9, 5, nullptr, nullptr, nullptr, nullptr, 0) == HGA_OK && g_launches == 0);
    tok.n_tokens = 0;
    EXPECT(attend(0, nullptr) == HGA_OK && g_launches == 0 && weigh(nullptr) == HGA_OK && g_launches == 1);  // (prev is copied)
    tok.max_pages = 0;
    EXPECT(weigh(nullptr, nullptr, 0, nullptr, nullptr) == HGA_OK && g_launches == 1);
}

int main() {
    bounds();
    refusals();
    return g_bad != 0;
}

// Host checks of the paged 4-bit cache: the page layout covers its bytes once, no table or list entry leads outside the
// pool, and the entry points refuse what they document before any launch (the launchers here only count).
#include <cstdarg>
#include <cstdio>
#include <vector>

#include "hga_abi_tokens.cpp"

alignas(16) static unsigned char buf[64];
static int g_launches = 0;
static int g_bad = 0;

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
static hipError_t count() {
    ++g_launches;
    return hipSuccess;
}
hipError_t launch_cache_append(const hga_plan&, const PoolView&, const TokensView&, const void*, int64_t, const void*,
                               int64_t, hipStream_t) { return count(); }
hipError_t launch_cache_read(const hga_plan&, const PoolView&, const TokensView&, void*, void*, hipStream_t) { return count(); }
hipError_t launch_copy_pages(const hga_plan&, const hga_pool&, void*, const int32_t*, const int32_t*, int, hipStream_t) { return count(); }
int64_t route_tokens_bytes(const hga_plan&, int, int max_pages, bool) { return max_pages > 100 ? 64 : 0; }
hipError_t launch_route_tokens(const hga_plan&, const PoolView&, const TokensView&, const void*, int64_t, int32_t*, int,
                               void*, int64_t, hipStream_t) { return count(); }
int64_t attend_tokens_bytes(const hga_plan&, int, int, int, int) { return 64; }
hipError_t launch_attend_tokens(const hga_plan&, const PoolView&, const TokensView&, const void*, int64_t, const int32_t*,
                                int, void*, float*, void*, int64_t, hipStream_t) { return count(); }
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

template <int D>
static void layout() {
    using F = hga::PageFormat<D>;
    EXPECT(F::kBytes == hga::page_head_bytes(D));
    std::vector<int> seen(F::kBytes, 0);
    for (int r = 0; r < 64; ++r) {
        for (int j = 0; j < D; j += 2) ++seen[F::key_code(r, j)], ++seen[F::value_code(r, j)];
        for (int b = 0; b < D / 32; ++b) ++seen[F::key_scale(r, b)], ++seen[F::value_scale(r, b)];
        for (int j = 0; j < D; ++j) EXPECT(F::key_code(r, j) == F::key_code(r, j & ~1) && F::value_code(r, j) == F::value_code(r, j & ~1));
    }
    for (int x : seen) EXPECT(x == 1);
    // the pieces a lane loads at once are contiguous and aligned
    for (int m = 0; m < 16; ++m)
        for (int g = 0; g < 4; ++g)
            for (int t = 0; t < 4; ++t) {
                const int k = F::key_code(16 * t + m, g * (D / 4)), v = F::value_code(16 * t + 4 * g, m * F::kLaneDims);
                EXPECT(k % (D / 8) == 0 && v % (D / 8) == 0);
                for (int i = 0; i < D / 4; i += 2) EXPECT(F::key_code(16 * t + m, g * (D / 4) + i) == k + i / 2);
                for (int i = 0; i < 4; ++i)
                    for (int j = 0; j < F::kLaneDims; j += 2)
                        EXPECT(F::value_code(16 * t + 4 * g + i, m * F::kLaneDims + j) == v + i * (F::kLaneDims / 2) + j / 2);
                const int kb = g * (D / 4) / 32, vb = m * F::kLaneDims / 32;
                EXPECT(F::key_scale(16 * t + m, kb) == F::key_scale(m, kb) + t && F::key_scale(m, kb) % 4 == 0);
                for (int i = 0; i < 4; ++i)
                    EXPECT(F::value_scale(16 * t + 4 * g + i, vb) == F::value_scale(4 * g, vb) + 4 * t + i);
                EXPECT(F::value_scale(4 * g, vb) % 16 == 0);
            }
}

static void bounds() {
    const int odd[] = {INT_MIN, INT_MIN + 1, -65, -64, -1, 0, 1, 2, 3, 4, 5, 63, 64, 127, 128, 191, 192, 255, 256, 1 << 30, INT_MAX - 1, INT_MAX};
    std::vector<unsigned char> hot(3 * 8), cold(2 * 8);
    const hga::PoolView pool{hot.data(), cold.data(), nullptr, 3, 2, 1, 8};
    std::vector<int32_t> table(2 * 4);
    for (int id : odd) {
        EXPECT(pool.has(id) == (id >= 0 && id < 5));
        if (pool.has(id)) {
            unsigned char* p = pool.page(id);
            EXPECT((p >= hot.data() && p + 8 <= hot.data() + hot.size()) || (p >= cold.data() && p + 8 <= cold.data() + cold.size()));
        }
        for (int s : odd)
            for (int pos : odd) {
                int32_t seq = s, at = pos;
                const hga::TokensView tok{&seq, &at, table.data(), 1, 2, 4};
                int s2, p2;
                const bool in = tok.at(0, s2, p2);
                EXPECT(in == (s >= 0 && s < 2 && pos >= 0 && pos < 256));
                if (!in) continue;
                for (int c : odd) {
                    for (int32_t& x : table) x = id;
                    const hga::SeenPage pg = hga::seen_page(pool, tok, s2, p2, c);
                    const bool sees = c >= 0 && c <= pos / 64 && id >= 0 && id < 5;
                    EXPECT((pg.rows > 0) == sees && (!sees || pg.id == id));
                    if (sees) EXPECT(pg.rows == (c < pos / 64 ? 64 : pos % 64 + 1));
                }
            }
    }
}

static void refusals() {
    hga_plan plan{};
    plan.p.n_q_heads = 4, plan.p.n_kv_heads = 2, plan.p.head_dim = 64, plan.p.keep_first = 1, plan.p.force_prev = 1;
    plan.p.topk_chunks = 3, plan.p.dtype = HGA_BF16;
    const auto at = [](int off) { return static_cast<void*>(buf + off); };
    hga_pool pool{};
    pool.pages = buf, pool.page_sum = reinterpret_cast<float*>(buf), pool.n_layers = 2, pool.n_pages = 5;
    hga_tokens tok{};
    const int32_t* ids = reinterpret_cast<int32_t*>(buf);
    tok.tok_seq = tok.tok_pos = tok.page_table = ids, tok.n_tokens = 3, tok.n_seqs = 2, tok.max_pages = 9;
    int32_t* list = reinterpret_cast<int32_t*>(buf);
    const auto append = [&](int layer = 0, const void* k = buf, int64_t ks = 128, int64_t vs = 128) {
        return hga_cache_append(&plan, &pool, layer, &tok, k, ks, buf, vs, nullptr);
    };
    const auto route = [&](int n = 6, const void* q = buf, int64_t qs = 256, int32_t* l = nullptr, void* w = nullptr, int64_t wb = 0) {
        return hga_route_tokens(&plan, &pool, 0, &tok, q, qs, l ? l : list, n, w, wb, nullptr);
    };
    const auto attend = [&](const int32_t* l = nullptr, int n = 0, void* o = buf, void* w = nullptr, int64_t wb = 0, float* lse = nullptr) {
        return hga_attend_tokens(&plan, &pool, 0, &tok, buf, 256, l, n, o, lse, w, wb, nullptr);
    };
    const auto copy = [&](int n, const void* s = buf) {
        return hga_copy_pages(&plan, &pool, static_cast<const int32_t*>(s), ids, n, nullptr);
    };
    EXPECT(append() == HGA_OK && route() == HGA_OK && attend() == HGA_OK && attend(ids, 1) == HGA_OK && copy(2) == HGA_OK);
    EXPECT(hga_cache_read(&plan, &pool, 1, &tok, buf, buf, nullptr) == HGA_OK && g_launches == 6);
    EXPECT(hga_token_list_size(&plan) == 6 && hga_page_bytes(&plan) == 2 * 64 * 68);
    g_launches = 0;
    EXPECT(hga_cache_append(nullptr, &pool, 0, &tok, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
    EXPECT(hga_cache_append(&plan, nullptr, 0, &tok, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
    EXPECT(hga_cache_append(&plan, &pool, 0, nullptr, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
    EXPECT(hga_page_bytes(nullptr) == HGA_EINVAL && hga_token_list_size(nullptr) == HGA_EINVAL);
    EXPECT(hga_route_tokens_workspace(nullptr, 1, 1) == HGA_EINVAL && hga_attend_tokens_workspace(nullptr, 1, 1, 1, 0) == HGA_EINVAL);
    EXPECT(hga_route_tokens_workspace(&plan, -1, 1) == HGA_EINVAL && hga_attend_tokens_workspace(&plan, 1, 1, 1, -1) == HGA_EINVAL);
    EXPECT(hga_route_tokens_workspace(&plan, 1, (1 << 18) + 1) == HGA_EUNSUPPORTED);
    EXPECT(append(-1) == HGA_EINVAL && append(2) == HGA_EINVAL && append(0, nullptr) == HGA_EINVAL && append(0, at(4)) == HGA_EALIGN);
    EXPECT(append(0, buf, 127) == HGA_EINVAL && append(0, buf, 132) == HGA_EALIGN && append(0, buf, 128, 0) == HGA_EINVAL);
    EXPECT(append(0, buf, -128) == HGA_EINVAL && append(0, buf, INT64_MAX & ~int64_t(15)) == HGA_EINVAL);
    EXPECT(hga_cache_read(&plan, &pool, 0, &tok, nullptr, buf, nullptr) == HGA_EINVAL);
    EXPECT(hga_cache_read(&plan, &pool, 0, &tok, buf, at(8), nullptr) == HGA_EALIGN);
    EXPECT(route(5) == HGA_EINVAL && route(6, nullptr) == HGA_EINVAL && route(6, buf, 255) == HGA_EINVAL && route(6, buf, 260) == HGA_EALIGN);
    EXPECT(route(6, buf, 256, reinterpret_cast<int32_t*>(buf + 2)) == HGA_EALIGN && route(6, buf, 256, nullptr, nullptr, 16) == HGA_EINVAL);
    EXPECT(route(6, buf, 256, nullptr, at(4), 16) == HGA_EALIGN && route(6, buf, 256, nullptr, buf, -1) == HGA_EINVAL);
    tok.max_pages = 101;
    EXPECT(route() == HGA_EINVAL && route(6, buf, 256, nullptr, buf, 63) == HGA_EINVAL && g_launches == 0);
    tok.max_pages = 9;
    EXPECT(attend(ids, 0) == HGA_EINVAL && attend(nullptr, 3) == HGA_EINVAL && attend(ids, -1) == HGA_EINVAL);
    EXPECT(attend(nullptr, 0, nullptr) == HGA_EINVAL && attend(nullptr, 0, at(2)) == HGA_EALIGN);
    EXPECT(attend(nullptr, 0, buf, at(8), 8) == HGA_EALIGN && attend(nullptr, 0, buf, nullptr, 8) == HGA_EINVAL);
    EXPECT(attend(nullptr, 0, buf, nullptr, 0, reinterpret_cast<float*>(buf + 1)) == HGA_EALIGN);
    EXPECT(attend(reinterpret_cast<int32_t*>(buf + 1), 2) == HGA_EALIGN);
    EXPECT(route((1 << 20) + 1) == HGA_EUNSUPPORTED && attend(ids, (1 << 20) + 1) == HGA_EUNSUPPORTED);
    EXPECT(hga_attend_tokens_workspace(&plan, 1, 1, 1, (1 << 20) + 1) == HGA_EUNSUPPORTED);
    EXPECT(append(0, buf, (int64_t(1) << 46) / 3 / 8 * 8 + 8) == HGA_EINVAL);
    plan.p.keep_first = INT_MAX;
    EXPECT(hga_token_list_size(&plan) == HGA_EUNSUPPORTED && route(1 << 20) == HGA_EINVAL);
    plan.p.keep_first = 1;
    EXPECT(copy(-1) == HGA_EINVAL && copy(1, nullptr) == HGA_EINVAL && copy(1, at(1)) == HGA_EALIGN && copy((1 << 29) + 1) == HGA_EUNSUPPORTED);
    for (int n : {-1, 1}) {
        hga_tokens bad = tok;
        if (n < 0) bad.n_tokens = n; else bad.tok_pos = nullptr;
        EXPECT(hga_cache_append(&plan, &pool, 0, &bad, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
        bad = tok;
        if (n < 0) bad.n_seqs = n; else bad.page_table = nullptr;
        EXPECT(hga_cache_append(&plan, &pool, 0, &bad, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
        bad = tok;
        if (n < 0) bad.max_pages = n; else bad.max_pages = (1 << 18) + 1;
        EXPECT(hga_cache_append(&plan, &pool, 0, &bad, buf, 128, buf, 128, nullptr) < 0);
        bad = tok;
        bad.n_tokens = (1 << 29) + 1;
        EXPECT(hga_cache_append(&plan, &pool, 0, &bad, buf, 128, buf, 128, nullptr) == HGA_EUNSUPPORTED);
        hga_pool p2 = pool;
        if (n < 0) p2.n_pages = n; else p2.pages = nullptr;
        EXPECT(hga_cache_append(&plan, &p2, 0, &tok, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
        p2 = pool;
        if (n < 0) p2.n_cold = n; else p2.n_cold = 2;   // no cold pages given
        EXPECT(hga_copy_pages(&plan, &p2, ids, ids, 1, nullptr) == HGA_EINVAL);
        p2 = pool;
        if (n < 0) p2.n_layers = 0; else p2.page_sum = nullptr;
        EXPECT(hga_cache_append(&plan, &p2, 0, &tok, buf, 128, buf, 128, nullptr) == HGA_EINVAL);
        p2 = pool;
        p2.n_pages = INT_MAX, p2.n_cold = 1, p2.cold = buf;
        EXPECT(hga_cache_append(&plan, &p2, 0, &tok, buf, 128, buf, 128, nullptr) == HGA_EUNSUPPORTED);
    }
    EXPECT(g_launches == 0);
    // nothing to do: nothing launched, pointers not looked at
    tok.n_tokens = 0;
    EXPECT(append(0, nullptr) == HGA_OK && attend(nullptr, 0, nullptr) == HGA_OK && copy(0, nullptr) == HGA_OK && g_launches == 0);
}

int main() {
    layout<64>();
    layout<128>();
    bounds();
    refusals();
    return g_bad != 0;
}

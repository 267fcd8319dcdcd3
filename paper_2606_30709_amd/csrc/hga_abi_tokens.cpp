// Host side of the paged 4-bit cache's entry points: argument checks before any launch.
#include <hip/hip_runtime.h>

#include <climits>

#include "abi_common.hpp"
#include "hga.h"
#include "tokens_internal.hpp"

using namespace hga::abi;

namespace {

constexpr int64_t kMaxUnits = int64_t(1) << 30;  // workgroups of a launch

// The device address of the cold tier's pages.
hga_status map_cold(const hga_pool* pool, void** cold) {
    *cold = nullptr;
    if (pool->n_cold == 0) return HGA_OK;
    HGA_TRY(check_tensor(pool->cold, "pool.cold"));
    const hipError_t e = hipHostGetDevicePointer(cold, pool->cold, 0);
    if (e != hipSuccess) {
        (void)hipGetLastError();  // the failed lookup must not surface at a later launch
        return fail(HGA_EINVAL, "pool.cold is not a mapped pinned host allocation (%s)", hipGetErrorString(e));
    }
    if (!aligned(*cold, 16)) return fail(HGA_EALIGN, "pool.cold's mapping is not 16-byte aligned");
    return HGA_OK;
}

hga_status check_pool(const hga_pool* pool) {
    if (!pool) return fail(HGA_EINVAL, "pool is NULL");
    if (pool->n_layers < 1) return fail(HGA_EINVAL, "pool.n_layers must be >= 1");
    if (pool->n_pages < 0 || pool->n_cold < 0)
        return fail(HGA_EINVAL, "pool.n_pages and pool.n_cold must be >= 0");
    if (static_cast<int64_t>(pool->n_pages) + pool->n_cold > INT32_MAX)
        return fail(HGA_EUNSUPPORTED, "a pool of more than 2^31 - 1 pages is not supported");
    if (pool->n_pages > 0) HGA_TRY(check_tensor(pool->pages, "pool.pages"));
    if (pool->n_pages + pool->n_cold > 0) HGA_TRY(check_tensor(pool->page_sum, "pool.page_sum"));
    return HGA_OK;
}

// One layer of the pool, by device addresses.
hga_status view_pool(const hga_plan* plan, const hga_pool* pool, int32_t layer, hga::PoolView* v) {
    HGA_TRY(check_pool(pool));
    if (layer < 0 || layer >= pool->n_layers)
        return fail(HGA_EINVAL, "layer %d is outside the pool's %d", layer, pool->n_layers);
    void* cold = nullptr;
    HGA_TRY(map_cold(pool, &cold));
    const hga_params& p = plan->p;
    v->page_bytes = static_cast<int64_t>(p.n_kv_heads) * hga::page_head_bytes(p.head_dim);
    v->n_hot = pool->n_pages;
    v->n_cold = pool->n_cold;
    v->n_kv = p.n_kv_heads;
    v->hot = static_cast<unsigned char*>(pool->pages);
    if (v->hot) v->hot += layer * v->page_bytes * v->n_hot;
    v->cold = static_cast<unsigned char*>(cold);
    if (v->cold) v->cold += layer * v->page_bytes * v->n_cold;
    v->sum = pool->page_sum;
    if (v->sum)
        v->sum += static_cast<int64_t>(layer) * (static_cast<int64_t>(v->n_hot) + v->n_cold) * p.n_kv_heads * p.head_dim;
    return HGA_OK;
}

hga_status check_counts(const hga_plan* plan, int32_t n_tokens, int32_t n_seqs, int32_t max_pages) {
    if (n_tokens < 0 || n_seqs < 0 || max_pages < 0)
        return fail(HGA_EINVAL, "n_tokens, n_seqs and max_pages must be >= 0");
    if (max_pages > hga::kMaxSeqPages)
        return fail(HGA_EUNSUPPORTED, "max_pages %d above %d is not supported", max_pages, hga::kMaxSeqPages);
    if (static_cast<int64_t>(n_tokens) * plan->p.n_kv_heads > kMaxUnits)
        return fail(HGA_EUNSUPPORTED, "n_tokens * n_kv_heads above 2^30 is not supported");
    return HGA_OK;
}

hga_status view_tokens(const hga_plan* plan, const hga_tokens* tok, const hga::PoolView& pool, hga::TokensView* v) {
    if (!tok) return fail(HGA_EINVAL, "tokens is NULL");
    HGA_TRY(check_counts(plan, tok->n_tokens, tok->n_seqs, tok->max_pages));
    if (tok->n_tokens > 0) {
        HGA_TRY(check_index(tok->tok_seq, "tokens.tok_seq"));
        HGA_TRY(check_index(tok->tok_pos, "tokens.tok_pos"));
        if (tok->n_seqs > 0 && tok->max_pages > 0) HGA_TRY(check_index(tok->page_table, "tokens.page_table"));
    }
    *v = hga::TokensView{tok->tok_seq, tok->tok_pos, tok->page_table, tok->n_tokens, tok->n_seqs, tok->max_pages};
    // without a page every one is absent, and so every token as an idle one; the kernels count on a first page
    if (static_cast<int64_t>(pool.n_hot) + pool.n_cold == 0) v->max_pages = 0;
    return HGA_OK;
}

// Rows of n_heads * head_dim elements, `stride` elements from token to token.
hga_status check_rows(const hga_plan* plan, int n_tokens, const void* x, int64_t stride, int n_heads, const char* name) {
    HGA_TRY(check_tensor(x, name));
    const int64_t elt = plan->p.dtype == HGA_F32 ? 4 : 2;
    if (stride < static_cast<int64_t>(n_heads) * plan->p.head_dim)
        return fail(HGA_EINVAL, "%s: a token stride of %lld elements is below a row's %d", name,
                    static_cast<long long>(stride), n_heads * plan->p.head_dim);
    // no address space holds rows that far apart
    if (stride > (int64_t(1) << 46) / n_tokens)
        return fail(HGA_EINVAL, "%s: %d rows %lld elements apart", name, n_tokens, static_cast<long long>(stride));
    if (stride * elt % 16 != 0)
        return fail(HGA_EALIGN, "%s: a token stride of %lld elements is not a multiple of 16 bytes", name,
                    static_cast<long long>(stride));
    return HGA_OK;
}

constexpr int32_t kMaxList = 1 << 20;

hga_status check_list(int32_t n_list) {
    if (n_list > kMaxList) return fail(HGA_EUNSUPPORTED, "n_list %d above %d is not supported", n_list, kMaxList);
    return HGA_OK;
}

// Chunks a token's list holds at most.
int64_t list_size(const hga_plan* plan) {
    return static_cast<int64_t>(plan->p.keep_first) + hga::recent_window(plan->p) + plan->p.topk_chunks + 1;
}

}  // namespace

extern "C" {

int64_t hga_page_bytes(const hga_plan* plan) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    return static_cast<int64_t>(plan->p.n_kv_heads) * hga::page_head_bytes(plan->p.head_dim);
}

int32_t hga_token_list_size(const hga_plan* plan) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    const int64_t n = list_size(plan);
    if (n > kMaxList) return fail(HGA_EUNSUPPORTED, "lists of more than %d chunks are not supported", kMaxList);
    return static_cast<int32_t>(n);
}

hga_status hga_cache_append(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                            const void* k, int64_t k_stride, const void* v, int64_t v_stride, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    if (tv.n_tokens == 0) return HGA_OK;
    HGA_TRY(check_rows(plan, tv.n_tokens, k, k_stride, plan->p.n_kv_heads, "k"));
    HGA_TRY(check_rows(plan, tv.n_tokens, v, v_stride, plan->p.n_kv_heads, "v"));
    clear_stale_error();
    return launched(hga::launch_cache_append(*plan, pv, tv, k, k_stride, v, v_stride, static_cast<hipStream_t>(stream)),
                    "hga_cache_append launch");
}

hga_status hga_cache_read(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                          void* k_out, void* v_out, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    if (tv.n_tokens == 0) return HGA_OK;
    HGA_TRY(check_tensor(k_out, "k_out"));
    HGA_TRY(check_tensor(v_out, "v_out"));
    clear_stale_error();
    return launched(hga::launch_cache_read(*plan, pv, tv, k_out, v_out, static_cast<hipStream_t>(stream)),
                    "hga_cache_read launch");
}

int64_t hga_route_tokens_workspace(const hga_plan* plan, int32_t n_tokens, int32_t max_pages) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    HGA_TRY(check_counts(plan, n_tokens, 0, max_pages));
    return hga::route_tokens_bytes(*plan, n_tokens, max_pages, false);
}

hga_status hga_route_tokens(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                            const void* q, int64_t q_stride, int32_t* chunk_list, int32_t n_list, void* workspace,
                            int64_t workspace_bytes, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    HGA_TRY(check_list(n_list));
    if (n_list < list_size(plan))
        return fail(HGA_EINVAL, "n_list %d is below the %lld chunks a token may list", n_list,
                    static_cast<long long>(list_size(plan)));
    HGA_TRY(check_workspace(workspace, workspace_bytes));
    if (tv.n_tokens == 0) return HGA_OK;
    HGA_TRY(check_rows(plan, tv.n_tokens, q, q_stride, plan->p.n_q_heads, "q"));
    HGA_TRY(check_index(chunk_list, "chunk_list"));
    const int64_t need = hga::route_tokens_bytes(*plan, tv.n_tokens, tv.max_pages, true);
    if (workspace_bytes < need)
        return fail(HGA_EINVAL, "workspace of %lld bytes is below the %lld needed",
                    static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    clear_stale_error();
    return launched(hga::launch_route_tokens(*plan, pv, tv, q, q_stride, chunk_list, n_list, workspace,
                                             workspace_bytes, static_cast<hipStream_t>(stream)),
                    "hga_route_tokens launch");
}

int64_t hga_attend_tokens_workspace(const hga_plan* plan, int32_t n_tokens, int32_t n_seqs, int32_t max_pages,
                                    int32_t n_list) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    HGA_TRY(check_counts(plan, n_tokens, n_seqs, max_pages));
    if (n_list < 0) return fail(HGA_EINVAL, "n_list must be >= 0");
    HGA_TRY(check_list(n_list));
    return hga::attend_tokens_bytes(*plan, n_tokens, n_seqs, max_pages, n_list);
}

hga_status hga_attend_tokens(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                             const void* q, int64_t q_stride, const int32_t* chunk_list, int32_t n_list, void* out,
                             float* lse, void* workspace, int64_t workspace_bytes, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    if (n_list < 0) return fail(HGA_EINVAL, "n_list must be >= 0");
    HGA_TRY(check_list(n_list));
    HGA_TRY(check_workspace(workspace, workspace_bytes));
    if (tv.n_tokens == 0) return HGA_OK;
    if ((chunk_list != nullptr) != (n_list > 0))
        return fail(HGA_EINVAL, "chunk_list and n_list: a list of n_list >= 1 entries, or NULL and 0");
    HGA_TRY(check_rows(plan, tv.n_tokens, q, q_stride, plan->p.n_q_heads, "q"));
    HGA_TRY(check_tensor(out, "out"));
    if (chunk_list) HGA_TRY(check_index(chunk_list, "chunk_list"));
    if (lse) HGA_TRY(check_index(lse, "lse"));
    clear_stale_error();
    return launched(hga::launch_attend_tokens(*plan, pv, tv, q, q_stride, chunk_list, n_list, out, lse, workspace,
                                              workspace_bytes, static_cast<hipStream_t>(stream)),
                    "hga_attend_tokens launch");
}

hga_status hga_copy_pages(const hga_plan* plan, const hga_pool* pool, const int32_t* src, const int32_t* dst, int32_t n,
                          void* stream) {
    HGA_TRY(check_plan(plan));
    HGA_TRY(check_pool(pool));
    if (n < 0) return fail(HGA_EINVAL, "n must be >= 0");
    if (n == 0 || pool->n_pages + pool->n_cold == 0) return HGA_OK;
    HGA_TRY(check_index(src, "src"));
    HGA_TRY(check_index(dst, "dst"));
    void* cold = nullptr;
    HGA_TRY(map_cold(pool, &cold));
    if (static_cast<int64_t>(n) * pool->n_layers > kMaxUnits)
        return fail(HGA_EUNSUPPORTED, "%d pages of %d layers in one call are not supported", n, pool->n_layers);
    clear_stale_error();
    return launched(hga::launch_copy_pages(*plan, *pool, cold, src, dst, n, static_cast<hipStream_t>(stream)),
                    "hga_copy_pages launch");
}

}  // extern "C"

// Host side of the paged 4-bit cache's entry points: argument checks before any launch.
#include "abi_tokens.hpp"

using namespace hga::abi;

namespace {

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

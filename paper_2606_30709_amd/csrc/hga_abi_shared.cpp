// Host side of the entry points for shared prefixes and eviction: argument checks before any launch.
#include "abi_tokens.hpp"
#include "prefixes.hpp"

using namespace hga::abi;

namespace {

constexpr int32_t kMaxGroups = 1 << 20;

// The hints as the launcher takes them: within the table, and with no bound given the table's width.
int32_t hint(int32_t pages, int32_t max_pages) { return pages <= 0 || pages > max_pages ? max_pages : pages; }

hga_status check_groups(const hga_plan* plan, int32_t n_tokens, int32_t n_groups, int32_t shared_hint, int32_t own_hint) {
    if (n_groups < 0) return fail(HGA_EINVAL, "prefixes.n_groups must be >= 0");
    if (n_groups > kMaxGroups) return fail(HGA_EUNSUPPORTED, "%d groups, above %d, are not supported", n_groups, kMaxGroups);
    if (shared_hint < 0 || own_hint < 0)
        return fail(HGA_EINVAL, "prefixes.shared_hint and prefixes.own_hint must be >= 0 (0: not known)");
    if (static_cast<int64_t>(n_tokens) * plan->p.n_q_heads > kMaxUnits)
        return fail(HGA_EUNSUPPORTED, "n_tokens * n_q_heads above 2^30 is not supported");
    return HGA_OK;
}

}  // namespace

extern "C" {

int64_t hga_attend_shared_workspace(const hga_plan* plan, int32_t n_tokens, int32_t n_seqs, int32_t max_pages,
                                    int32_t n_groups, int32_t shared_hint, int32_t own_hint) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    HGA_TRY(check_counts(plan, n_tokens, n_seqs, max_pages));
    HGA_TRY(check_groups(plan, n_tokens, n_groups, shared_hint, own_hint));
    const int32_t shared = hint(shared_hint, max_pages), own = hint(own_hint, max_pages);
    return hga::attend_shared_pays(*plan, n_tokens, n_seqs, max_pages, n_groups, shared)
               ? hga::attend_shared_bytes(*plan, n_tokens, n_seqs, max_pages, n_groups, shared, own, false)
               : hga::attend_tokens_bytes(*plan, n_tokens, n_seqs, max_pages, 0);
}

hga_status hga_attend_shared(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                             const hga_prefixes* prefixes, const void* q, int64_t q_stride, void* out, float* lse,
                             void* workspace, int64_t workspace_bytes, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    if (!prefixes) return fail(HGA_EINVAL, "prefixes is NULL");
    HGA_TRY(check_groups(plan, tv.n_tokens, prefixes->n_groups, prefixes->shared_hint, prefixes->own_hint));
    HGA_TRY(check_workspace(workspace, workspace_bytes));
    if (tv.n_tokens == 0) return HGA_OK;
    HGA_TRY(check_index(prefixes->order, "prefixes.order"));
    if (prefixes->n_groups > 0) {
        HGA_TRY(check_index(prefixes->group_begin, "prefixes.group_begin"));
        HGA_TRY(check_index(prefixes->group_pages, "prefixes.group_pages"));
    }
    HGA_TRY(check_rows(plan, tv.n_tokens, q, q_stride, plan->p.n_q_heads, "q"));
    HGA_TRY(check_tensor(out, "out"));
    if (lse) HGA_TRY(check_index(lse, "lse"));
    const int shared = hint(prefixes->shared_hint, tv.max_pages), own = hint(prefixes->own_hint, tv.max_pages);
    clear_stale_error();
    // token by token where sharing does not pay, or without room for a partial result each of the groups' and the tokens' own
    // pages
    if (!hga::attend_shared_pays(*plan, tv.n_tokens, tv.n_seqs, tv.max_pages, prefixes->n_groups, shared) ||
        workspace_bytes <
            hga::attend_shared_bytes(*plan, tv.n_tokens, tv.n_seqs, tv.max_pages, prefixes->n_groups, shared, own, true))
        return launched(hga::launch_attend_tokens(*plan, pv, tv, q, q_stride, nullptr, 0, out, lse, workspace,
                                                  workspace_bytes, static_cast<hipStream_t>(stream)),
                        "hga_attend_shared launch");
    const hga::PrefixView px{prefixes->order, prefixes->group_begin, prefixes->group_pages, prefixes->n_groups};
    return launched(hga::launch_attend_shared(*plan, pv, tv, px, shared, own, q, q_stride, out, lse, workspace,
                                              workspace_bytes, static_cast<hipStream_t>(stream)),
                    "hga_attend_shared launch");
}

int64_t hga_weigh_pages_workspace(const hga_plan* plan, int32_t n_tokens, int32_t n_seqs, int32_t max_pages,
                                  int32_t n_list) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    HGA_TRY(check_counts(plan, n_tokens, n_seqs, max_pages));
    if (n_list < 0) return fail(HGA_EINVAL, "n_list must be >= 0");
    HGA_TRY(check_list(n_list));
    return hga::weigh_pages_bytes(*plan, n_tokens, n_seqs, max_pages, n_list);
}

hga_status hga_weigh_pages(const hga_plan* plan, const hga_pool* pool, int32_t layer, const hga_tokens* tokens,
                           const void* q, int64_t q_stride, const float* lse, const int32_t* chunk_list, int32_t n_list,
                           const float* prev, float* weights, void* workspace, int64_t workspace_bytes, void* stream) {
    HGA_TRY(check_plan(plan));
    hga::PoolView pv;
    hga::TokensView tv;
    HGA_TRY(view_pool(plan, pool, layer, &pv));
    HGA_TRY(view_tokens(plan, tokens, pv, &tv));
    if (n_list < 0) return fail(HGA_EINVAL, "n_list must be >= 0");
    HGA_TRY(check_list(n_list));
    if ((chunk_list != nullptr) != (n_list > 0) && tv.n_tokens > 0)
        return fail(HGA_EINVAL, "chunk_list and n_list: a list of n_list >= 1 entries, or NULL and 0");
    HGA_TRY(check_workspace(workspace, workspace_bytes));
    // the weights are those of the whole table, whatever the pool holds
    tv.max_pages = tokens->max_pages;
    const int64_t cells = static_cast<int64_t>(tv.n_seqs) * plan->p.n_kv_heads;
    if (cells == 0 || tv.max_pages == 0) return HGA_OK;
    if (cells > kMaxUnits || cells * tv.max_pages > kMaxUnits * 256)
        return fail(HGA_EUNSUPPORTED, "weights of more than 2^38 entries, or 2^30 rows, are not supported");
    HGA_TRY(check_index(weights, "weights"));
    if (prev) HGA_TRY(check_index(prev, "prev"));
    if (tv.n_tokens > 0) {
        HGA_TRY(check_rows(plan, tv.n_tokens, q, q_stride, plan->p.n_q_heads, "q"));
        HGA_TRY(check_index(lse, "lse"));
        if (chunk_list) HGA_TRY(check_index(chunk_list, "chunk_list"));
    }
    clear_stale_error();
    return launched(hga::launch_weigh_pages(*plan, pv, tv, q, q_stride, lse, chunk_list, n_list, prev, weights, workspace,
                                            workspace_bytes, static_cast<hipStream_t>(stream)),
                    "hga_weigh_pages launch");
}

int64_t hga_choose_evictions_workspace(const hga_plan* plan, int32_t n_seqs, int32_t max_pages) {
    if (!plan) return fail(HGA_EINVAL, "plan is NULL");
    HGA_TRY(check_counts(plan, 0, n_seqs, max_pages));
    return hga::choose_evictions_bytes(n_seqs, max_pages);
}

hga_status hga_choose_evictions(const hga_plan* plan, const int32_t* page_table, int32_t n_seqs, int32_t max_pages,
                                int32_t n_ids, const int32_t* seq_len, const float* weights, const int32_t* budget,
                                int32_t* evicted, int32_t n_evict, void* workspace, int64_t workspace_bytes,
                                void* stream) {
    HGA_TRY(check_plan(plan));
    HGA_TRY(check_counts(plan, 0, n_seqs, max_pages));
    if (n_ids < 0 || n_evict < 0) return fail(HGA_EINVAL, "n_ids and n_evict must be >= 0");
    HGA_TRY(check_workspace(workspace, workspace_bytes));
    if (n_seqs == 0 || n_evict == 0) return HGA_OK;
    if (n_seqs > kMaxUnits) return fail(HGA_EUNSUPPORTED, "n_seqs above 2^30 is not supported");
    HGA_TRY(check_index(evicted, "evicted"));
    HGA_TRY(check_index(seq_len, "seq_len"));
    HGA_TRY(check_index(budget, "budget"));
    if (max_pages > 0) {
        HGA_TRY(check_index(page_table, "page_table"));
        HGA_TRY(check_index(weights, "weights"));
    }
    const int64_t need = hga::choose_evictions_bytes(n_seqs, max_pages);
    if (workspace_bytes < need)
        return fail(HGA_EINVAL, "workspace of %lld bytes is below the %lld needed",
                    static_cast<long long>(workspace_bytes), static_cast<long long>(need));
    clear_stale_error();
    return launched(hga::launch_choose_evictions(*plan, page_table, n_seqs, max_pages, n_ids, seq_len, weights, budget,
                                                 evicted, n_evict, workspace, workspace_bytes,
                                                 static_cast<hipStream_t>(stream)),
                    "hga_choose_evictions launch");
}

}  // extern "C"

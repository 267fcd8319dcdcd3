// Argument checks of the paged 4-bit cache's entry points: pool, tokens and strided rows, before any launch.
#pragma once

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

}  // namespace

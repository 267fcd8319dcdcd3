// Internal declarations of the paged 4-bit cache's calls, shared by the host ABI and the kernel launchers.
#pragma once

#include "hga_internal.hpp"
#include "prefixes.hpp"
#include "tokens.hpp"

namespace hga {

// The plan's phase table of a whole page, [2][chunk][head_dim/2]: cos then sin of phi_p(o), span = chunk.  It lies behind the
// group tables.
inline float* phase_chunk(const hga_plan& plan) {
    return plan.phase_psi + 2 * (plan.p.chunk / plan.p.group) * (plan.p.head_dim / 2);
}

// The paged 4-bit cache: appending tokens (and summarising the
// pages they fill), reading rows back, copying pages.  cold: the device
// address of the pool's cold tier.
hipError_t launch_cache_append(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                               const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                               hipStream_t stream);
hipError_t launch_cache_read(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                             void* k, void* v, hipStream_t stream);
hipError_t launch_copy_pages(const hga_plan& plan, const hga_pool& pool, void* cold,
                             const int32_t* src, const int32_t* dst, int n, hipStream_t stream);

// Routing of single tokens to pages, and the workspace bytes it makes use of
// (or cannot do without).
int64_t route_tokens_bytes(const hga_plan& plan, int n_tokens, int max_pages, bool must);
hipError_t launch_route_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                               const void* q, int64_t q_stride, int32_t* list, int n_list, void* ws,
                               int64_t ws_bytes, hipStream_t stream);

// Attention of single tokens over listed pages (list NULL: all), and the
// bytes its workspace may take.
int64_t attend_tokens_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages,
                            int n_list);
hipError_t launch_attend_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                                const void* q, int64_t q_stride, const int32_t* list, int n_list,
                                void* out, float* lse, void* ws, int64_t ws_bytes,
                                hipStream_t stream);

// Attention over prefixes that sequences share, the bytes its workspace may
// take (must: the fewest with which anything is shared), whether it pays, the
// pages' attention weight, and the choice of pages to evict.
int64_t attend_shared_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages,
                            int n_groups, int shared_hint, int own_hint, bool must);
bool attend_shared_pays(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups,
                        int shared_hint);
hipError_t launch_attend_shared(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                                const PrefixView& prefixes, int shared_hint, int own_hint,
                                const void* q, int64_t q_stride, void* out, float* lse, void* ws,
                                int64_t ws_bytes, hipStream_t stream);
int64_t weigh_pages_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_list);
hipError_t launch_weigh_pages(const hga_plan& plan, const PoolView& pool, const TokensView& tok,
                              const void* q, int64_t q_stride, const float* lse, const int32_t* list,
                              int n_list, const float* prev, float* weights, void* ws,
                              int64_t ws_bytes, hipStream_t stream);
int64_t choose_evictions_bytes(int n_seqs, int max_pages);
hipError_t launch_choose_evictions(const hga_plan& plan, const int32_t* table, int n_seqs,
                                   int max_pages, int n_ids, const int32_t* seq_len,
                                   const float* weights, const int32_t* budget, int32_t* evicted,
                                   int n_evict, void* ws, int64_t ws_bytes, hipStream_t stream);

}  // namespace hga

// Sequences that share leading pages: how a call's tokens stand in groups, and how a call's work is cut.
#pragma once

#include "tokens.hpp"

namespace hga {

// Slot i holds token order[i]; slots [begin[g], begin[g + 1]) are the tokens of group g, which share their first pages[g]
// pages.  Every word may hold anything: what these functions return stays inside the call.
struct PrefixView {
    const int32_t* order;
    const int32_t* begin;
    const int32_t* pages;
    int n_groups;

    __host__ __device__ static int clamp(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
    // Token of slot i, or -1.
    __host__ __device__ int token(int i, int n_tokens) const {
        const int t = order[i];
        return static_cast<uint32_t>(t) < static_cast<uint32_t>(n_tokens) ? t : -1;
    }
    __host__ __device__ int first(int g, int n_tokens) const { return clamp(begin[g], 0, n_tokens); }
    __host__ __device__ int end(int g, int n_tokens) const { return clamp(begin[g + 1], first(g, n_tokens), n_tokens); }
    __host__ __device__ int shared(int g, int max_pages) const { return clamp(pages[g], 0, max_pages); }
};

// Runs of `run` pages that n pages are cut into, at most `most` (the last then takes what is left).
__host__ __device__ inline int runs_of(int n, int run, int most) {
    if (n <= 0) return 0;
    const int r = (n - 1) / run + 1;
    return r < most ? r : most;
}
// Pages [a, b) of run j, of n in all.
struct PageRun {
    int a, b;
};
__host__ __device__ inline PageRun page_run(int j, int n, int run, int most) {
    const int r = runs_of(n, run, most);
    if (j >= r) return PageRun{0, 0};
    return PageRun{j * run, j + 1 == r ? n : (j + 1) * run};
}

}  // namespace hga

// The pages to evict from each sequence: of its middle pages those with the least attention weight.
//
// A workgroup a sequence.  A page's key is its weight, summed over the KV heads in 64 bits, as an integer of the same order;
// the border of the choice is found digit by digit from the top (a histogram of the digit's 256 values each), then the
// pages below it, and of those at it the first, are listed in order.
#include <algorithm>

#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

struct ChooseArgs {
    const int32_t* table;
    int max_pages, n_ids, n_kv;
    int first, window;  // pages that stay: the first ones, and the last ones before a sequence's last
    const int32_t* seq_len;
    const float* weights;
    const int32_t* budget;
    int32_t* evicted;
    int n_evict;
    uint64_t* keys;  // [n_seqs][max_pages]
};

// A double as an integer of the same order; what is not a number comes first.
__device__ __forceinline__ uint64_t order_key(double x) {
    if (x != x) return 0;
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));  // -0 as +0
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}

// Inclusive sum over the workgroup of x (small counts), and the total.
__device__ __forceinline__ int block_scan(int x, int32_t* s_sum, int& total) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int in = wave_incl_scan_add(x);
    __syncthreads();
    if (lane == 63) s_sum[wave] = in;
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < kWaves; ++w) {
        if (w < wave) before += s_sum[w];
        total += s_sum[w];
    }
    return before + in;
}

__global__ __launch_bounds__(kThreads) void choose_kernel(ChooseArgs a, int n_seqs) {
    __shared__ int32_t s_sum[kWaves], s_hist[256], s_pick[2];
    const int s = static_cast<int>(linear_block<kThreads>()), tid = threadIdx.x;
    if (s >= n_seqs) return;
    const int32_t* table = a.table + static_cast<int64_t>(s) * a.max_pages;
    const float* weights = a.weights + static_cast<int64_t>(s) * a.n_kv * a.max_pages;
    uint64_t* keys = a.keys + static_cast<int64_t>(s) * a.max_pages;
    int32_t* out = a.evicted + static_cast<int64_t>(s) * a.n_evict;
    const int len = a.seq_len[s];
    // positions past the table have no page: such a sequence is none
    const int last = len > 0 && (len - 1) / kPageRows < a.max_pages ? (len - 1) / kPageRows : -1;
    const int lo = min(a.first, last), hi = max(lo, last - a.window);  // middle chunks [lo, hi)
    int here = 0, may = 0;
    for (int c = tid; c <= last; c += kThreads) {
        const bool present = static_cast<uint32_t>(table[c]) < static_cast<uint32_t>(a.n_ids);
        here += present;
        uint64_t key = ~uint64_t(0);
        if (present && c >= lo && c < hi) {
            ++may;
            double sum = 0.0;
            for (int h = 0; h < a.n_kv; ++h) sum += static_cast<double>(weights[static_cast<int64_t>(h) * a.max_pages + c]);
            key = order_key(sum);
        }
        keys[c] = key;
    }
    int n_here, n_may;
    block_scan(here, s_sum, n_here);
    block_scan(may, s_sum, n_may);
    const int64_t over = static_cast<int64_t>(n_here) - a.budget[s];
    const int n = last < 0 ? 0 : static_cast<int>(min(max(over, int64_t(0)), static_cast<int64_t>(min(n_may, a.n_evict))));
    // the n-th smallest key, from the top digit down; `rest` of those equal to it so far are wanted
    uint64_t border = 0;
    int rest = n;
    for (int shift = 56; n > 0 && shift >= 0; shift -= 8) {
        __syncthreads();
        if (tid < 256) s_hist[tid] = 0;
        __syncthreads();
        for (int c = tid; c < hi; c += kThreads) {
            const uint64_t key = keys[c];
            if (key != ~uint64_t(0) && (shift == 56 || key >> (shift + 8) == border >> (shift + 8)))
                atomicAdd(&s_hist[key >> shift & 255], 1);
        }
        __syncthreads();
        int total;
        const int mine = tid < 256 ? s_hist[tid] : 0, to = block_scan(mine, s_sum, total);
        if (tid < 256 && to >= rest && to - mine < rest) {
            s_pick[0] = tid;
            s_pick[1] = rest - (to - mine);
        }
        __syncthreads();
        border |= static_cast<uint64_t>(s_pick[0]) << shift;
        rest = s_pick[1];
    }
    int done = 0, ties = 0;
    for (int c0 = 0; n > 0 && c0 < hi; c0 += kThreads) {
        const int c = c0 + tid;
        const uint64_t key = c < hi ? keys[c] : ~uint64_t(0);
        const bool tie = key == border && key != ~uint64_t(0);
        int n_tie, n_take;
        const int tie_at = ties + block_scan(tie, s_sum, n_tie);
        const bool take = key < border || (tie && tie_at <= rest);
        const int at = done + block_scan(take, s_sum, n_take) - 1;
        if (take) out[at] = c;
        ties += n_tie;
        done += n_take;
    }
    for (int i = n + tid; i < a.n_evict; i += kThreads) out[i] = -1;
}

}  // namespace

int64_t choose_evictions_bytes(int n_seqs, int max_pages) { return static_cast<int64_t>(n_seqs) * max_pages * 8; }

hipError_t launch_choose_evictions(const hga_plan& plan, const int32_t* table, int n_seqs, int max_pages, int n_ids,
                                   const int32_t* seq_len, const float* weights, const int32_t* budget, int32_t* evicted,
                                   int n_evict, void* ws, int64_t, hipStream_t stream) {
    const ChooseArgs a{table,  max_pages, n_ids,   plan.p.n_kv_heads, plan.p.keep_first, recent_window(plan.p), seq_len,
                       weights, budget,   evicted, n_evict,           static_cast<uint64_t*>(ws)};
    choose_kernel<<<grid_of(n_seqs, kThreads), kThreads, 0, stream>>>(a, n_seqs);
    return hipGetLastError();
}

}  // namespace hga

// The pages to evict from each sequence: of its middle pages those with the least attention weight.
//
// A workgroup a sequence.  A page's key is its weight, summed over the KV heads in 64 bits, as an integer of the same order.
// The border of the choice (the n-th smallest key) lies between the smallest and the largest; a histogram over the 2,048
// values of the digit below what these two have in common names the one it is in, whose smallest and largest keys are
// next, until all that are left of it are taken or are equal.  The pages below the border, and of those at it the first, are
// then listed in order, placed by the counts of each wavefront's 64 neighbouring pages.
//
// Up to 16,384 pages the keys stay in registers; of longer tables they lie in the workspace.
//
// Bound by latency, and for long tables by one CU's arithmetic: 2,048 pages of 4 heads 11.5 us (loads 1.0, counts 1.2, two
// rounds of 2.5, the list 0.9), 8 times 16,384 pages of 8 heads 30 us (loads and sums 7, two or three rounds of 4, the list 3;
// with the keys in memory 72, with 64-bit shuffles for the ends of the range and a head's weights at a time 33).
#include <algorithm>
#include <type_traits>

#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kDigit = 11, kBins = 1 << kDigit;
constexpr int kMostHeld = 16;  // keys of a thread in registers
constexpr uint64_t kNone = ~uint64_t(0);  // no page to evict (as a key: a NaN, which order_key does not return)

struct ChooseArgs {
    const int32_t* table;
    int max_pages, n_ids, n_kv;
    int first, window;  // pages that stay: the first ones, and the last ones before a sequence's last
    const int32_t* seq_len;
    const float* weights;
    const int32_t* budget;
    int32_t* evicted;
    int n_evict;
    int per_thread;  // pages of a thread, where they are not a constant
    uint64_t* keys;  // [n_seqs][per_thread][kThreads]
};

// A double as an integer of the same order; what is not a number comes first.
__device__ __forceinline__ uint64_t order_key(double x) {
    if (x != x) return 0;
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x + 0.0));  // -0 as +0
    return u >> 63 ? ~u : u | uint64_t(1) << 63;
}

// Sum over the workgroup of a count before this thread's, and in all.
struct Sums {
    int before, total;
};
__device__ __forceinline__ Sums block_sum(int x, int32_t* s_sum) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int in = wave_incl_scan_add(x);
    __syncthreads();
    if (lane == 63) s_sum[wave] = in;
    __syncthreads();
    const int mine = s_sum[lane & (kWaves - 1)], to = wave_incl_scan_add(lane < kWaves ? mine : 0);
    const int total = __builtin_amdgcn_readlane(to, kWaves - 1);
    const int before = wave == 0 ? 0 : __builtin_amdgcn_readlane(to, wave - 1);
    return Sums{before + in - x, total};
}
// kHeld: pages of a thread, whose keys it holds; 0: a.per_thread, in a.keys.
template <int kHeld>
__global__ __launch_bounds__(kThreads) void choose_kernel(ChooseArgs a, int n_seqs) {
    __shared__ int32_t s_sum[kWaves], s_hist[kBins], s_pick[3], s_count[kMostHeld * kWaves];
    __shared__ uint64_t s_lo[kWaves], s_hi[kWaves];
    const int s = static_cast<int>(linear_block<kThreads>()), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    if (s >= n_seqs) return;
    const int per = kHeld ? kHeld : a.per_thread;
    const int32_t* table = a.table + static_cast<int64_t>(s) * a.max_pages;
    const float* weights = a.weights + static_cast<int64_t>(s) * a.n_kv * a.max_pages;
    uint64_t* keys = a.keys + static_cast<int64_t>(s) * per * kThreads;
    int32_t* out = a.evicted + static_cast<int64_t>(s) * a.n_evict;
    const int len = a.seq_len[s];
    // positions past the table have no page: such a sequence is none
    const int last = len > 0 && (len - 1) / kPageRows < a.max_pages ? (len - 1) / kPageRows : -1;
    const int lo = min(a.first, last), hi = max(lo, last - a.window);  // middle chunks [lo, hi)
    uint64_t held[kHeld ? kHeld : 1];
    int here = 0, may = 0;
    const auto put = [&](int r, bool present, double sum) {
        const int c = r * kThreads + tid;
        here += present;
        const bool can = present && c >= lo && c < hi;
        may += can;
        const uint64_t key = can ? order_key(sum) : kNone;
        if constexpr (kHeld)
            held[r] = key;
        else
            keys[static_cast<int64_t>(r) * kThreads + tid] = key;
    };
    if constexpr (kHeld) {
        double sum[kHeld];
        bool present[kHeld];
#pragma unroll
        for (int r = 0; r < kHeld; ++r) {
            const int c = r * kThreads + tid;
            sum[r] = 0.0;
            present[r] = c <= last && static_cast<uint32_t>(table[c]) < static_cast<uint32_t>(a.n_ids);
        }
        // kHeads of a page's words on their way at once (64 tables of 2,048 pages, eight heads: 13.5 us a call a head at a
        // time, 11.5 so); a head past the last is the last one again, and is not added
        constexpr int kHeads = kHeld >= 4 ? 32 / kHeld : 8;
        for (int h0 = 0; h0 < a.n_kv && last >= 0; h0 += kHeads) {
            float x[kHeads][kHeld];
#pragma unroll
            for (int y = 0; y < kHeads; ++y) {
                const float* from = weights + static_cast<int64_t>(min(h0 + y, a.n_kv - 1)) * a.max_pages;
#pragma unroll
                for (int r = 0; r < kHeld; ++r) x[y][r] = from[min(r * kThreads + tid, last)];
            }
#pragma unroll
            for (int y = 0; y < kHeads; ++y)
                if (h0 + y < a.n_kv)
#pragma unroll
                    for (int r = 0; r < kHeld; ++r) sum[r] += static_cast<double>(x[y][r]);
        }
#pragma unroll
        for (int r = 0; r < kHeld; ++r) put(r, present[r], sum[r]);
    } else {
        for (int r = 0; r < per; ++r) {
            const int c = r * kThreads + tid;
            const bool present = c <= last && static_cast<uint32_t>(table[c]) < static_cast<uint32_t>(a.n_ids);
            double sum = 0.0;
            if (present)
                for (int h = 0; h < a.n_kv; ++h) sum += static_cast<double>(weights[static_cast<int64_t>(h) * a.max_pages + c]);
            put(r, present, sum);
        }
    }
    const auto for_keys = [&](auto f) {
        if constexpr (kHeld) {
#pragma unroll
            for (int r = 0; r < kHeld; ++r) f(r, held[r]);
        } else {
            for (int r = 0; r < per; ++r) f(r, keys[static_cast<int64_t>(r) * kThreads + tid]);
        }
    };
    const int n_here = block_sum(here, s_sum).total, n_may = block_sum(may, s_sum).total;
    const int64_t over = static_cast<int64_t>(n_here) - a.budget[s];
    const int n = last < 0 ? 0 : static_cast<int>(min(max(over, int64_t(0)), static_cast<int64_t>(min(n_may, a.n_evict))));
    // Keys in [from, to] hold the border; `rest` of their smallest are wanted.  Keys below `from` are taken.
    uint64_t from = 0, to = kNone - 1;
    int rest = n;
    bool all = n == n_may;  // every key of the range is taken
    while (n > 0 && !all) {
        // the range's smallest and largest key
        uint64_t least = kNone, most = 0;
        for_keys([&](int, uint64_t k) {
            if (k >= from && k <= to) {
                least = min(least, k);
                most = max(most, k);
            }
        });
        least = ~wave_max_u64(~least);
        most = wave_max_u64(most);
        __syncthreads();  // the last round's words have been read
        if (lane == 0) {
            s_lo[wave] = least;
            s_hi[wave] = most;
        }
        for (int i = tid; i < kBins; i += kThreads) s_hist[i] = 0;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            least = min(least, s_lo[w]);
            most = max(most, s_hi[w]);
        }
        from = least;
        to = most;
        if (from == to) break;  // the first `rest` of equal ones
        const int bits = 64 - __clzll(static_cast<long long>(from ^ to));  // below what they have in common
        const int shift = bits > kDigit ? bits - kDigit : 0;
        const uint64_t high = bits < 64 ? from >> bits << (bits - shift) : 0;
        for_keys([&](int, uint64_t k) {
            if (k >= from && k <= to) atomicAdd(&s_hist[static_cast<int>((k >> shift) - high)], 1);
        });
        __syncthreads();
        const int h0 = s_hist[2 * tid], h1 = s_hist[2 * tid + 1];
        const int before = block_sum(h0 + h1, s_sum).before;
        if (before < rest && rest <= before + h0 + h1) {
            const bool second = rest > before + h0;
            s_pick[0] = 2 * tid + second;
            s_pick[1] = second ? before + h0 : before;
            s_pick[2] = second ? h1 : h0;
        }
        __syncthreads();
        rest -= s_pick[1];
        all = rest == s_pick[2];
        const uint64_t digit = high + static_cast<uint64_t>(s_pick[0]);
        const uint64_t bin = digit << shift;
        from = max(from, bin);
        to = min(to, bin | ((uint64_t(1) << shift) - 1));
    }
    // taken: keys below `from`, and of those in the range all, or (they are equal) the first `rest`; 16 words of a thread at
    // a time, the counts of both kinds in the halves of a word
    const int limit = all ? INT32_MAX : rest;
    int below0 = 0, equal0 = 0;
    for (int r0 = 0; r0 < per && n > 0; r0 += kMostHeld) {
        const int r1 = min(r0 + kMostHeld, per);
        __syncthreads();
        for (int i = tid; i < kMostHeld * kWaves; i += kThreads) s_count[i] = 0;
        __syncthreads();
        const auto chunk = [&](auto f) {
            if constexpr (kHeld)
                for_keys(f);
            else
                for (int r = r0; r < r1; ++r) f(r, keys[static_cast<int64_t>(r) * kThreads + tid]);
        };
        chunk([&](int r, uint64_t k) {
            const int below = __popcll(__builtin_amdgcn_ballot_w64(k < from));
            const int equal = __popcll(__builtin_amdgcn_ballot_w64(k >= from && k <= to));
            if (lane == 0) s_count[(r - r0) * kWaves + wave] = below | equal << 16;
        });
        __syncthreads();
        // every wavefront adds up all counts, four a lane
        static_assert(kMostHeld * kWaves == 256, "");
        int part[4], sum = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            part[y] = sum;
            sum += s_count[4 * lane + y];
        }
        const int upto = wave_incl_scan_add(sum);
        const int total = __builtin_amdgcn_readlane(upto, 63);
#pragma unroll
        for (int y = 0; y < 4; ++y) part[y] += upto - sum;
        // the count before this wavefront's word r: entry 16 r + wave
        const int mine = (wave & 2) ? ((wave & 1) ? part[3] : part[2]) : ((wave & 1) ? part[1] : part[0]);
        const uint64_t earlier = (uint64_t(1) << lane) - 1;
        chunk([&](int r, uint64_t k) {
            const bool is_below = k < from, is_equal = k >= from && k <= to;
            const uint64_t below = __builtin_amdgcn_ballot_w64(is_below), equal = __builtin_amdgcn_ballot_w64(is_equal);
            const int before = __builtin_amdgcn_readlane(mine, 4 * (r - r0) + (wave >> 2));
            const int b = below0 + (before & 0xffff) + __popcll(below & earlier);
            const int e = equal0 + (before >> 16) + __popcll(equal & earlier);
            if (is_below || (is_equal && e < limit)) out[b + min(e, limit)] = r * kThreads + tid;
        });
        below0 += total & 0xffff;
        equal0 += total >> 16;
    }
    for (int i = n + tid; i < a.n_evict; i += kThreads) out[i] = -1;
}

int pages_of_thread(int max_pages) { return (max_pages + kThreads - 1) / kThreads; }

}  // namespace

int64_t choose_evictions_bytes(int n_seqs, int max_pages) {
    const int64_t per = pages_of_thread(max_pages);
    return per <= kMostHeld ? 0 : n_seqs * per * kThreads * 8;
}

hipError_t launch_choose_evictions(const hga_plan& plan, const int32_t* table, int n_seqs, int max_pages, int n_ids,
                                   const int32_t* seq_len, const float* weights, const int32_t* budget, int32_t* evicted,
                                   int n_evict, void* ws, int64_t, hipStream_t stream) {
    const int per = pages_of_thread(max_pages);
    const ChooseArgs a{table,   max_pages, n_ids,   plan.p.n_kv_heads, plan.p.keep_first, recent_window(plan.p), seq_len,
                       weights, budget,    evicted, n_evict,           per,               static_cast<uint64_t*>(ws)};
    const auto f = per <= 1 ? choose_kernel<1> : per <= 2 ? choose_kernel<2> : per <= 4 ? choose_kernel<4>
                   : per <= 8 ? choose_kernel<8> : per <= kMostHeld ? choose_kernel<kMostHeld> : choose_kernel<0>;
    f<<<grid_of(n_seqs, kThreads), kThreads, 0, stream>>>(a, n_seqs);
    return hipGetLastError();
}

}  // namespace hga

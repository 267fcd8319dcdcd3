// Routing of single tokens to pages (Sec. 3.3 at the token's grain): the chunks a token sees are its own, the
// deterministic ones (the first keep_first, the window before its own) and, of the middle ones, the topk_chunks whose
// page summaries have the largest products with the mean of the token's query heads.
//
// Scores are sums of 64-bit products: an fp32 score's error exceeds the gap at the border of the selection once in some
// tens of thousands of selections, a 64-bit one's practically never, and the fp64 rate of the vector unit equals its fp32
// rate, so a decode step stays bound by the summaries' bytes.  A score becomes a 64-bit key that orders as the score does;
// the K_c-th largest key is found from its most significant byte down, by counting.
#include "hga_device.hpp"
#include "hga_internal.hpp"
#include "tokens.hpp"

namespace hga {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
// Pages of a sequence up to which a unit's keys lie in LDS (128 of its 160 KiB).
constexpr int kLdsPages = 1 << 14;

// A key that orders as the score: 0 is no candidate, 1 a score that is not a number.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (s != s) return 1;
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(s + 0.0));
    return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}

struct RouteArgs {
    int first, window, topk, ratio, n_list;
};

__device__ __forceinline__ double shfl_xor_f64(double x, int mask) {
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x));
    const uint32_t lo = __shfl_xor(static_cast<uint32_t>(u), mask), hi = __shfl_xor(static_cast<uint32_t>(u >> 32), mask);
    return __longlong_as_double(static_cast<long long>(static_cast<uint64_t>(hi) << 32 | lo));
}

// The k-th largest of keys[0..n): every key k or more of which are as large is taken, of those equal to `key` the first
// `ties`.  0 < k; n candidates at least k are not 0.  All threads of the workgroup call.
struct Border {
    uint64_t key, mask;  // keys are compared under the mask
    int ties;
};
__device__ __forceinline__ Border find_border(const uint64_t* keys, int n, int k, uint32_t* hist) {
    const int tid = threadIdx.x;
    Border b{0, 0, k};
    for (int shift = 56; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t v = keys[i];
            if (v != 0 && (v & b.mask) == b.key) atomicAdd(&hist[v >> shift & 255], 1u);
        }
        __syncthreads();
        // every thread walks down from the top bin to the one that holds the border
        int bin = 255, above = 0;
        while (bin > 0 && above + static_cast<int>(hist[bin]) < b.ties) above += static_cast<int>(hist[bin--]);
        const int in = static_cast<int>(hist[bin]);
        b.key |= static_cast<uint64_t>(bin) << shift;
        b.mask |= uint64_t(255) << shift;
        b.ties -= above;
        __syncthreads();
        if (in == b.ties) break;  // all of the bin
    }
    return b;
}

// A workgroup per (token, KV head).
template <typename T, int D, bool kLds>
__global__ __launch_bounds__(kThreads) void route_tokens_kernel(PoolView pool, TokensView tok, RouteArgs a,
                                                                const T* __restrict__ q, int64_t q_stride,
                                                                int32_t* __restrict__ list, uint64_t* __restrict__ ws) {
    constexpr int kLanes = 8;               // lanes of a summary row
    constexpr int kPieces = D / 4 / kLanes;  // 16-byte pieces a lane takes of it
    extern __shared__ __align__(16) uint64_t lds_keys[];
    __shared__ uint32_t hist[256];
    __shared__ int counts[2][kWaves];
    const int64_t unit = linear_block<kThreads>();
    const int t = static_cast<int>(unit / pool.n_kv), h = static_cast<int>(unit % pool.n_kv);
    if (t >= tok.n_tokens) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int32_t* out = list + unit * a.n_list;
    int s, p;
    if (!tok.at(t, s, p)) {
        for (int i = tid; i < a.n_list; i += kThreads) out[i] = -1;
        return;
    }
    const int own = p / kPageRows;
    const int lo = min(a.first, own), hi = max(lo, own - a.window);  // middle chunks [lo, hi)
    const int n = hi - lo;
    uint64_t* keys = kLds ? lds_keys : ws + unit * tok.max_pages;

    // the lane's dimensions of the summed query heads
    double qs[kPieces * 4];
#pragma unroll
    for (int i = 0; i < kPieces * 4; ++i) qs[i] = 0.0;
    const T* qt = q + t * q_stride + static_cast<int64_t>(h) * a.ratio * D;
    for (int r = 0; r < a.ratio; ++r)
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                qs[4 * i + j] += static_cast<double>(elem<T>::to_f32(qt[r * D + (i * kLanes + (lane & 7)) * 4 + j]));

    int found = 0;
    for (int i0 = 0; i0 < n; i0 += kThreads / kLanes) {
        const int i = i0 + tid / kLanes;
        const int id = i < n ? tok.page_id(s, lo + i) : -1;
        const bool has = i < n && pool.has(id);
        double acc = 0.0;
        if (has) {
            const float* row = pool.sum + (static_cast<int64_t>(id) * pool.n_kv + h) * D;
#pragma unroll
            for (int x = 0; x < kPieces; ++x) {
                const float4 w = *reinterpret_cast<const float4*>(row + (x * kLanes + (lane & 7)) * 4);
                acc = fma(qs[4 * x], static_cast<double>(w.x), acc);
                acc = fma(qs[4 * x + 1], static_cast<double>(w.y), acc);
                acc = fma(qs[4 * x + 2], static_cast<double>(w.z), acc);
                acc = fma(qs[4 * x + 3], static_cast<double>(w.w), acc);
            }
        }
#pragma unroll
        for (int m = 1; m < kLanes; m *= 2) acc += shfl_xor_f64(acc, m);
        if ((lane & 7) == 0 && i < n) keys[i] = has ? score_key(acc) : 0;
        found += has && (lane & 7) == 0;
    }
    // candidates present
    for (int m = 1; m < 64; m *= 2) found += __shfl_xor(found, m);
    if (lane == 0) counts[0][wave] = found;
    __syncthreads();
    int total = 0;
    for (int w = 0; w < kWaves; ++w) total += counts[0][w];
    Border b{0, 0, 0};
    const bool choose = total > a.topk;
    if (choose) b = find_border(keys, n, a.topk, hist);
    __syncthreads();

    // the list in ascending order: a position's rank is the number of listed ones before it
    int base = 0, ties = 0;
    for (int c0 = 0; c0 <= own; c0 += kThreads) {
        const int c = c0 + tid;
        bool tie = false, pick = false;
        if (c <= own) {
            if (c >= lo && c < hi) {
                const uint64_t v = keys[c - lo];
                pick = v != 0 && (v & b.mask) >= b.key;
                tie = choose && pick && (v & b.mask) == b.key;
            } else {
                pick = pool.has(tok.page_id(s, c));
            }
        }
        const uint64_t below = (uint64_t(1) << lane) - 1;
        const uint64_t tm = __builtin_amdgcn_ballot_w64(tie);
        if (lane == 0) counts[0][wave] = __popcll(tm);
        __syncthreads();
        int before = ties + __popcll(tm & below);
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) before += counts[0][w];
            ties += counts[0][w];
        }
        if (tie && before >= b.ties) pick = false;
        const uint64_t pm = __builtin_amdgcn_ballot_w64(pick);
        if (lane == 0) counts[1][wave] = __popcll(pm);
        __syncthreads();
        int rank = base + __popcll(pm & below);
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) rank += counts[1][w];
            base += counts[1][w];
        }
        if (pick && rank < a.n_list) out[rank] = c;
        __syncthreads();
    }
    for (int i = base + tid; i < a.n_list; i += kThreads) out[i] = -1;
}

template <typename T, int D, bool kLds>
hipError_t run(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const RouteArgs& a, const void* q,
               int64_t q_stride, int32_t* list, void* ws, hipStream_t stream) {
    const size_t lds = kLds ? sizeof(uint64_t) * tok.max_pages : 0;
    if (kLds) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = once_per_device(done, plan.device, [] {
            return hipFuncSetAttribute(reinterpret_cast<const void*>(route_tokens_kernel<T, D, true>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(sizeof(uint64_t) * kLdsPages));
        });
        if (e != hipSuccess) return e;
    }
    const int64_t n = static_cast<int64_t>(tok.n_tokens) * pool.n_kv;
    route_tokens_kernel<T, D, kLds><<<grid_of(n, kThreads), kThreads, lds, stream>>>(
        pool, tok, a, static_cast<const T*>(q), q_stride, list, static_cast<uint64_t*>(ws));
    return hipGetLastError();
}

}  // namespace

int64_t route_tokens_bytes(const hga_plan& plan, int n_tokens, int max_pages) {
    if (max_pages <= kLdsPages) return 0;
    return static_cast<int64_t>(n_tokens) * plan.p.n_kv_heads * max_pages * static_cast<int64_t>(sizeof(uint64_t));
}

hipError_t launch_route_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                               int64_t q_stride, int32_t* list, int n_list, void* ws, hipStream_t stream) {
    RouteArgs a;
    a.first = plan.p.keep_first;
    a.window = recent_window(plan.p);
    a.topk = plan.p.topk_chunks;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.n_list = n_list;
    const bool f32 = plan.p.dtype == HGA_F32, lds = tok.max_pages <= kLdsPages;
    const auto f = plan.p.head_dim == 128
                       ? (f32 ? (lds ? run<float, 128, true> : run<float, 128, false>)
                              : (lds ? run<bf16_t, 128, true> : run<bf16_t, 128, false>))
                       : (f32 ? (lds ? run<float, 64, true> : run<float, 64, false>)
                              : (lds ? run<bf16_t, 64, true> : run<bf16_t, 64, false>));
    return f(plan, pool, tok, a, q, q_stride, list, ws, stream);
}

}  // namespace hga

// Attention weight of pages: what each page of a sequence got of the attention of a call's tokens,
//   W[s][h][c] = prev[s][h][c] + sum over tokens t of s, query heads of h, rows o of page c up to t's position of
//                exp(q . k~_o / sqrt(d) - lse),
// from the queries and the lse that their attention gave.  Only keys are read: half of a page.
//
// The weights of a (sequence, KV head) are formed by whoever owns a page of it, over all of its tokens in the call's order:
// no sum depends on what runs beside it, and no two writers meet.
#include <algorithm>
#include <type_traits>

#include "attend_pages.hpp"
#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;
constexpr int kScan = 1024;  // tokens looked at, at a time, for those of a sequence

struct WeighArgs {
    const int32_t* list;  // NULL: every chunk
    int n_list, ratio;
    int blocks;           // workgroups of a (sequence, KV head)
    const float* lse;
    const float* prev;    // NULL: zeros
    float* weights;
};

// Which of the tokens [t0, t0 + kScan) are of sequence s, in order, into LDS; how many.  Every thread calls it.
__device__ __forceinline__ int tokens_of(const TokensView& tok, int s, int t0, int32_t* s_tok, int32_t* s_count) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    __syncthreads();  // the last ones have been used
    int n = 0;
    for (int i0 = 0; i0 < kScan; i0 += kThreads) {
        const int t = t0 + i0 + tid;
        int sc = -1, pc;
        const bool mine = t < tok.n_tokens && tok.at(t, sc, pc) && sc == s;
        const uint64_t mask = __builtin_amdgcn_ballot_w64(mine);
        if (lane == 0) s_count[wave] = __popcll(mask);
        __syncthreads();
        int at = n + __popcll(mask & ((uint64_t(1) << lane) - 1));
        for (int w = 0; w < kWaves; ++w) {
            if (w < wave) at += s_count[w];
            n += s_count[w];
        }
        if (mine) s_tok[at] = t;
        __syncthreads();
    }
    return n;
}

// The queries of up to 16 columns, and what else a column needs.
template <typename T, int D, int kTerms>
struct Columns {
    u32x4 qf[1][kTerms][D / 32];
    float base;  // lse in log2 units; +inf: the column sees nothing
    int pos;
};
template <typename T, int D, int kTerms>
__device__ __forceinline__ Columns<T, D, kTerms> load_columns(const TokensView& tok, const WeighArgs& a, const T* q,
                                                              int64_t q_stride, int h, int n_kv, const int32_t* s_tok,
                                                              int c0, int columns, int m, int g) {
    Columns<T, D, kTerms> r;
    const int c = c0 + m;
    const bool real = c < columns;
    const int t = s_tok[real ? c / a.ratio : 0], head = h * a.ratio + (real ? c % a.ratio : 0);
    r.pos = real ? tok.pos[t] : -1;
    const float lse = real ? a.lse[static_cast<int64_t>(t) * n_kv * a.ratio + head] : -INFINITY;
    r.base = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
    const T* from = q + t * q_stride + static_cast<int64_t>(head) * D + g * (D / 4);
#pragma unroll
    for (int kk = 0; kk < D / 32; ++kk) {
        float x[8];
        load8(from + 8 * kk, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t w[kTerms];
            split2<kTerms>(x[2 * e], x[2 * e + 1], w);
#pragma unroll
            for (int y = 0; y < kTerms; ++y) r.qf[0][y][kk][e] = w[y];
        }
    }
    return r;
}

// A lane's share of what a page gets from 16 columns.
template <typename T, int D, int kTerms>
__device__ __forceinline__ float page_weight(const Keys<D>& k, const Columns<T, D, kTerms>& col, int chunk, int g) {
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));
    f32x4 sc[1][4];
    page_scores<D, kTerms, 1>(k, col.qf, sc);
    float sum = 0.f;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = chunk * kPageRows + 16 * tt + 4 * g + x;
            const float p = __builtin_amdgcn_exp2f(fmaf(sc[0][tt][x], scale, -col.base));
            sum += row <= col.pos && col.base != INFINITY ? p : 0.f;
        }
    return sum;
}
__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
    return x;
}

// Whole histories: a wavefront a page at a time.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void weigh_kernel(PoolView pool, TokensView tok, WeighArgs a,
                                                         const T* __restrict__ q, int64_t q_stride) {
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    using F = PageFormat<D>;
    __shared__ int32_t s_tok[kScan], s_count[kWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const uint32_t block = linear_block<kThreads>();
    const auto [sb, h] = token_head(block, pool.n_kv);
    const int s = sb / a.blocks, part = sb % a.blocks;
    if (s >= tok.n_seqs) return;
    const int64_t at = (static_cast<int64_t>(s) * pool.n_kv + h) * tok.max_pages;
    for (int c = part * kWaves + wave; c < tok.max_pages; c += a.blocks * kWaves)
        if (lane == 0) a.weights[at + c] = a.prev ? a.prev[at + c] : 0.f;
    for (int t0 = 0; t0 < tok.n_tokens; t0 += kScan) {
        const int n = tokens_of(tok, s, t0, s_tok, s_count);
        int last = -1;
        for (int i = 0; i < n; ++i) last = max(last, tok.pos[s_tok[i]]);
        for (int c = part * kWaves + wave; c < tok.max_pages && c <= last / kPageRows && last >= 0; c += a.blocks * kWaves) {
            const SeenPage p = seen_page(pool, tok, s, last, c);
            if (p.rows == 0) continue;
            Keys<D> k;
            load_keys<D>(make_rsrc(pool.page(p.id) + h * F::kBytes, F::kBytes), m, g, k);
            float sum = 0.f;
            for (int c0 = 0; c0 < n * a.ratio; c0 += 16) {
                const auto col = load_columns<T, D, kTerms>(tok, a, q, q_stride, h, pool.n_kv, s_tok, c0, n * a.ratio, m, g);
                sum += page_weight<T, D, kTerms>(k, col, c, g);
            }
            sum = wave_sum(sum);
            if (lane == 0) a.weights[at + c] += sum;
        }
    }
}

// Listed pages: a workgroup owns every a.blocks-th line of 16 pages, its wavefronts every kWaves-th page of those.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void weigh_listed_kernel(PoolView pool, TokensView tok, WeighArgs a,
                                                                const T* __restrict__ q, int64_t q_stride) {
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    using F = PageFormat<D>;
    __shared__ int32_t s_tok[kScan], s_count[kWaves];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const uint32_t block = linear_block<kThreads>();
    const auto [sb, h] = token_head(block, pool.n_kv);
    const int s = sb / a.blocks, part = sb % a.blocks;
    if (s >= tok.n_seqs) return;
    const int64_t at = (static_cast<int64_t>(s) * pool.n_kv + h) * tok.max_pages;
    for (int c = wave; c < tok.max_pages; c += kWaves)
        if (c / 16 % a.blocks == part && lane == 0) a.weights[at + c] = a.prev ? a.prev[at + c] : 0.f;
    for (int t0 = 0; t0 < tok.n_tokens; t0 += kScan) {
        const int n = tokens_of(tok, s, t0, s_tok, s_count);
        for (int i = 0; i < n; ++i) {
            const int t = s_tok[i], pos = tok.pos[t];
            const int32_t* list = a.list + (static_cast<int64_t>(t) * pool.n_kv + h) * a.n_list;
            Columns<T, D, kTerms> col;
            bool loaded = false;
            for (int e0 = 0; e0 < a.n_list; e0 += 64) {
                const int c = e0 + lane < a.n_list ? list[e0 + lane] : -1;
                SeenPage p{-1, 0};
                if (c >= 0 && c / 16 % a.blocks == part && c % kWaves == wave) p = seen_page(pool, tok, s, pos, c);
                for (uint64_t left = __builtin_amdgcn_ballot_w64(p.rows > 0); left; left &= left - 1) {
                    const int l = static_cast<int>(__builtin_ctzll(left)), chunk = __builtin_amdgcn_readlane(c, l);
                    if (!loaded) col = load_columns<T, D, kTerms>(tok, a, q, q_stride, h, pool.n_kv, s_tok + i, 0, a.ratio, m, g);
                    loaded = true;
                    Keys<D> k;
                    load_keys<D>(make_rsrc(pool.page(__builtin_amdgcn_readlane(p.id, l)) + h * F::kBytes, F::kBytes), m, g, k);
                    const float sum = wave_sum(page_weight<T, D, kTerms>(k, col, chunk, g));
                    if (lane == 0) a.weights[at + chunk] += sum;
                }
            }
        }
    }
}

}  // namespace

int64_t weigh_pages_bytes(const hga_plan&, int, int, int, int) { return 0; }

hipError_t launch_weigh_pages(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                              int64_t q_stride, const float* lse, const int32_t* list, int n_list, const float* prev,
                              float* weights, void*, int64_t, hipStream_t stream) {
    const int64_t units = static_cast<int64_t>(tok.n_seqs) * pool.n_kv;
    if (units == 0 || tok.max_pages == 0) return hipSuccess;
    WeighArgs a;
    a.list = list;
    a.n_list = n_list;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.lse = lse;
    a.prev = prev;
    a.weights = weights;
    const int64_t want = 8 * static_cast<int64_t>(plan.n_cu);
    const int64_t most = list ? (tok.max_pages + 15) / 16 : (tok.max_pages + kWaves - 1) / kWaves;
    a.blocks = static_cast<int>(std::clamp<int64_t>((want + units - 1) / units, 1, most));
    const auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value;
        const dim3 grid = grid_of(units * a.blocks, kThreads);
        if (list)
            weigh_listed_kernel<T, D><<<grid, kThreads, 0, stream>>>(pool, tok, a, static_cast<const T*>(q), q_stride);
        else
            weigh_kernel<T, D><<<grid, kThreads, 0, stream>>>(pool, tok, a, static_cast<const T*>(q), q_stride);
        return hipGetLastError();
    };
    const bool f32 = plan.p.dtype == HGA_F32;
    if (plan.p.head_dim == 128)
        return f32 ? go(0.f, std::integral_constant<int, 128>()) : go(bf16_t(0), std::integral_constant<int, 128>());
    return f32 ? go(0.f, std::integral_constant<int, 64>()) : go(bf16_t(0), std::integral_constant<int, 64>());
}

}  // namespace hga

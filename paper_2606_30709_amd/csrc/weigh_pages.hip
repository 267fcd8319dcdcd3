// Attention weight of pages: what each page of a sequence got of the attention of a call's tokens,
//   W[s][h][c] = prev[s][h][c] + sum over tokens t of s, query heads of h, rows o of page c up to t's position of
//                exp(q . k~_o / sqrt(d) - lse),
// from the queries and the lse that their attention gave.  Only keys are read: half of a page.
//
// Query heads are the columns of a 16-column tile and scores its S^T, as in the attention (attend_pages.hpp); a page's
// weight is the sum over all of them, a lane's 16 of each tile and then the wavefront's.
//
// Bound by the keys' bytes over whole histories: 32 sequences of 1K to 32K tokens, 4 heads of d128, 37 us (4.0 TB/s; with a
// page's keys fetched when it is its turn 59).  Listed pages are bound by the chain token, list, table, page: 64 sequences of
// 31 pages each 13 us, a list's pages to eight wavefronts (to one: 80).
//
// Sums depend on nothing that runs beside them: whoever owns a page of a (sequence, KV head) takes all the tokens of the
// sequence, in the call's order, and no two writers meet.  Where that leaves the device idle (many tokens of few pages) the
// call's tokens are cut into slices, which a second kernel adds up in order.
#include <algorithm>
#include <type_traits>

#include "attend_pages.hpp"
#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr double kLog2E = 1.44269504088896340736;
constexpr int kScan = 1024;  // tokens looked at, at a time, for those of a sequence

struct WeighArgs {
    const int32_t* list;  // NULL: every chunk
    int n_list, ratio;
    int run;              // pages of a wavefront, 64 at most (whole histories)
    int blocks;           // workgroups of a (sequence, KV head)
    int slices;           // of the call's tokens
    int slice;            // tokens of one
    const float* lse;
    const float* prev;    // NULL: zeros
    float* out;           // the weights, or [slice] of them
};

// Which of the tokens [t0, t1), kScan at most, are of sequence s, in order, into LDS; how many.  Every wavefront of the
// workgroup writes the same words.
__device__ __forceinline__ int tokens_of(const TokensView& tok, int s, int t0, int t1, int32_t* s_tok) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int i0 = t0; i0 < t1; i0 += 256) {
        uint64_t mine[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int t = i0 + 64 * y + lane;
            int sc = -1, pc;
            mine[y] = __builtin_amdgcn_ballot_w64(t < t1 && tok.at(t, sc, pc) && sc == s);
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (mine[y] >> lane & 1) s_tok[n + __popcll(mine[y] & ((uint64_t(1) << lane) - 1))] = i0 + 64 * y + lane;
            n += __popcll(mine[y]);
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    return n;
}

// The queries of up to 16 columns, and what else a column needs.
template <typename T, int D>
struct Columns {
    static constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    u32x4 qf[1][kTerms][D / 32];
    float hi, lo;  // lse in log2 units, two floats that add up to it; +inf: the column sees nothing
    int pos;
};
template <typename T, int D>
__device__ __forceinline__ void load_columns(const TokensView& tok, const WeighArgs& a, const T* q, int64_t q_stride, int h,
                                             int n_kv, const int32_t* s_tok, int c0, int columns, int m, int g,
                                             Columns<T, D>& r) {
    constexpr int kTerms = Columns<T, D>::kTerms;
    const int c = c0 + m;
    const bool real = c < columns;
    const int t = s_tok[real ? c / a.ratio : 0], head = h * a.ratio + (real ? c % a.ratio : 0);
    r.pos = real ? tok.pos[t] : -1;
    const float lse = real ? a.lse[static_cast<int64_t>(t) * n_kv * a.ratio + head] : -INFINITY;
    constexpr float kLog = static_cast<float>(kLog2E), kLogRest = static_cast<float>(kLog2E - static_cast<double>(kLog));
    r.hi = lse * kLog;
    r.lo = fmaf(lse, kLog, -r.hi) + lse * kLogRest;
    if (!(fabsf(lse) < INFINITY) && lse == lse) r.hi = INFINITY, r.lo = 0.f;
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
}

// A lane's share of what a page gets from 16 columns: rows from first_row on, up to each column's position.
template <typename T, int D>
__device__ __forceinline__ float page_weight(const Keys<D>& k, const Columns<T, D>& col, int first_row, int g) {
    // log2(e) / sqrt(d) as two floats: with one, the exponent's argument would be off by its rounding times the score
    constexpr double kScale = kLog2E / (D == 64 ? 8.0 : 11.3137084989847603904);
    constexpr float kHi = static_cast<float>(kScale), kLo = static_cast<float>(kScale - static_cast<double>(kHi));
    f32x4 sc[1][4];
    page_scores<D, Columns<T, D>::kTerms, 1>(k, col.qf, sc);
    float sum = 0.f;
    const int seen = col.hi == INFINITY ? -1 : col.pos - first_row - 4 * g;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const float s = sc[0][tt][x];
            const float p = __builtin_amdgcn_exp2f(fmaf(s, kHi, -col.hi) + fmaf(s, kLo, -col.lo));
            sum += 16 * tt + x <= seen ? p : 0.f;
        }
    return sum;
}
template <int kCtrl>
__device__ __forceinline__ float add_dpp_f32(float x) {
    return x + __uint_as_float(static_cast<uint32_t>(
                   __builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(x)), kCtrl, 0xf, 0xf, true)));
}
// The sum over the wavefront, in every lane.
__device__ __forceinline__ float wave_sum(float x) {
    x = add_dpp_f32<0xB1>(x);   // quads
    x = add_dpp_f32<0x4E>(x);
    x = add_dpp_f32<0x124>(x);  // rotations by 4 and 8 of a row of 16
    x = add_dpp_f32<0x128>(x);
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const uint32_t v = __float_as_uint(x);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// Where the workgroup's share lies.
struct Share {
    int s, h, part, slice, t0, t1;
    int64_t row;  // of [s][h], in pages
    const float* prev;
    float* out;
};
template <int kThreads>
__device__ __forceinline__ Share share_of(const PoolView& pool, const TokensView& tok, const WeighArgs& a) {
    Share r;
    const uint32_t block = linear_block<kThreads>();
    const TokenHead w = token_head(block, pool.n_kv);
    r.h = w.h;
    const int per = tok.n_seqs * a.blocks;
    r.slice = w.t / per;
    const int sp = w.t - r.slice * per;
    // the parts of a sequence in the outer order: short histories have none of the later ones
    r.part = sp / tok.n_seqs;
    r.s = sp - r.part * tok.n_seqs;
    r.t0 = static_cast<int>(min(static_cast<int64_t>(r.slice) * a.slice, static_cast<int64_t>(tok.n_tokens)));
    r.t1 = static_cast<int>(min(static_cast<int64_t>(r.t0) + a.slice, static_cast<int64_t>(tok.n_tokens)));
    r.row = (static_cast<int64_t>(r.s) * pool.n_kv + r.h) * tok.max_pages;
    r.prev = a.slices == 1 ? a.prev : nullptr;
    r.out = a.out + (a.slices == 1 ? 0 : static_cast<int64_t>(r.slice) * tok.n_seqs * pool.n_kv * tok.max_pages);
    return r;
}

// Whole histories: a wavefront takes a run of pages, a lane keeping the sum of each; its next page's keys are fetched while
// it works on one.
template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, (sizeof(T) == 4 && D == 128 ? 3 : 4)) void weigh_kernel(
    PoolView pool, TokensView tok, WeighArgs a, const T* __restrict__ q, int64_t q_stride) {
    using F = PageFormat<D>;
    __shared__ int32_t s_tok[kScan];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const Share w = share_of<64 * kWaves>(pool, tok, a);
    if (w.slice >= a.slices) return;
    const int from = (w.part * kWaves + wave) * a.run, page = from + lane;
    const bool mine = lane < a.run && page < tok.max_pages;
    float total = mine && w.prev ? w.prev[w.row + page] : 0.f;
    for (int t0 = w.t0; t0 < w.t1; t0 += kScan) {
        if (t0 > w.t0) __syncthreads();  // the last ones have been used
        const int n = tokens_of(tok, w.s, t0, min(t0 + kScan, w.t1), s_tok);
        const int columns = n * a.ratio;
        if (n == 0 || from >= tok.max_pages) continue;
        int last = -1;
        for (int i = lane; i < n; i += 64) last = max(last, tok.pos[s_tok[i]]);
#pragma unroll
        for (int x = 1; x < 64; x *= 2) last = max(last, __shfl_xor(last, x));
        last = __builtin_amdgcn_readfirstlane(last);
        SeenPage p{-1, 0};
        if (mine) p = seen_page(pool, tok, w.s, last, page);
        const uint64_t there = __builtin_amdgcn_ballot_w64(p.rows > 0);
        float sum = 0.f;
        const auto part = [&](int i, bool any) {
            return make_rsrc(pool.page(__builtin_amdgcn_readlane(p.id, i)) + w.h * F::kBytes, any ? F::kBytes : 0);
        };
        for (int c0 = 0; there && c0 < columns; c0 += 16) {
            uint64_t left = there;
            int cur = static_cast<int>(__builtin_ctzll(left));
            Keys<D> k;
            load_keys<D>(part(cur, true), m, g, k);
            Columns<T, D> col;
            load_columns<T, D>(tok, a, q, q_stride, w.h, pool.n_kv, s_tok, c0, columns, m, g, col);
            while (left) {
                left &= left - 1;
                const int next = left ? static_cast<int>(__builtin_ctzll(left)) : cur;
                Keys<D> kn;
                load_keys<D>(part(next, left != 0), m, g, kn);
                const float x = wave_sum(page_weight<T, D>(k, col, (from + cur) * kPageRows, g));
                if (lane == cur) sum += x;
                k = kn;
                cur = next;
            }
        }
        total += sum;
    }
    if (mine) w.out[w.row + page] = total;
}

// Listed pages: a workgroup a (sequence, KV head), its tokens one after another.  The entries of a list that are pages go to
// the wavefronts in turn; then one of them adds what they found to the weights, an entry a lane, those of one page in the
// list's order.
template <typename T, int D, int kWaves>
__global__ __launch_bounds__(64 * kWaves, (sizeof(T) == 4 && D == 128 ? 3 : 4)) void weigh_listed_kernel(
    PoolView pool, TokensView tok, WeighArgs a, const T* __restrict__ q, int64_t q_stride) {
    using F = PageFormat<D>;
    __shared__ int32_t s_tok[kScan];
    __shared__ float s_sum[64];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const Share w = share_of<64 * kWaves>(pool, tok, a);
    if (w.slice >= a.slices) return;
    if (w.prev != w.out)
        for (int c = tid; c < tok.max_pages; c += 64 * kWaves) w.out[w.row + c] = w.prev ? w.prev[w.row + c] : 0.f;
    for (int t0 = w.t0; t0 < w.t1; t0 += kScan) {
        if (t0 > w.t0) __syncthreads();
        const int n = tokens_of(tok, w.s, t0, min(t0 + kScan, w.t1), s_tok);
        for (int i = 0; i < n; ++i) {
            const int t = s_tok[i], pos = tok.pos[t];
            const int32_t* list = a.list + (static_cast<int64_t>(t) * pool.n_kv + w.h) * a.n_list;
            Columns<T, D> col;
            load_columns<T, D>(tok, a, q, q_stride, w.h, pool.n_kv, s_tok + i, 0, a.ratio, m, g, col);
            for (int e0 = 0; e0 < a.n_list; e0 += 64) {
                const int c = e0 + lane < a.n_list ? list[e0 + lane] : -1;
                const SeenPage p = c < 0 ? SeenPage{-1, 0} : seen_page(pool, tok, w.s, pos, c);
                const uint64_t there = __builtin_amdgcn_ballot_w64(p.rows > 0);
                if (!there) continue;  // the same in every wavefront
                // this wavefront's: every kWaves-th of them
                const int rank = __popcll(there & ((uint64_t(1) << lane) - 1));
                uint64_t left = __builtin_amdgcn_ballot_w64(p.rows > 0 && rank % kWaves == wave);
                const auto part = [&](int j, bool any) {
                    return make_rsrc(pool.page(__builtin_amdgcn_readlane(p.id, j)) + w.h * F::kBytes, any ? F::kBytes : 0);
                };
                if (left) {
                    int cur = static_cast<int>(__builtin_ctzll(left));
                    Keys<D> k;
                    load_keys<D>(part(cur, true), m, g, k);
                    while (left) {
                        left &= left - 1;
                        const int next = left ? static_cast<int>(__builtin_ctzll(left)) : cur;
                        Keys<D> kn;
                        load_keys<D>(part(next, left != 0), m, g, kn);
                        const float x =
                            wave_sum(page_weight<T, D>(k, col, __builtin_amdgcn_readlane(c, cur) * kPageRows, g));
                        if (lane == cur) s_sum[lane] = x;
                        k = kn;
                        cur = next;
                    }
                }
                __syncthreads();
                if (wave == 0) {
                    const float mine = p.rows > 0 ? s_sum[lane] : 0.f;
                    float sum = 0.f;
                    bool first = p.rows > 0;
                    for (uint64_t all = there; all; all &= all - 1) {
                        const int j = static_cast<int>(__builtin_ctzll(all));
                        const float x = __uint_as_float(
                            static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(__float_as_uint(mine)), j)));
                        if (__builtin_amdgcn_readlane(c, j) == c) {
                            sum += x;
                            if (j < lane) first = false;
                        }
                    }
                    if (first) w.out[w.row + c] += sum;
                }
                __syncthreads();
            }
        }
    }
}

__global__ __launch_bounds__(256) void add_slices_kernel(const float* __restrict__ part, int slices, int64_t n, const float* prev,
                                                         float* weights) {
    const int64_t i = static_cast<int64_t>(linear_block<256>()) * 256 + threadIdx.x;
    if (i >= n) return;
    float sum = prev ? prev[i] : 0.f;
    for (int y = 0; y < slices; ++y) sum += part[y * n + i];
    weights[i] = sum;
}

struct Cut {
    int run, blocks, slices, slice, waves;
    int64_t bytes;
};

Cut cut_call(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_list, int64_t ws_bytes) {
    const int ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    const int64_t units = std::max<int64_t>(static_cast<int64_t>(n_seqs) * plan.p.n_kv_heads, 1);
    Cut c{0, 1, 1, std::max(n_tokens, 1), 4, 0};
    const int64_t want = 16 * static_cast<int64_t>(plan.n_cu);  // wavefronts
    if (n_list) {
        c.waves = 8;
    } else {
        const int64_t most = std::max<int64_t>(1, units * max_pages / want);
        c.run = static_cast<int>(std::clamp<int64_t>(most, 1, 64));
        c.blocks = (max_pages + c.run * c.waves - 1) / (c.run * c.waves);
    }
    // Slices of the tokens where the pages alone do not fill the device: of two tiles' tokens at least.  us with and without:
    // 512 tokens of one sequence of 1,024, 12 heads of d64 fp32, 16 slices 14.4 and 45.4; 256 of 2,048, 32/4 d128 bf16, 32 slices
    // 27.6 and 155; 8 times 256 tokens of 31 listed pages, 16 slices 1,072 and 2,125.  Units, pages and tokens of a sequence are
    // counted by the table's rows and width, as the host knows no better: in a table of many more, runs are longer and slices
    // fewer than the batch would need.
    const int64_t have = units * c.blocks * c.waves;
    const int least = std::max(1, n_list ? 2 : 32 / ratio);
    const int per_seq = static_cast<int>((static_cast<int64_t>(n_tokens) + n_seqs - 1) / std::max(n_seqs, 1));
    const int64_t cells = units * max_pages * 4;
    int64_t slices = std::min<int64_t>({want / std::max<int64_t>(have, 1), per_seq / least, 64, (int64_t(1) << 26) / std::max<int64_t>(cells, 1)});
    slices = std::min(slices, ws_bytes / std::max<int64_t>(cells, 1));
    if (slices > 1) {
        c.slices = static_cast<int>(slices);
        c.slice = (n_tokens + c.slices - 1) / c.slices;
        c.bytes = slices * cells;
    }
    return c;
}

}  // namespace

int64_t weigh_pages_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_list) {
    if (n_tokens == 0 || n_seqs == 0 || max_pages == 0) return 0;
    return cut_call(plan, n_tokens, n_seqs, max_pages, n_list, INT64_MAX).bytes;
}

hipError_t launch_weigh_pages(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                              int64_t q_stride, const float* lse, const int32_t* list, int n_list, const float* prev,
                              float* weights, void* ws, int64_t ws_bytes, hipStream_t stream) {
    const int64_t units = static_cast<int64_t>(tok.n_seqs) * pool.n_kv;
    if (units == 0 || tok.max_pages == 0) return hipSuccess;
    const Cut c = cut_call(plan, tok.n_tokens, tok.n_seqs, tok.max_pages, list ? n_list : 0, ws_bytes);
    WeighArgs a;
    a.list = list;
    a.n_list = n_list;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.run = c.run;
    a.blocks = c.blocks;
    a.slices = c.slices;
    a.slice = c.slice;
    a.lse = lse;
    a.prev = prev;
    a.out = c.slices > 1 ? static_cast<float*>(ws) : weights;
    const auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value;
        const T* x = static_cast<const T*>(q);
        if (list)
            weigh_listed_kernel<T, D, 8><<<grid_of(units * c.slices, 512), 512, 0, stream>>>(pool, tok, a, x, q_stride);
        else
            weigh_kernel<T, D, 4><<<grid_of(units * c.blocks * c.slices, 256), 256, 0, stream>>>(pool, tok, a, x, q_stride);
        return hipGetLastError();
    };
    const bool f32 = plan.p.dtype == HGA_F32;
    const hipError_t e = plan.p.head_dim == 128 ? (f32 ? go(0.f, std::integral_constant<int, 128>()) : go(bf16_t(0), std::integral_constant<int, 128>()))
                                                : (f32 ? go(0.f, std::integral_constant<int, 64>()) : go(bf16_t(0), std::integral_constant<int, 64>()));
    if (e != hipSuccess || c.slices == 1) return e;
    const int64_t n = units * tok.max_pages;
    add_slices_kernel<<<grid_of((n + 255) / 256, 256), 256, 0, stream>>>(a.out, c.slices, n, prev, weights);
    return hipGetLastError();
}

}  // namespace hga

// Attention of single tokens over the paged 4-bit cache (Sec. 3.4 at the token's grain, every query head of a KV head in
// one tile).
//
// A unit is one KV head and one token, or (over whole histories) up to 16 kTiles / r adjacent tokens of one sequence: its
// query heads are the columns of kTiles 16-column tiles,
//   S^T [16 keys x 16 columns] = K~ [16 x d] q^T      (d/32 instructions of 16x16x32)
//   O^T [16 dims x 16 columns] += V~^T [16 x 32] P^T  (a 32-key half page, d/16 instructions)
// Codes become bf16 in registers, two an instruction with their scale.  The layout of a page (tokens.hpp) is that of these
// operands, so codes go straight from memory to the lane that multiplies them.  A lane of S^T holds keys 4 g .. 4 g + 3 of
// its tile, and takes those as its reduction indices of the second product: P never leaves the lane.  One pass over the
// keys with a running reference (the maximum, or up to 2^kSlack below it) and sum of each column, in log2 units.
//
// The stored keys and values are exact in bf16, and so is a bf16 query.  A bf16 call's weights enter the second product as
// two bf16 terms each: at most 2^-16 of a weight is left out, against 2^-8 of the result that its own rounding takes.  One
// term would leave out 2^-8 of each weight, which for values of either sign is as much as that rounding (32 histories up to
// 32K 57 and 61 us with one term and two, 512 tokens of a 16K prompt 156 and 198).  fp32 queries and weights enter as three
// terms each (24 bits).  With up to four query heads the terms are columns of their own (kSpread): column 4 r + x holds
// term x of head r, the scores of four columns are added up, and each multiplies its own term of the weight.  A third of
// the matrix instructions and half the work of splitting: 1,325 tokens of 12 heads of d64 over 11 pages each 115 -> 95 us.
//
// A wavefront loads its next page while it works on one; the wavefronts of a workgroup take every kWaves-th page and are
// joined in LDS.  Long histories of few units are cut into equal runs of pages, a workgroup each, whose partial results a
// second kernel joins in order.
#include <algorithm>
#include <type_traits>

#include "attend_pages.hpp"
#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

struct AttendArgs {
    const int32_t* list;  // NULL: every chunk
    int n_list, ratio;
    int run;              // pages of a workgroup
    int splits;           // workgroups of a unit at most
    float* lse;
    const int32_t* units;  // [0]: how many, then their first tokens and the call's end; NULL: every token is a unit
    int32_t* parts;       // [token]: workgroups that took its unit
    float* part;          // their results [split][token][query head][d], not divided by the sum
    float* part_ml;       // ... and [split][token][query head][2]: reference, sum
};

// The units of a call whose tokens share them: a unit is of one sequence and ends at a multiple of `tokens`.  One workgroup.
__global__ __launch_bounds__(1024) void list_units_kernel(const int32_t* __restrict__ seq, int n_tokens, int tokens,
                                                          int32_t* __restrict__ units) {
    __shared__ int counts[16];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int base = 0;
    for (int t0 = 0; t0 < n_tokens; t0 += 1024) {
        const int t = t0 + tid;
        const bool first = t < n_tokens && (t % tokens == 0 || seq[t] != seq[t - 1]);
        const uint64_t mask = __builtin_amdgcn_ballot_w64(first);
        if (lane == 0) counts[wave] = __popcll(mask);
        __syncthreads();
        int at = base + __popcll(mask & ((uint64_t(1) << lane) - 1));
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += counts[w];
            base += counts[w];
        }
        if (first) units[1 + at] = t;
        __syncthreads();
    }
    if (tid == 0) {
        units[0] = base;
        units[1 + base] = n_tokens;
    }
}

// Wavefronts of a SIMD that the registers are kept to (one tile: as many as fit without spills).
template <typename T, int D, int kTiles, bool kShared, bool kSpread>
constexpr int kResident = kTiles == 2 || kShared || (sizeof(T) == 4 && D == 128 && !kSpread) ? 2
                          : sizeof(T) == 2 && D == 64                                       ? 4
                                                                                            : 3;

// kShared: units of several tokens, from a.units, of which a workgroup may take more than one; else every token is a unit.
// kSpread: fp32, at most four heads and one token a unit, terms as columns.
template <typename T, int D, int kTiles, int kWaves, bool kShared, bool kSpread>
__global__ __launch_bounds__(64 * kWaves, (kResident<T, D, kTiles, kShared, kSpread>)) void attend_tokens_kernel(
    PoolView pool, TokensView tok, AttendArgs a, const T* __restrict__ q, int64_t q_stride, T* __restrict__ out,
    int grid_units) {
    using F = PageFormat<D>;
    constexpr int kThreads = 64 * kWaves;
    static_assert(!kSpread || (sizeof(T) == 4 && !kShared && kTiles == 1), "");
    constexpr int kTerms = sizeof(T) == 4 && !kSpread ? 3 : 1;  // of a query
    constexpr int kParts = sizeof(T) == 2 ? 2 : kTerms;         // of a weight
    constexpr int DL = F::kLaneDims;
    constexpr int kSteps = D / 32;
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));  // log2(e) / sqrt(d)
    extern __shared__ __align__(16) float smem[];
    float(*s_o)[16 * kTiles][D + 4] = reinterpret_cast<float(*)[16 * kTiles][D + 4]>(smem);
    float(*s_m)[16 * kTiles] = reinterpret_cast<float(*)[16 * kTiles]>(smem + kWaves * 16 * kTiles * (D + 4));
    float(*s_l)[16 * kTiles] = s_m + kWaves;
    const int n_units = kShared ? a.units[0] : tok.n_tokens;
    const uint32_t block = linear_block<kThreads>();
    // splits in the outer order: short histories have none of the later ones, and a split as the inner one would be an XCD
    const uint32_t row = static_cast<uint32_t>(grid_units) * pool.n_kv;
    const int split = static_cast<int>(block / row);
    const auto [unit0, h] = token_head(block % row, pool.n_kv);
    if (split >= a.splits) return;
    for (int unit = unit0; unit < n_units; unit += grid_units) {
    const int t = kShared ? a.units[1 + unit] : unit;
    const int n_tok = kShared ? a.units[2 + unit] - t : 1;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int columns = n_tok * a.ratio;

    // column 16 i + m: query head column % r of token t + column / r; zeros past the last
    const TermMask terms = term_mask(m);
    int pos[kTiles];
    int s = 0, last = -1, first = INT32_MAX;  // the unit's sequence, its tokens' largest and smallest positions
    u32x4 qf[kTiles][kTerms][kSteps];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int c = kSpread ? m >> 2 : 16 * i + m;
        const bool real = c < columns;
        const int tc = t + (real ? c / a.ratio : 0);
        int sc = 0, pc = 0;
        const bool in = tok.at(tc, sc, pc);
        pos[i] = in ? pc : -1;
        last = max(last, pos[i]);
        first = min(first, pos[i]);
        s = in ? sc : s;
        const T* row = q + tc * q_stride + (static_cast<int64_t>(h) * a.ratio + c % a.ratio) * D + g * (D / 4);
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            float x[8] = {};
            if (real && in) load8(row + 8 * kk, x);
            if constexpr (kSpread)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[e] = term_of(x[e], terms);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t w[kTerms];
                split2<kTerms>(x[2 * e], x[2 * e + 1], w);
#pragma unroll
                for (int y = 0; y < kTerms; ++y) qf[i][y][kk][e] = w[y];
            }
        }
    }
    if (kShared) {
#pragma unroll
        for (int x = 1; x < 16; x *= 2) {
            last = max(last, __shfl_xor(last, x));
            first = min(first, __shfl_xor(first, x));
            s = max(s, __shfl_xor(s, x));
        }
    }
    s = __builtin_amdgcn_readfirstlane(s);
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    const int32_t* list = a.list ? a.list + (static_cast<int64_t>(t) * pool.n_kv + h) * a.n_list : nullptr;
    const int n_all = last < 0 ? 0 : list ? a.n_list : last / kPageRows + 1;
    const int parts = min(a.splits, max(1, (n_all + a.run - 1) / a.run));
    if (split >= parts) {
        if (!kShared) break;
        continue;
    }
    if (a.splits > 1 && split == 0 && h == 0 && tid < n_tok) a.parts[t + tid] = parts;
    const int n_entries = parts == 1 ? n_all : min(n_all, (split + 1) * a.run);

    Acc<D, kTiles> acc;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        acc.m[i] = -INFINITY;
        acc.l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < DL; ++j) acc.o[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int e0 = split * a.run + wave; e0 < n_entries; e0 += 64 * kWaves) {
        // the next 64 entries of this wavefront, one a lane
        SeenPage mine{-1, 0};
        int chunk = 0;
        const int e = e0 + lane * kWaves;
        if (e < n_entries) {
            chunk = list ? list[e] : e;
            mine = seen_page(pool, tok, s, last, chunk);
        }
        uint64_t left = __builtin_amdgcn_ballot_w64(mine.rows > 0);
        if (!left) continue;
        int cur = static_cast<int>(__builtin_ctzll(left));
        const auto part = [&](int i, bool any) {
            return make_rsrc(pool.page(__builtin_amdgcn_readlane(mine.id, i)) + h * F::kBytes, any ? F::kBytes : 0);
        };
        // keys of the next page are fetched once this one's scores are formed (with two tiles once half of this one's values
        // are used too, in their registers), its values once this one's are used
        Keys<D> k;
        Values<D> v;
        {
            const buf_rsrc r = part(cur, true);
            load_keys<D>(r, m, g, k);
            load_values<D>(r, m, g, v);
        }
        while (left) {
            left &= left - 1;
            const int next = left ? static_cast<int>(__builtin_ctzll(left)) : cur;
            const buf_rsrc r = part(next, left != 0);
            const int c = __builtin_amdgcn_readlane(chunk, cur);
            f32x4 sc[kTiles][4];
            page_scores<D, kTerms, kTiles>(k, qf, sc);
            if constexpr (kSpread)
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sc[0][tt][x] = quad_sum(sc[0][tt][x]);
            if constexpr (kTiles == 1) load_keys<D>(r, m, g, k);
            if (kShared ? first < c * kPageRows + kPageRows - 1 : __builtin_amdgcn_readlane(mine.rows, cur) < kPageRows) {
                // rows past a column's position are not seen; those behind the last stored one hold anything, whose
                // values count as some number (times a weight of 0)
                __asm__ volatile("");  // a branch: most pages need none of this
                const int rows = __builtin_amdgcn_readlane(mine.rows, cur);
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int row = 16 * tt + 4 * g + x;
                        if (row >= rows) v.s[tt] = (v.s[tt] & ~(255u << (8 * x))) | 127u << (8 * x);
#pragma unroll
                        for (int i = 0; i < kTiles; ++i)
                            if (kShared ? row > pos[i] - c * kPageRows : row >= rows) sc[i][tt][x] = -INFINITY;
                    }
                if constexpr (kShared) {
                    int seen[kTiles];
#pragma unroll
                    for (int i = 0; i < kTiles; ++i) seen[i] = pos[i] - c * kPageRows;
                    take_out_nan<D, kTiles>(v, m, g, seen, acc);
                }
            }
            page_reference<D, kTiles>(sc, scale, acc);
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 w[kTiles][kParts];
                half_weights<D, kParts, kTiles>(u, sc, scale, acc, w, kSpread ? &terms : nullptr);
                if constexpr (kTiles > 1) __builtin_amdgcn_sched_barrier(0);  // or the registers do not suffice
                half_values<D, kParts, kTiles>(u, v, w, acc);
                if constexpr (kTiles > 1) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (u == 0) load_keys<D>(r, m, g, k);
                }
            }
            load_values<D>(r, m, g, v);
            cur = next;
        }
    }

    // join the wavefronts: lane (m, g) of tile i holds column 16 i + m, dimensions (4 g + x) DL + j
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const float l = sum_groups(acc.l[i]);
        const int c = kSpread ? m >> 2 : 16 * i + m;
        const bool holds = !kSpread || (m & 3) == 0;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < DL; ++j) {
                const float y = kSpread ? quad_sum(acc.o[i][j][x]) : acc.o[i][j][x];
                if (holds) s_o[wave][c][(4 * g + x) * DL + j] = y;
            }
        if (g == 0 && holds) {
            s_m[wave][c] = acc.m[i];
            s_l[wave][c] = l;
        }
    }
    __syncthreads();
    for (int i = tid; i < columns * D; i += kThreads) {
        const int r = i / D, c = i % D;
        float top = s_m[0][r];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        const float ref = top == -INFINITY ? 0.f : top;
        float l = 0.f, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = part_weight(s_m[w][r], ref);
            l += f * s_l[w][r];
            sum += f * s_o[w][r][c];
        }
        const int64_t at_row = static_cast<int64_t>(t + r / a.ratio) * pool.n_kv * a.ratio + h * a.ratio + r % a.ratio;
        if (parts == 1) {
            out[at_row * D + c] = elem<T>::from_f32(l == 0.f ? 0.f : sum / l);
            if (a.lse && c == 0) a.lse[at_row] = natural_lse(ref, l);
        } else {
            const int64_t at = static_cast<int64_t>(split) * tok.n_tokens * pool.n_kv * a.ratio + at_row;
            a.part[at * D + c] = sum;
            if (c == 0) {
                a.part_ml[2 * at] = top;
                a.part_ml[2 * at + 1] = l;
            }
        }
    }
    if (!kShared) break;
    __syncthreads();  // LDS is the next unit's
    }
}

// Joins the partial results of a token's query head, in a fixed order: a workgroup a head, its threads D/4 columns of four
// dimensions by the groups of parts they add up.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_parts_kernel(int n_rows, int heads, AttendArgs a, T* __restrict__ out) {
    constexpr int kCols = D / 4, kGroups = 256 / kCols;
    __shared__ float4 s_o[kGroups][kCols];
    __shared__ float s_l[kGroups], s_m[kGroups];
    const int64_t row = linear_block<256>();
    if (row >= n_rows) return;
    const int parts = a.parts[row / heads];
    if (parts == 1) return;
    const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w0 = grp; w0 < parts; w0 += 4 * kGroups) {
        float2 ml[4];
        float4 x[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int64_t at = static_cast<int64_t>(min(w0 + y * kGroups, parts - 1)) * n_rows + row;
            ml[y] = reinterpret_cast<const float2*>(a.part_ml)[at];
            x[y] = reinterpret_cast<const float4*>(a.part)[at * kCols + col];
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (w0 + y * kGroups >= parts) break;
            const float top = fmaxf(m, ml[y].x), ref = top == -INFINITY ? 0.f : top;
            const float f = part_weight(m, ref), e = part_weight(ml[y].x, ref);
            m = top;
            l = l * f + ml[y].y * e;
            o.x = o.x * f + x[y].x * e;
            o.y = o.y * f + x[y].y * e;
            o.z = o.z * f + x[y].z * e;
            o.w = o.w * f + x[y].w * e;
        }
    }
    s_o[grp][col] = o;
    if (col == 0) {
        s_m[grp] = m;
        s_l[grp] = l;
    }
    __syncthreads();
    if (threadIdx.x >= D) return;
    float top = s_m[0];
#pragma unroll
    for (int w = 1; w < kGroups; ++w) top = fmaxf(top, s_m[w]);
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    l = 0.f;
#pragma unroll
    for (int w = 0; w < kGroups; ++w) {
        const float f = part_weight(s_m[w], ref);
        l += f * s_l[w];
        sum += f * reinterpret_cast<const float*>(s_o[w])[threadIdx.x];
    }
    out[row * D + threadIdx.x] = elem<T>::from_f32(l == 0.f ? 0.f : sum / l);
    if (a.lse && threadIdx.x == 0) a.lse[row] = natural_lse(ref, l);
}

template <typename T, int D, int kTiles, int kWaves, bool kShared, bool kSpread = false>
hipError_t run(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const AttendArgs& a, const void* q,
               int64_t q_stride, void* out, int grid_units, hipStream_t stream) {
    constexpr int kThreads = 64 * kWaves;
    constexpr size_t lds = sizeof(float) * kWaves * 16 * kTiles * (D + 4 + 2);
    if (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = once_per_device(done, plan.device, [] {
            return hipFuncSetAttribute(reinterpret_cast<const void*>(attend_tokens_kernel<T, D, kTiles, kWaves, kShared, kSpread>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
        });
        if (e != hipSuccess) return e;
    }
    const int64_t n = static_cast<int64_t>(grid_units) * pool.n_kv * a.splits;
    attend_tokens_kernel<T, D, kTiles, kWaves, kShared, kSpread><<<grid_of(n, kThreads), kThreads, lds, stream>>>(
        pool, tok, a, static_cast<const T*>(q), q_stride, static_cast<T*>(out), grid_units);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    const int heads = pool.n_kv * a.ratio, rows = tok.n_tokens * heads;
    join_parts_kernel<T, D><<<grid_of(rows, 256), 256, 0, stream>>>(rows, heads, a, static_cast<T*>(out));
    return hipGetLastError();
}

// How a call is cut: tokens of a unit and their tiles, pages of a workgroup, workgroups of a unit, their wavefronts; and the
// workspace that takes, in bytes from its start.
struct Cut {
    int tokens, tiles, run, splits, waves, grid_units;
    int64_t parts, part, part_ml, bytes;
};

int64_t pad16(int64_t n) { return (n + 15) / 16 * 16; }

Cut cut_call(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_list, int64_t ws_bytes) {
    const int ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    const int64_t rows = static_cast<int64_t>(n_tokens) * plan.p.n_q_heads;
    Cut c{1, 1, 0, 1, 4, n_tokens, 0, 0, 0, 0};
    const int64_t entries = std::max(n_list ? n_list : max_pages, 1);
    // tokens of one sequence share its pages unless they have lists of their own
    const int per_seq = n_list || n_seqs < 1 ? 1 : static_cast<int>((static_cast<int64_t>(n_tokens) + n_seqs - 1) / n_seqs);
    const int64_t list_bytes = pad16((static_cast<int64_t>(n_tokens) + 2) * 4);
    if (per_seq > 1 && ws_bytes >= list_bytes) {
        // two tiles where one does not hold a sequence's tokens, but for fp32 at 128 dimensions (registers)
        c.tiles = per_seq * ratio > 16 && !(plan.p.dtype == HGA_F32 && plan.p.head_dim == 128) ? 2 : 1;
        c.tokens = std::min(per_seq, 16 * c.tiles / ratio);
        if (c.tokens > 1) {
            c.grid_units = static_cast<int>(std::min<int64_t>(n_tokens, (n_tokens + c.tokens - 1) / c.tokens + int64_t(n_seqs)));
            c.bytes = list_bytes;
        }
    }
    const int64_t units = static_cast<int64_t>((n_tokens + c.tokens - 1) / c.tokens) * plan.p.n_kv_heads;
    c.run = static_cast<int>(entries);
    // workgroups that the device holds at once or a few more (decode of 32 histories up to 32K, 4 heads of d128: 61 us with 4
    // a CU, 68-73 with 2, 3 or 6; 512 tokens of a 16K prompt in two tiles: 198 us with 2, 216 with 4)
    const int64_t want = (c.tiles == 2 ? 2 : 4) * static_cast<int64_t>(plan.n_cu);
    // A history is split where the join costs less than the pages that a workgroup would take one after another: over 64
    // pages, and from fewer where the units leave half of the device idle. 4 heads of d128, split and whole, in us: 1
    // sequence of 20 pages 8.8 and 9.9, of 32 9.0 and 13.4, of 64 9.3 and 20.5; 16 of 20 11.2 and 10.8, of 32 11.5 and
    // 14.0; 32 of 32 14.3 and 14.8, of 64 20.1 and 23.4. Tokens of one sequence in two tiles: 4 at 20 pages 18.0 and 23.6,
    // 64 at 20 pages 23.0 and 23.9, at 32 24.9 and 29.2; 128 at 32 33.5 and 29.4, at 60 38.0 and 40.9.
    const int64_t whole = 2 * units > plan.n_cu ? 64 : 16 + units / 8;
    if (entries > whole && units < want) {
        // A run is 16 pages or more where the device is filled: a part is written and read again. Below that it is the run
        // that gives each compute unit a workgroup, of two tiles every other one, 4 pages at the least (1 sequence of 64
        // pages: 9.3 us in runs of 4, 10.3 of 8, 12.0 of 16; 8 sequences: 12.7, 11.6, 13.0; 32 tokens in two tiles at 100
        // pages: 29.7 in runs of 7, 25.3 of 16).
        const int64_t fill = std::max<int64_t>(1, plan.n_cu / (units * c.tiles));
        const int64_t least = std::clamp<int64_t>((entries + fill - 1) / fill, 4, 16);
        const int64_t run = std::max(least, (units * entries + want - 1) / want);
        const int64_t counts = pad16(int64_t(n_tokens) * 4);
        const int64_t split_bytes = pad16(rows * plan.p.head_dim * 4) + pad16(rows * 8);
        const int64_t splits = std::min((entries + run - 1) / run, (ws_bytes - c.bytes - counts) / split_bytes);
        if (splits > 1) {
            c.splits = static_cast<int>(splits);
            c.run = static_cast<int>((entries + splits - 1) / splits);
            c.parts = c.bytes;
            c.part = c.parts + counts;
            c.part_ml = c.part + splits * rows * plan.p.head_dim * 4;
            c.bytes += counts + splits * split_bytes;
        }
    }
    // A workgroup of 8 wavefronts where a compute unit has one workgroup only (16 sequences of 20 pages, 4 heads of d128:
    // 10.8 us, 11.8 with 4; 64 of 31 listed pages: 16.6 and 17.4; 100 of 32 pages 30.2 and 25.3). One wavefront, which joins
    // nothing, from 24 a compute unit on (16K units of an fp32 head of d64: 95 us, 119 with 4; 6.4K units of 8 bf16 heads of
    // d128 over 10 pages: 112 and 126; at 1.6K units 31 and 27).
    if (c.tiles == 1 && units * c.splits <= plan.n_cu) c.waves = 8;
    if (c.tiles == 1 && c.splits == 1 && units >= 24 * plan.n_cu) c.waves = 1;
    return c;
}

}  // namespace

int64_t attend_tokens_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_list) {
    if (n_tokens == 0) return 0;
    const Cut c = cut_call(plan, n_tokens, n_seqs, max_pages, n_list, INT64_MAX);
    return c.bytes;
}

hipError_t launch_attend_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                                int64_t q_stride, const int32_t* list, int n_list, void* out, float* lse, void* ws,
                                int64_t ws_bytes, hipStream_t stream) {
    const Cut c = cut_call(plan, tok.n_tokens, tok.n_seqs, tok.max_pages, n_list, ws_bytes);
    AttendArgs a;
    a.list = list;
    a.n_list = n_list;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.run = c.run;
    a.splits = c.splits;
    a.lse = lse;
    char* w = static_cast<char*>(ws);
    int32_t* units = c.tokens > 1 ? reinterpret_cast<int32_t*>(w) : nullptr;
    a.units = units;
    a.parts = reinterpret_cast<int32_t*>(w + c.parts);
    a.part = reinterpret_cast<float*>(w + c.part);
    a.part_ml = reinterpret_cast<float*>(w + c.part_ml);
    if (units) {
        list_units_kernel<<<1, 1024, 0, stream>>>(tok.seq, tok.n_tokens, c.tokens, units);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value;
        constexpr bool kF32 = sizeof(T) == 4;
        constexpr int kTwo = kF32 && D == 128 ? 1 : 2;  // (cut_call gives those one tile)
        const auto by_waves = [&](auto one, auto four, auto eight) { return c.waves == 1 ? one : c.waves == 8 ? eight : four; };
        const auto f = c.tokens > 1 && c.tiles == 2 ? run<T, D, kTwo, 4, true>
                       : c.tokens > 1
                           ? by_waves(run<T, D, 1, 1, true>, run<T, D, 1, 4, true>, run<T, D, 1, 8, true>)
                       : kF32 && a.ratio <= 4
                           ? by_waves(run<T, D, 1, 1, false, kF32>, run<T, D, 1, 4, false, kF32>, run<T, D, 1, 8, false, kF32>)
                           : by_waves(run<T, D, 1, 1, false>, run<T, D, 1, 4, false>, run<T, D, 1, 8, false>);
        return f(plan, pool, tok, a, q, q_stride, out, c.grid_units, stream);
    };
    const bool f32 = plan.p.dtype == HGA_F32;
    if (plan.p.head_dim == 128)
        return f32 ? go(0.f, std::integral_constant<int, 128>()) : go(bf16_t(0), std::integral_constant<int, 128>());
    return f32 ? go(0.f, std::integral_constant<int, 64>()) : go(bf16_t(0), std::integral_constant<int, 64>());
}

}  // namespace hga

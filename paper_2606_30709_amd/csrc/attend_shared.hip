// Attention of a batch whose sequences share leading pages (Sec. 3.4 at the token's grain): the shared pages are read and
// multiplied once for many tokens, each token's own pages by itself, and the two are joined.
//
// A unit is one KV head and up to 16 kTiles / r slots: of one group, over its shared pages, or of one sequence, over the
// pages behind them.  Its query heads are the columns of the tiles, as in the attention of single tokens (attend_pages.hpp);
// a unit's pages are cut into runs, a workgroup each, whose partial results a second kernel joins in order.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "attend_pages.hpp"
#include "hga_device.hpp"
#include "prefixes.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

// How a call is cut: slots of a unit, pages of a run and runs of a unit at most, units; [0] the groups' pages, [1] the
// tokens' own.
struct Cut {
    int slots[2], run[2], most[2], units[2];
    int64_t counts, part, part_ml, bytes;  // the workspace, in bytes from its start
};

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A bf16 call's weights and values enter their product as f16.  A value is exact there: one code has two significant bits,
// and pages with a scale outside 2^-18 .. 2^13 (where f16 would run out of bits, or overflow) take bf16 and its further terms
// instead.  A weight has 11 bits, which leaves out 2^-12 of it at most where the result's own rounding to bf16 takes 2^-9,
// with one product where two bf16 terms need two.  Weights reach 2^kTop, 2^kLead when a reference is set: what lies below
// 2^-24 in f16, 2^-35 of the column's largest weight, counts as none.  fp32 calls take three bf16 terms throughout.
constexpr float kTop = 15.0f, kLead = 11.0f;

__device__ __forceinline__ f32x4 mfma_f16(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2h(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}
template <int kByte>
__device__ __forceinline__ uint32_t decode2h(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, kByte));
}

// Whether every scale of a page's values has an exponent byte of 109 .. 140.
template <int D>
__device__ __forceinline__ bool values_fit(const Values<D>& v) {
    uint32_t any = 0, all = ~0u;
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const uint32_t w = v.s[t] + 0x13131313u;  // 128 .. 159; a byte that carries into the next is out of range itself
        any |= w;
        all &= w;
    }
    return !__builtin_amdgcn_ballot_w64((any & 0x60606060u) != 0 || (~all & 0x80808080u) != 0);
}

// The running reference of every column, raised where a lane's scores exceed it by more than the slack.
template <int D, int kTiles>
__device__ __forceinline__ void raise_reference(const f32x4 (&sc)[kTiles][4], float scale, Acc<D, kTiles>& acc) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        float top = sc[i][0][0];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, sc[i][tt][x]);
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(top * scale > acc.m[i] + kTop) != 0, 0)) {
            top = max_groups(top) * scale;
            const bool grow = top > acc.m[i] + kTop;
            const float to = top - kLead;
            const float alpha = grow ? __builtin_amdgcn_exp2f(acc.m[i] - to) : 1.f;
            if (grow) acc.m[i] = to;
            acc.l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc.o[i][j] *= alpha;
        }
    }
}

template <int... kAt, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, kAt...>, F f) {
    (f(std::integral_constant<int, kAt>()), ...);
}

// Weights of half a page and their product with its values: kHalf in f16, else in bf16 of kParts terms a weight.  Two
// dimensions of the lane's at a time, so that few registers hold decoded values.
template <int D, bool kHalf, int kParts, int kTiles>
__device__ __forceinline__ void half_page(int u, const f32x4 (&sc)[kTiles][4], float scale, const Values<D>& v,
                                          Acc<D, kTiles>& acc) {
    constexpr int DL = D / 16;
    u32x4 w[kTiles][kParts];
    if constexpr (kHalf) {
#pragma unroll
        for (int i = 0; i < kTiles; ++i) {
            const float base = acc.m[i] == -INFINITY ? 0.f : acc.m[i];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float pv[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    pv[x] = __builtin_amdgcn_exp2f(fmaf(sc[i][2 * u + b][x], scale, -base));
                    acc.l[i] += pv[x];
                }
                w[i][0][2 * b] = pack2h(pv[0], pv[1]);
                w[i][0][2 * b + 1] = pack2h(pv[2], pv[3]);
            }
        }
    } else {
        half_weights<D, kParts, kTiles>(u, sc, scale, acc, w, nullptr);
    }
    if constexpr (kTiles > 1) __builtin_amdgcn_sched_barrier(0);  // or the registers do not suffice
    float vs[2][4];  // scales of the lane's rows
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) vs[b][r] = scale_of(v.s[2 * u + b] >> (8 * r) & 255u);
    each(std::make_integer_sequence<int, DL / 2>(), [&](auto at) {
        constexpr int j = decltype(at)::value;
        u32x4 even, odd;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r2 = 0; r2 < 2; ++r2) {
                const uint32_t* c = v.c[2 * u + b];
                uint32_t lo, hi;
                if constexpr (DL == 8) {
                    lo = kHalf ? decode2h<j>(c[2 * r2], vs[b][2 * r2]) : decode2<j>(c[2 * r2], vs[b][2 * r2]);
                    hi = kHalf ? decode2h<j>(c[2 * r2 + 1], vs[b][2 * r2 + 1]) : decode2<j>(c[2 * r2 + 1], vs[b][2 * r2 + 1]);
                } else {
                    lo = kHalf ? decode2h<j>(c[r2], vs[b][2 * r2]) : decode2<j>(c[r2], vs[b][2 * r2]);
                    hi = kHalf ? decode2h<j + 2>(c[r2], vs[b][2 * r2 + 1]) : decode2<j + 2>(c[r2], vs[b][2 * r2 + 1]);
                }
                even[2 * b + r2] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
                odd[2 * b + r2] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
            }
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int x = 0; x < kParts; ++x) {
                acc.o[i][2 * j] = kHalf ? mfma_f16(even, w[i][x], acc.o[i][2 * j]) : mfma(even, w[i][x], acc.o[i][2 * j]);
                acc.o[i][2 * j + 1] = kHalf ? mfma_f16(odd, w[i][x], acc.o[i][2 * j + 1]) : mfma(odd, w[i][x], acc.o[i][2 * j + 1]);
            }
        if constexpr (!kHalf) __builtin_amdgcn_sched_barrier(0);
    });
}

struct SharedArgs {
    int ratio;
    int slots[2], run[2], most[2], units[2];
    float* lse;
    int32_t* counts;  // [slot][2]: runs of its group's pages, of its own
    float* part;      // their results [run][slot][query head][d], not divided by the sum; the groups' runs first
    float* part_ml;   // ... and [run][slot][query head][2]: reference, sum
};

// The group of a slot: of the groups that begin at or before it the last, if the slot is inside it; -1: none.
__device__ __forceinline__ int group_of(const PrefixView& px, int n_tokens, int slot) {
    const int lane = threadIdx.x & 63;
    int n = 0;
    for (int g0 = 0; g0 <= px.n_groups; g0 += 64) {
        const int g = g0 + lane;
        const bool before = px.n_groups > 0 && g <= px.n_groups && px.begin[g] <= slot;
        n += __popcll(__builtin_amdgcn_ballot_w64(before));
    }
    if (n == 0 || n > px.n_groups) return -1;
    return slot >= px.first(n - 1, n_tokens) && slot < px.end(n - 1, n_tokens) ? n - 1 : -1;
}

// Slots [a, b) of unit `unit` of the groups, and its group; g -1: there is no such unit.
struct GroupUnit {
    int g, a, b;
};
__device__ __forceinline__ GroupUnit group_unit(const PrefixView& px, int n_tokens, int slots, int unit) {
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < px.n_groups; g0 += 64) {
        const int g = g0 + lane;
        int n = 0;
        if (g < px.n_groups) n = (px.end(g, n_tokens) - px.first(g, n_tokens) + slots - 1) / slots;
        const int to = wave_incl_scan_add(n);
        const uint64_t past = __builtin_amdgcn_ballot_w64(to > unit);
        if (past) {
            const int l = static_cast<int>(__builtin_ctzll(past));
            const int i = unit - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(n, l));
            const int a = px.first(g0 + l, n_tokens) + i * slots;
            return GroupUnit{g0 + l, a, min(a + slots, px.end(g0 + l, n_tokens))};
        }
        unit -= __builtin_amdgcn_readlane(to, 63);
    }
    return GroupUnit{-1, 0, 0};
}

// Slots of one group (over its shared pages, [0, shared)) or of one sequence (over its own, from `shared` on): their
// queries against run `split` of the pages.
template <typename T, int D, int kTiles, int kWaves, bool kOwn>
__device__ __forceinline__ void attend_slots(const PoolView& pool, const TokensView& tok, const PrefixView& px,
                                             const SharedArgs& a, const T* __restrict__ q, int64_t q_stride,
                                             T* __restrict__ out, float* smem, int h, int at, int n_slots, int shared,
                                             int split) {
    using F = PageFormat<D>;
    constexpr int kThreads = 64 * kWaves;
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;       // of a query
    constexpr int DL = F::kLaneDims;
    constexpr int kSteps = D / 32;
    constexpr int kAux = kOwn ? kNt : 0;  // a group's pages are read by its other units too
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));  // log2(e) / sqrt(d)
    float(*s_o)[16 * kTiles][D + 4] = reinterpret_cast<float(*)[16 * kTiles][D + 4]>(smem);
    float(*s_m)[16 * kTiles] = reinterpret_cast<float(*)[16 * kTiles]>(smem + kWaves * 16 * kTiles * (D + 4));
    float(*s_l)[16 * kTiles] = s_m + kWaves;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int columns = n_slots * a.ratio, heads = pool.n_kv * a.ratio;

    int pos[kTiles];
    int s = 0, last = -1, first = INT32_MAX;  // the row of the table, the tokens' largest and smallest positions
    u32x4 qf[kTiles][kTerms][kSteps];
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int c = 16 * i + m;
        const bool real = c < columns;
        const int t = real ? px.token(at + c / a.ratio, tok.n_tokens) : -1;
        int sc = 0, pc = 0;
        const bool in = t >= 0 && tok.at(t, sc, pc);
        pos[i] = in ? pc : -1;
        last = max(last, pos[i]);
        // columns past the last are no reason to look at rows one by one
        first = min(first, real ? pos[i] : INT32_MAX);
        s = in ? max(s, sc) : s;
        const T* from = q + (in ? t * q_stride : 0) + (static_cast<int64_t>(h) * a.ratio + c % a.ratio) * D + g * (D / 4);
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            float x[8] = {};
            if (in) load8(from + 8 * kk, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t w[kTerms];
                split2<kTerms>(x[2 * e], x[2 * e + 1], w);
#pragma unroll
                for (int y = 0; y < kTerms; ++y) qf[i][y][kk][e] = w[y];
            }
        }
    }
#pragma unroll
    for (int x = 1; x < 16; x *= 2) {
        last = max(last, __shfl_xor(last, x));
        first = min(first, __shfl_xor(first, x));
        s = max(s, __shfl_xor(s, x));
    }
    s = __builtin_amdgcn_readfirstlane(s);
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);
    const int n_all = !kOwn ? shared : last < 0 ? 0 : last / kPageRows + 1 - shared;
    bool whole = false;  // no other workgroup has a part of it
    if constexpr (kOwn) {
        const int parts = runs_of(n_all, a.run[1], a.most[1]);
        const int parts_group = last >= 0 ? runs_of(shared, a.run[0], a.most[0]) : 0;
        if (split == 0 && h == 0 && tid < n_slots) {
            a.counts[2 * (at + tid)] = parts_group;
            a.counts[2 * (at + tid) + 1] = parts;
        }
        if (split >= (parts_group == 0 ? max(parts, 1) : parts)) return;
        whole = parts_group == 0 && parts <= 1;
    }
    PageRun run = page_run(split, n_all, a.run[kOwn], a.most[kOwn]);
    if (kOwn) run = PageRun{run.a + shared, run.b + shared};
    const int to = last < 0 ? run.a : min(run.b, last / kPageRows + 1);

    Acc<D, kTiles> acc;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        acc.m[i] = -INFINITY;
        acc.l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < DL; ++j) acc.o[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    for (int e0 = run.a + wave; e0 < to; e0 += 64 * kWaves) {
        // the next 64 pages of this wavefront, one a lane
        SeenPage mine{-1, 0};
        const int chunk = e0 + lane * kWaves;
        if (chunk < to) mine = seen_page(pool, tok, s, last, chunk);
        uint64_t left = __builtin_amdgcn_ballot_w64(mine.rows > 0);
        if (!left) continue;
        int cur = static_cast<int>(__builtin_ctzll(left));
        const auto part = [&](int i, bool any) {
            return make_rsrc(pool.page(__builtin_amdgcn_readlane(mine.id, i)) + h * F::kBytes, any ? F::kBytes : 0);
        };
        Keys<D> k;
        Values<D> v;
        {
            const buf_rsrc r = part(cur, true);
            load_keys<D, kAux>(r, m, g, k);
            load_values<D, kAux>(r, m, g, v);
        }
        while (left) {
            left &= left - 1;
            const int nxt = left ? static_cast<int>(__builtin_ctzll(left)) : cur;
            const buf_rsrc r = part(nxt, left != 0);
            const int c = __builtin_amdgcn_readlane(chunk, cur);
            f32x4 sc[kTiles][4];
            page_scores<D, kTerms, kTiles>(k, qf, sc);
            if constexpr (kTiles == 1) load_keys<D, kAux>(r, m, g, k);
            if (__builtin_expect(first < c * kPageRows + kPageRows - 1, 0)) {
                __asm__ volatile("");  // a branch: most pages need none of this
                const int rows = __builtin_amdgcn_readlane(mine.rows, cur);
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int at_row = 16 * tt + 4 * g + x;
                        if (at_row >= rows) v.s[tt] = (v.s[tt] & ~(255u << (8 * x))) | 127u << (8 * x);
#pragma unroll
                        for (int i = 0; i < kTiles; ++i)
                            if (at_row > pos[i] - c * kPageRows) sc[i][tt][x] = -INFINITY;
                    }
                int seen[kTiles];
#pragma unroll
                for (int i = 0; i < kTiles; ++i) seen[i] = pos[i] - c * kPageRows;
                take_out_nan<D, kTiles>(v, m, g, seen, acc);
            }
            raise_reference<D, kTiles>(sc, scale, acc);
            const auto both_halves = [&](auto half, auto terms) {
                half_page<D, decltype(half)::value, decltype(terms)::value, kTiles>(0, sc, scale, v, acc);
                if constexpr (kTiles > 1) {
                    __builtin_amdgcn_sched_barrier(0);
                    load_keys<D, kAux>(r, m, g, k);
                }
                half_page<D, decltype(half)::value, decltype(terms)::value, kTiles>(1, sc, scale, v, acc);
            };
            if constexpr (sizeof(T) == 4)
                both_halves(std::false_type(), std::integral_constant<int, 3>());
            else if (__builtin_expect(values_fit<D>(v), 1))
                both_halves(std::true_type(), std::integral_constant<int, 1>());
            else
                both_halves(std::false_type(), std::integral_constant<int, 2>());
            load_values<D, kAux>(r, m, g, v);
            cur = nxt;
        }
    }

    // join the wavefronts: lane (m, g) of tile i holds column 16 i + m, dimensions (4 g + x) DL + j
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const float l = sum_groups(acc.l[i]);
        const int c = 16 * i + m;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < DL; ++j) s_o[wave][c][(4 * g + x) * DL + j] = acc.o[i][j][x];
        if (g == 0) {
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
        const int slot = at + r / a.ratio, head = h * a.ratio + r % a.ratio;
        if (whole) {
            const int t = px.token(slot, tok.n_tokens);
            if (t < 0) continue;
            const int64_t at_row = static_cast<int64_t>(t) * heads + head;
            out[at_row * D + c] = elem<T>::from_f32(l == 0.f ? 0.f : sum / l);
            if (a.lse && c == 0) a.lse[at_row] = natural_lse(ref, l);
        } else {
            const int64_t to_row = (static_cast<int64_t>(kOwn ? a.most[0] + split : split) * tok.n_tokens + slot) * heads + head;
            a.part[to_row * D + c] = sum;
            if (c == 0) {
                a.part_ml[2 * to_row] = top;
                a.part_ml[2 * to_row + 1] = l;
            }
        }
    }
}

template <typename T, int D, int kTiles, int kOwnTiles, int kWaves>
__global__ __launch_bounds__(64 * kWaves, 2) void attend_shared_kernel(PoolView pool, TokensView tok, PrefixView px,
                                                                       SharedArgs a, const T* __restrict__ q,
                                                                       int64_t q_stride, T* __restrict__ out) {
    extern __shared__ __align__(16) float smem[];
    // the groups' runs first, then the tokens' own; a unit's runs in the outer order
    uint32_t block = linear_block<64 * kWaves>();
    const uint32_t n_group = static_cast<uint32_t>(a.units[0]) * pool.n_kv * a.most[0];
    const bool own = block >= n_group;
    if (own) block -= n_group;
    const uint32_t row = static_cast<uint32_t>(a.units[own]) * pool.n_kv;
    if (block >= row * static_cast<uint32_t>(a.most[own])) return;
    const int split = static_cast<int>(block / row);
    const TokenHead where = token_head(block % row, pool.n_kv);
    if (!own) {
        const GroupUnit u = group_unit(px, tok.n_tokens, a.slots[0], where.t);
        if (u.g < 0) return;
        const int shared = px.shared(u.g, tok.max_pages);
        if (split >= runs_of(shared, a.run[0], a.most[0])) return;
        attend_slots<T, D, kTiles, kWaves, false>(pool, tok, px, a, q, q_stride, out, smem, where.h, u.a, u.b - u.a, shared,
                                                  split);
        return;
    }
    // a unit of own pages sequence by sequence
    const int end = min((where.t + 1) * a.slots[1], tok.n_tokens);
    for (int at = where.t * a.slots[1], next; at < end; at = next) {
        const int group = group_of(px, tok.n_tokens, at);
        const int first = px.token(at, tok.n_tokens), seq = first < 0 ? -1 : tok.seq[first];
        // the slots behind it of the same sequence and group
        for (next = at + 1; next < end; ++next) {
            const int t = px.token(next, tok.n_tokens);
            if (t < 0 || first < 0 || tok.seq[t] != seq || group_of(px, tok.n_tokens, next) != group) break;
        }
        attend_slots<T, D, kOwnTiles, kWaves, true>(pool, tok, px, a, q, q_stride, out, smem, where.h, at, next - at,
                                                    group < 0 ? 0 : px.shared(group, tok.max_pages), split);
        __syncthreads();  // LDS is the next sequence's
    }
}

// Joins the partial results of a slot's query head, in a fixed order: a workgroup a head, its threads D/4 columns of four
// dimensions by the groups of parts they add up.
template <typename T, int D>
__global__ __launch_bounds__(256) void join_shared_kernel(int n_tokens, int heads, PrefixView px, SharedArgs a,
                                                          T* __restrict__ out) {
    constexpr int kCols = D / 4, kGroups = 256 / kCols;
    __shared__ float4 s_o[kGroups][kCols];
    __shared__ float s_l[kGroups], s_m[kGroups];
    const int64_t row = linear_block<256>(), rows = static_cast<int64_t>(n_tokens) * heads;
    if (row >= rows) return;
    const int slot = static_cast<int>(row / heads), head = static_cast<int>(row % heads);
    const int t = px.token(slot, n_tokens);
    const int of_group = a.counts[2 * slot], of_own = a.counts[2 * slot + 1], parts = of_group + of_own;
    if (t < 0 || (of_group == 0 && of_own <= 1)) return;
    const int col = threadIdx.x % kCols, grp = threadIdx.x / kCols;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w0 = grp; w0 < parts; w0 += 4 * kGroups) {
        float2 ml[4];
        float4 x[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int w = min(w0 + y * kGroups, parts - 1);
            const int64_t at = (w < of_group ? w : a.most[0] + w - of_group) * rows + row;
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
    const int64_t to = static_cast<int64_t>(t) * heads + head;
    out[to * D + threadIdx.x] = elem<T>::from_f32(l == 0.f ? 0.f : sum / l);
    if (a.lse && threadIdx.x == 0) a.lse[to] = natural_lse(ref, l);
}

int64_t pad16(int64_t n) { return (n + 15) / 16 * 16; }

// Tiles of a group's unit: two, but for fp32 at 128 dimensions (registers).
template <typename T, int D>
constexpr int kTilesOf = sizeof(T) == 4 && D == 128 ? 1 : 2;

Cut cut_call(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups, int shared_hint, int own_hint,
             int64_t ws_bytes) {
    const int ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    const int tiles = plan.p.dtype == HGA_F32 && plan.p.head_dim == 128 ? 1 : 2;
    const int64_t rows = static_cast<int64_t>(n_tokens) * plan.p.n_q_heads;
    Cut c{};
    const int most_slots = 16 * tiles / ratio;
    const int per_seq = static_cast<int>((static_cast<int64_t>(n_tokens) + n_seqs - 1) / std::max(n_seqs, 1));
    c.slots[0] = most_slots;
    c.slots[1] = std::clamp(per_seq, 1, most_slots);
    c.units[0] = n_groups ? static_cast<int>(std::min<int64_t>(n_tokens, n_tokens / most_slots + static_cast<int64_t>(n_groups))) : 0;
    c.units[1] = (n_tokens + c.slots[1] - 1) / c.slots[1];
    const int64_t pages[2] = {std::clamp(shared_hint, 1, std::max(max_pages, 1)), std::clamp(own_hint, 1, std::max(max_pages, 1))};
    const int64_t want = 4 * static_cast<int64_t>(plan.n_cu);
    for (int i = 0; i < 2; ++i) {
        const int64_t units = static_cast<int64_t>(c.units[i]) * plan.p.n_kv_heads;
        c.run[i] = static_cast<int>(pages[i]);
        c.most[i] = 1;
        if (units == 0 || units >= want) continue;
        const int64_t run = std::max<int64_t>(16, (units * pages[i] + want - 1) / want);
        c.most[i] = static_cast<int>((pages[i] + run - 1) / run);
        c.run[i] = static_cast<int>((pages[i] + c.most[i] - 1) / c.most[i]);
    }
    const int64_t counts = pad16(static_cast<int64_t>(n_tokens) * 8);
    // fewer runs where the workspace holds no more
    const int64_t run_bytes = rows * (plan.p.head_dim + 2) * 4;
    const int64_t room = ws_bytes < counts ? 0 : (ws_bytes - counts) / run_bytes;
    while (c.most[0] + c.most[1] > room && (c.most[0] > 1 || c.most[1] > 1)) {
        const int i = c.most[0] >= c.most[1] ? 0 : 1;
        c.run[i] = static_cast<int>((pages[i] + --c.most[i] - 1) / std::max(c.most[i], 1));
    }
    c.part = counts;
    c.part_ml = c.part + (c.most[0] + c.most[1]) * rows * plan.p.head_dim * 4;
    c.bytes = c.part_ml + (c.most[0] + c.most[1]) * rows * 8;
    return c;
}

template <typename T, int D, int kOwnTiles>
hipError_t run(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const PrefixView& px, const SharedArgs& a,
               const void* q, int64_t q_stride, void* out, hipStream_t stream) {
    constexpr int kTiles = kTilesOf<T, D>, kWaves = 4, kThreads = 64 * kWaves;
    constexpr size_t lds = sizeof(float) * kWaves * 16 * kTiles * (D + 4 + 2);
    if (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = once_per_device(done, plan.device, [] {
            return hipFuncSetAttribute(reinterpret_cast<const void*>(attend_shared_kernel<T, D, kTiles, kOwnTiles, kWaves>),
                                       hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
        });
        if (e != hipSuccess) return e;
    }
    const int64_t n = static_cast<int64_t>(pool.n_kv) *
                      (static_cast<int64_t>(a.units[0]) * a.most[0] + static_cast<int64_t>(a.units[1]) * a.most[1]);
    attend_shared_kernel<T, D, kTiles, kOwnTiles, kWaves><<<grid_of(n, kThreads), kThreads, lds, stream>>>(
        pool, tok, px, a, static_cast<const T*>(q), q_stride, static_cast<T*>(out));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int heads = pool.n_kv * a.ratio;
    join_shared_kernel<T, D><<<grid_of(static_cast<int64_t>(tok.n_tokens) * heads, 256), 256, 0, stream>>>(
        tok.n_tokens, heads, px, a, static_cast<T*>(out));
    return hipGetLastError();
}

}  // namespace

int64_t attend_shared_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups, int shared_hint,
                            int own_hint, bool must) {
    if (n_tokens == 0) return 0;
    return cut_call(plan, n_tokens, n_seqs, max_pages, n_groups, shared_hint, own_hint, must ? 0 : INT64_MAX).bytes;
}

hipError_t launch_attend_shared(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const PrefixView& px,
                                int shared_hint, int own_hint, const void* q, int64_t q_stride, void* out, float* lse,
                                void* ws, int64_t ws_bytes, hipStream_t stream) {
    const Cut c = cut_call(plan, tok.n_tokens, tok.n_seqs, tok.max_pages, px.n_groups, shared_hint, own_hint, ws_bytes);
    SharedArgs a;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    for (int i = 0; i < 2; ++i) {
        a.slots[i] = c.slots[i];
        a.run[i] = c.run[i];
        a.most[i] = c.most[i];
        a.units[i] = c.units[i];
    }
    a.lse = lse;
    char* w = static_cast<char*>(ws);
    a.counts = reinterpret_cast<int32_t*>(w);
    a.part = reinterpret_cast<float*>(w + c.part);
    a.part_ml = reinterpret_cast<float*>(w + c.part_ml);
    const auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value;
        // one tile where a sequence's slots fill no more
        const auto f = c.slots[1] * a.ratio > 16 ? run<T, D, kTilesOf<T, D>> : run<T, D, 1>;
        return f(plan, pool, tok, px, a, q, q_stride, out, stream);
    };
    const bool f32 = plan.p.dtype == HGA_F32;
    if (plan.p.head_dim == 128)
        return f32 ? go(0.f, std::integral_constant<int, 128>()) : go(bf16_t(0), std::integral_constant<int, 128>());
    return f32 ? go(0.f, std::integral_constant<int, 64>()) : go(bf16_t(0), std::integral_constant<int, 64>());
}

}  // namespace hga

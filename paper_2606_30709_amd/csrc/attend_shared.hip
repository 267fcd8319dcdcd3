// Attention of a batch whose sequences share leading pages (Sec. 3.4 at the token's grain): the shared pages are read and
// multiplied once for many tokens, each token's own pages by itself, and the two are joined.  With keys o of the shared pages
// and o' of the own ones, m a reference near the largest score, l = sum exp(s - m), O = sum exp(s - m) v:
//   out = (e O + e' O') / (e l + e' l'),  e = exp(m - M), e' = exp(m' - M), M = max(m, m'),  lse = M + log(e l + e' l').
//
// A unit is one KV head and the slots that fill its tiles with columns, a column a query head (attend_pages.hpp): of one
// group, over its shared pages, or of one sequence, over the pages behind them.  Groups of few columns: a tile a workgroup,
// whose wavefronts take pages in turns and decode each for itself.  Of many: a workgroup's wavefronts hold columns of their
// own (4 times 32, or 16 in fp32 at 128 dimensions) and decode each page once for all of them, into LDS.  A unit's pages are cut into runs, a workgroup
// each, so that some 512 are at work; a second kernel joins the runs' results in order.
//
// 64 samples of a 16K prompt (32/4 heads d128 bf16): 49 us; 16 questions of 128 tokens about 16K: 545 us (1.0 PFLOP/s; 1.9 us
// a page, 1.14 PFLOP/s, 93 % of a large matrix product's rate here).
#include <algorithm>
#include <type_traits>
#include <utility>

#include "attend_pages.hpp"
#include "hga_device.hpp"
#include "prefixes.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// A bf16 call's weights and values enter their product as f16.  A value is exact there: one code has two significant bits,
// and pages with a scale outside 2^-18 .. 2^13 (where f16 would run out of bits, or overflow) take bf16 and its further terms
// instead.  A weight has 11 bits, which leaves out 2^-11 of it at most where the result's own rounding to bf16 takes 2^-8,
// with one product where two bf16 terms need two.  Weights reach 2^kTop, 2^kLead when a reference is set: f16 holds multiples
// of 2^-24, so that a weight is off by up to 2^-35 of the column's largest where that is more, and one below that counts as
// none.  fp32 calls take three bf16 terms throughout.
constexpr float kTop = 15.0f, kLead = 11.0f;
// References from here on are off by 1 or more in their last place, and by so much the weights from where f16 holds them (from
// 2^27 on the largest may pass its end).  Columns with such a one go on in bf16 terms.
constexpr float kFar = 0x1p24f;

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
struct ScaleRange {
    uint32_t any = 0, all = ~0u;  // of the bytes + 19: 128 .. 159 (one that carries into the next is out of range itself)

    __device__ __forceinline__ void add(const uint32_t (&s)[4]) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const uint32_t w = s[t] + 0x13131313u;
            any |= w;
            all &= w;
        }
    }
    __device__ __forceinline__ bool fits() const {
        return !__builtin_amdgcn_ballot_w64((any & 0x60606060u) != 0 || (~all & 0x80808080u) != 0);
    }
};
// Zeros fit whatever their scale (a block of zeros is stored with the smallest one), unless they stand for NaN: whether rows
// whose scales do not fit hold nothing else in any lane's dimensions.
template <int D>
__device__ __forceinline__ bool zeros_fit(const Values<D>& v) {
    uint32_t bad = 0;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const uint32_t e = v.s[t] >> (8 * x) & 255u;
            const uint32_t codes = D == 128 ? v.c[t][x % (D / 32)] : v.c[t][x / 2] >> (16 * (x % 2)) & 0xffffu;
            bad |= e - 109u > 31u ? (codes & 0x77777777u) | static_cast<uint32_t>(e == 255u) : 0u;
        }
    return !__builtin_amdgcn_ballot_w64(bad != 0);
}
template <int D>
__device__ __forceinline__ bool values_fit(const Values<D>& v) {
    ScaleRange r;
    r.add(v.s);
    return __builtin_expect(r.fits(), 1) || zeros_fit<D>(v);
}

// The largest of a lane's scores.
template <int kTiles>
__device__ __forceinline__ void largest(const f32x4 (&sc)[kTiles][4], float (&top)[kTiles]) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        top[i] = sc[i][0][0];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int x = 0; x < 4; ++x) top[i] = fmaxf(top[i], sc[i][tt][x]);
    }
}
// The running reference of every column, raised where a lane's scores exceed it by more than the slack, compared as the
// weights' exponents are formed: rounded once.  far(): some column's is kFar or more now.
template <int D, int kTiles, typename F>
__device__ __forceinline__ void raise_reference(const float (&tops)[kTiles], float scale, Acc<D, kTiles>& acc, F far) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(fmaf(tops[i], scale, -acc.m[i]) > kTop) != 0, 0)) {
            const float top = max_groups(tops[i]);
            const bool grow = fmaf(top, scale, -acc.m[i]) > kTop;
            const float to = fmaf(top, scale, -kLead);
            const float alpha = grow ? __builtin_amdgcn_exp2f(acc.m[i] - to) : 1.f;
            if (grow) acc.m[i] = to;
            if (__builtin_amdgcn_ballot_w64(grow && !(fabsf(to) < kFar))) far();
            acc.l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc.o[i][j] *= alpha;
        }
}
template <int D, int kTiles, typename F>
__device__ __forceinline__ void raise_reference(const f32x4 (&sc)[kTiles][4], float scale, Acc<D, kTiles>& acc, F far) {
    float top[kTiles];
    largest<kTiles>(sc, top);
    raise_reference<D, kTiles>(top, scale, acc, far);
}

template <int... kAt, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, kAt...>, F f) {
    (f(std::integral_constant<int, kAt>()), ...);
}

// The lane's dimensions 2 j and 2 j + 1 of half a page's rows, whose scales are vs, paired by row: what byte kByte of each
// row's codes holds (kRow: bytes from one row's codes to the next one's in a word).
template <int D, bool kHalf, int kByte>
__device__ __forceinline__ void value_pair(const uint32_t (&c0)[D / 32], const uint32_t (&c1)[D / 32], const float (&vs)[2][4],
                                           u32x4& even, u32x4& odd) {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r2 = 0; r2 < 2; ++r2) {
            const uint32_t* c = b ? c1 : c0;
            const float s0 = vs[b][2 * r2], s1 = vs[b][2 * r2 + 1];
            uint32_t lo, hi;
            if constexpr (D == 128) {
                lo = kHalf ? decode2h<kByte>(c[2 * r2], s0) : decode2<kByte>(c[2 * r2], s0);
                hi = kHalf ? decode2h<kByte>(c[2 * r2 + 1], s1) : decode2<kByte>(c[2 * r2 + 1], s1);
            } else {
                lo = kHalf ? decode2h<kByte>(c[r2], s0) : decode2<kByte>(c[r2], s0);
                hi = kHalf ? decode2h<kByte + 2>(c[r2], s1) : decode2<kByte + 2>(c[r2], s1);
            }
            even[2 * b + r2] = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
            odd[2 * b + r2] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        }
}

// Weights of half a page and their product with its values: kHalf in f16, else in bf16 of kParts terms a weight.  `values`
// gives the lane's dimensions 2 j and 2 j + 1 at a time, so that few registers hold decoded values.
template <int D, bool kHalf, int kParts, int kTiles, typename V>
__device__ __forceinline__ void half_page(int u, const f32x4 (&sc)[kTiles][4], float scale, V values, Acc<D, kTiles>& acc) {
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
    each(std::make_integer_sequence<int, D / 32>(), [&](auto at) {
        constexpr int j = decltype(at)::value;
        u32x4 even, odd;
        values(at, even, odd);
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
            for (int x = 0; x < kParts; ++x) {
                acc.o[i][2 * j] = kHalf ? mfma_f16(even, w[i][x], acc.o[i][2 * j]) : mfma(even, w[i][x], acc.o[i][2 * j]);
                acc.o[i][2 * j + 1] = kHalf ? mfma_f16(odd, w[i][x], acc.o[i][2 * j + 1]) : mfma(odd, w[i][x], acc.o[i][2 * j + 1]);
            }
    });
}

// The scales of a lane's eight rows of half a page.
__device__ __forceinline__ void row_scales(uint32_t w0, uint32_t w1, float (&vs)[2][4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        vs[0][r] = scale_of(w0 >> (8 * r) & 255u);
        vs[1][r] = scale_of(w1 >> (8 * r) & 255u);
    }
}
// Rows of a lane from `rows` on get a scale of 1: they may hold anything.
__device__ __forceinline__ void cut_rows(uint32_t (&s)[4], int g, int rows) {
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (16 * tt + 4 * g + x >= rows) s[tt] = (s[tt] & ~(255u << (8 * x))) | 127u << (8 * x);
}

constexpr int kWaves = 4, kThreads = 64 * kWaves;

struct SharedArgs {
    int ratio;
    int slots[2], run[2], most[2], units[2];
    bool alone;       // a wavefront by itself takes a unit of own pages, not a workgroup
    float* lse;
    int32_t* counts;  // [slot][2]: runs of its group's pages, of its own
    float* part;      // their results [run][slot][query head][d], not divided by the sum; the groups' runs first
    float* part_ml;   // ... and [run][slot][query head][2]: reference, sum
};

// Slots [a, b) of a unit of the groups, its group (-1: there is no such unit) and the pages that this shares.
struct GroupUnit {
    int g, a, b, shared;
};
__device__ __forceinline__ GroupUnit group_unit(const PrefixView& px, const TokensView& tok, int slots, int unit) {
    const int lane = threadIdx.x & 63;
    for (int g0 = 0; g0 < px.n_groups; g0 += 64) {
        const int g = g0 + lane;
        int a = 0, b = 0, shared = 0;
        if (g < px.n_groups) {
            a = px.first(g, tok.n_tokens);
            b = px.end(g, tok.n_tokens);
            shared = px.shared(g, tok.max_pages);
        }
        const int n = (b - a + slots - 1) / slots, to = wave_incl_scan_add(n);
        const uint64_t past = __builtin_amdgcn_ballot_w64(to > unit);
        if (past) {
            const int l = static_cast<int>(__builtin_ctzll(past));
            const int i = unit - (__builtin_amdgcn_readlane(to, l) - __builtin_amdgcn_readlane(n, l));
            const int from = __builtin_amdgcn_readlane(a, l) + i * slots;
            return GroupUnit{g0 + l, from, min(from + slots, __builtin_amdgcn_readlane(b, l)),
                             __builtin_amdgcn_readlane(shared, l)};
        }
        unit -= __builtin_amdgcn_readlane(to, 63);
    }
    return GroupUnit{-1, 0, 0, 0};
}

// The groups of slots [from, from + n), n <= 16, a lane each (of the groups that begin at or before a slot the last, if the
// slot is inside it; -1: none), and the pages that they share.
struct SlotGroup {
    int g, shared;
};
__device__ __forceinline__ SlotGroup slot_groups(const PrefixView& px, const TokensView& tok, int from, int n) {
    const int lane = threadIdx.x & 63, slot = from + min(lane, n - 1);
    int lo = 0, hi = px.n_groups > 0 ? px.n_groups + 1 : 0;  // begin[0, lo) <= slot < begin[hi, ...)
    if (hi > 0 && hi <= 64) {
        const int begin = lane < hi ? px.begin[lane] : INT32_MAX;
        for (int i = 0; i < n; ++i) {
            const int before = __popcll(__builtin_amdgcn_ballot_w64(begin <= from + i));
            if (slot == from + i) lo = before;
        }
    } else {
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (px.begin[mid] <= slot)
                lo = mid + 1;
            else
                hi = mid;
        }
    }
    if (lo == 0 || lo > px.n_groups || slot < px.first(lo - 1, tok.n_tokens) || slot >= px.end(lo - 1, tok.n_tokens))
        return SlotGroup{-1, 0};
    return SlotGroup{lo - 1, px.shared(lo - 1, tok.max_pages)};
}

__device__ __forceinline__ void add_scaled(float4& o, float f, const float4& x) {
    o.x += f * x.x;
    o.y += f * x.y;
    o.z += f * x.z;
    o.w += f * x.w;
}
// Four dimensions of a result, o / l.
__device__ __forceinline__ void store4(float* to, const float4& o, float l) {
    *reinterpret_cast<float4*>(to) =
        l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x / l, o.y / l, o.z / l, o.w / l);
}
__device__ __forceinline__ void store4(bf16_t* to, const float4& o, float l) {
    *reinterpret_cast<uint2*>(to) =
        l == 0.f ? make_uint2(0u, 0u) : make_uint2(pack2(o.x / l, o.y / l), pack2(o.z / l, o.w / l));
}
// Four dimensions of a row: of the results (whole), or of the partial ones.
template <typename T, int D>
__device__ __forceinline__ void put4(const SharedArgs& a, T* out, bool whole, int64_t row, int dim, const float4& o, float top,
                                     float l) {
    if (whole) {
        store4(out + row * D + dim, o, l);
        if (a.lse && dim == 0) a.lse[row] = natural_lse(top == -INFINITY ? 0.f : top, l);
    } else {
        *reinterpret_cast<float4*>(a.part + row * D + dim) = o;
        if (dim == 0) *reinterpret_cast<float2*>(a.part_ml + 2 * row) = make_float2(top, l);
    }
}

// The largest of a row of 16 lanes, in all of them.
template <int kCtrl>
__device__ __forceinline__ int max_by(int x) {
    return max(x, __builtin_amdgcn_mov_dpp(x, kCtrl, 0xf, 0xf, true));
}
__device__ __forceinline__ int row_max(int x) {
    return max_by<0x128>(max_by<0x124>(max_by<0x4E>(max_by<0xB1>(x))));  // pairs, quads, then rotations by 4 and 8
}

// A wavefront's columns: columns c0 + 16 i + m of the slots from `at` on.
template <typename T, int D, int kTiles>
struct Columns {
    static constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;  // of a query
    u32x4 qf[kTiles][kTerms][D / 32];
    int pos[kTiles];
    int s, last, first;  // the row of the table, the tokens' largest and smallest positions
};
template <typename T, int D, int kTiles>
__device__ __forceinline__ void load_columns(const PoolView& pool, const TokensView& tok, const PrefixView& px, int ratio,
                                             const T* q, int64_t q_stride, int h, int at, int c0, int columns, int m, int g,
                                             Columns<T, D, kTiles>& r) {
    constexpr int kTerms = Columns<T, D, kTiles>::kTerms;
    int s = 0, last = -1, first = INT32_MAX;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const int c = c0 + 16 * i + m;
        const bool real = c < columns;
        // (a column past the last has the last slot's query)
        const int t = px.token(at + min(c, columns - 1) / ratio, tok.n_tokens);
        int sc = 0, pc = 0;
        const bool there = t >= 0 && tok.at(t, sc, pc), in = real && there;
        r.pos[i] = in ? pc : -1;
        last = max(last, r.pos[i]);
        // columns past the last are no reason to look at rows one by one
        first = min(first, real ? r.pos[i] : INT32_MAX);
        s = in ? max(s, sc) : s;
        // (not only if it is in the table: its place need not be known yet)
        const T* from = q + max(t, 0) * q_stride + (static_cast<int64_t>(h) * ratio + c % ratio) * D + g * (D / 4);
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            float x[8];
            load8(from + 8 * kk, x);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t w[kTerms];
                split2<kTerms>(x[2 * e], x[2 * e + 1], w);
#pragma unroll
                for (int y = 0; y < kTerms; ++y) r.qf[i][y][kk][e] = w[y];
            }
        }
        // an idle token's query may be anything, and would decide which types the others' products take
        if (__builtin_expect(__builtin_amdgcn_ballot_w64(!there) != 0, 0))
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
#pragma unroll
                for (int y = 0; y < kTerms; ++y) r.qf[i][y][kk] = there ? r.qf[i][y][kk] : u32x4{0u, 0u, 0u, 0u};
    }
    r.s = __builtin_amdgcn_readfirstlane(row_max(s));
    r.first = -1 - __builtin_amdgcn_readfirstlane(row_max(-1 - first));
    r.last = __builtin_amdgcn_readfirstlane(row_max(last));
}
template <int D, int kTiles>
__device__ __forceinline__ void clear(Acc<D, kTiles>& acc) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        acc.m[i] = -INFINITY;
        acc.l[i] = 0.f;
#pragma unroll
        for (int j = 0; j < D / 16; ++j) acc.o[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
}
// Scores of rows that a column does not see (`seen`: the last it sees) to -infinity.
template <int kTiles>
__device__ __forceinline__ void hide_rows(const int (&seen)[kTiles], int g, f32x4 (&sc)[kTiles][4]) {
#pragma unroll
    for (int tt = 0; tt < 4; ++tt)
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
                if (16 * tt + 4 * g + x > seen[i]) sc[i][tt][x] = -INFINITY;
}
// A bf16 call's page in f16 if its values allow that, in two bf16 terms if not; an fp32 call's in three.
template <typename T, typename F>
__device__ __forceinline__ void by_terms(bool fit, F f) {
    if constexpr (sizeof(T) == 4)
        f(std::false_type(), std::integral_constant<int, 3>());
    else if (__builtin_expect(fit, 1))
        f(std::true_type(), std::integral_constant<int, 1>());
    else
        f(std::false_type(), std::integral_constant<int, 2>());
}

// A wavefront's results, from its registers: lane (m, g) of tile i holds column c0 + 16 i + m, dimensions (4 g + x) DL + j.
template <typename T, int D, int kTiles, typename R>
__device__ __forceinline__ void put_columns(const SharedArgs& a, T* out, const Acc<D, kTiles>& acc, int c0, int columns, int m,
                                            int g, R row_of) {
    constexpr int DL = D / 16;
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        const float l = sum_groups(acc.l[i]);
        const int c = c0 + 16 * i + m;
        if (c >= columns) continue;
        bool whole;
        const int64_t row = row_of(c, whole);
        if (row < 0) continue;
#pragma unroll
        for (int x = 0; x < 4; ++x)
#pragma unroll
            for (int j = 0; j < DL; j += 4)
                put4<T, D>(a, out, whole, row, (4 * g + x) * DL + j,
                           make_float4(acc.o[i][j][x], acc.o[i][j + 1][x], acc.o[i][j + 2][x], acc.o[i][j + 3][x]), acc.m[i], l);
    }
}

// Up to 16 columns of one group (over its shared pages, [0, shared)) or of one sequence (over its own, from `shared` on):
// their queries against run `split` of the pages, which the workgroup's wavefronts take in turns and join (kAlone: this one by
// itself, without a barrier).
template <typename T, int D, bool kOwn, bool kAlone>
__device__ __forceinline__ void attend_slots(const PoolView& pool, const TokensView& tok, const PrefixView& px,
                                             const SharedArgs& a, const T* __restrict__ q, int64_t q_stride,
                                             T* __restrict__ out, float* smem, int h, int at, int n_slots, int shared,
                                             int split) {
    using F = PageFormat<D>;
    constexpr int kTerms = Columns<T, D, 1>::kTerms, DL = D / 16, kTeam = kAlone ? 1 : kWaves;
    constexpr int kAux = kOwn ? kNt : 0;  // a group's pages are read by its other units too
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));  // log2(e) / sqrt(d)
    const int tid = threadIdx.x, wave = kAlone ? 0 : tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    const int columns = n_slots * a.ratio, heads = pool.n_kv * a.ratio;

    Columns<T, D, 1> col;
    load_columns<T, D, 1>(pool, tok, px, a.ratio, q, q_stride, h, at, 0, columns, m, g, col);
    const int last = col.last;
    const int n_all = !kOwn ? shared : last < 0 ? 0 : last / kPageRows + 1 - shared;
    bool whole = false;  // there is no other part of it
    if constexpr (kOwn) {
        const int parts = runs_of(n_all, a.run[1], a.most[1]), of_group = last >= 0 ? runs_of(shared, a.run[0], a.most[0]) : 0;
        if (split == 0 && h == 0 && wave == 0 && lane < n_slots) {
            a.counts[2 * (at + lane)] = of_group;
            a.counts[2 * (at + lane) + 1] = parts;
        }
        whole = of_group == 0 && parts <= 1;
        if (split >= (whole ? 1 : parts)) return;
    }
    PageRun run = page_run(split, n_all, a.run[kOwn], a.most[kOwn]);
    if (kOwn) run = PageRun{run.a + shared, run.b + shared};
    const int to = last < 0 ? run.a : min(run.b, last / kPageRows + 1);

    Acc<D, 1> acc;
    clear(acc);
    bool far = false;
    for (int e0 = run.a + wave; e0 < to; e0 += 64 * kTeam) {
        // the next 64 pages of this wavefront, one a lane
        SeenPage mine{-1, 0};
        const int chunk = e0 + lane * kTeam;
        if (chunk < to) mine = seen_page(pool, tok, col.s, last, chunk);
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
            f32x4 sc[1][4];
            page_scores<D, kTerms, 1>(k, col.qf, sc);
            load_keys<D, kAux>(r, m, g, k);
            if (__builtin_expect(col.first < c * kPageRows + kPageRows - 1, 0)) {
                __asm__ volatile("");  // a branch: most pages need none of this
                cut_rows(v.s, g, __builtin_amdgcn_readlane(mine.rows, cur));
                const int seen[1] = {col.pos[0] - c * kPageRows};
                hide_rows<1>(seen, g, sc);
                take_out_nan<D, 1>(v, m, g, seen, acc);
            }
            raise_reference<D, 1>(sc, scale, acc, [&] { far = true; });
            by_terms<T>(sizeof(T) == 2 && !far && values_fit<D>(v), [&](auto half, auto terms) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    float vs[2][4];
                    row_scales(v.s[2 * u], v.s[2 * u + 1], vs);
                    half_page<D, decltype(half)::value, decltype(terms)::value, 1>(u, sc, scale, [&](auto j, u32x4& even, u32x4& odd) {
                        value_pair<D, decltype(half)::value, decltype(j)::value>(v.c[2 * u], v.c[2 * u + 1], vs, even, odd);
                    }, acc);
                }
            });
            load_values<D, kAux>(r, m, g, v);
            cur = nxt;
        }
    }

    const int64_t rows = static_cast<int64_t>(tok.n_tokens) * heads;
    // the row of column c's results: of its token, of its slot if they are partial
    const auto row_of = [&](int c, bool& all) {
        const int slot = at + c / a.ratio, head = h * a.ratio + c % a.ratio;
        all = kOwn && whole;
        if (!all) return (kOwn ? a.most[0] + split : split) * rows + static_cast<int64_t>(slot) * heads + head;
        const int t = px.token(slot, tok.n_tokens);
        return t < 0 ? int64_t(-1) : static_cast<int64_t>(t) * heads + head;
    };
    if constexpr (kAlone) {
        put_columns<T, D, 1>(a, out, acc, 0, columns, m, g, row_of);
        return;
    }
    // join the wavefronts
    float(*s_o)[16][D + 4] = reinterpret_cast<float(*)[16][D + 4]>(smem);
    float(*s_m)[16] = reinterpret_cast<float(*)[16]>(smem + kWaves * 16 * (D + 4));
    float(*s_l)[16] = s_m + kWaves;
    const float l0 = sum_groups(acc.l[0]);
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int j = 0; j < DL; ++j) s_o[wave][m][(4 * g + x) * DL + j] = acc.o[0][j][x];
    if (g == 0) {
        s_m[wave][m] = acc.m[0];
        s_l[wave][m] = l0;
    }
    __syncthreads();
    // four dimensions of a column a thread
    for (int i = tid; i < columns * (D / 4); i += kThreads) {
        const int c = i / (D / 4), dim = i % (D / 4) * 4;
        float top = s_m[0][c];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][c]);
        const float ref = top == -INFINITY ? 0.f : top;
        float l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = part_weight(s_m[w][c], ref);
            l += f * s_l[w][c];
            add_scaled(o, f, *reinterpret_cast<const float4*>(&s_o[w][c][dim]));
        }
        bool all;
        const int64_t row = row_of(c, all);
        if (row >= 0) put4<T, D>(a, out, all, row, dim, o, top, l);
    }
}

// A wavefront's share of decoding a page that the workgroup uses: words of key codes, of one 16-key tile; and the codes of
// half the page's values, of which it decodes kPairs dimensions 2 j, 2 j + 1 of the lane's.  In LDS a page is operands of a
// wavefront's 64 lanes: [4 tiles][kSteps] of keys, then [2 halves][D/16 dimensions] of values.
template <int D>
struct RawKeys {
    static constexpr int kSteps = D / 32, kWords = 4 * kSteps / kWaves;
    uint32_t k[kWords], s;

    __device__ __forceinline__ void load(buf_rsrc r, int wave, int m, int g) {
        using F = PageFormat<D>;
        const uint32_t key = F::key_code(16 * wave + m, g * (D / 4));
        if constexpr (kWords == 4) {
            const vec16 x = buf_load16(r, key);
#pragma unroll
            for (int i = 0; i < 4; ++i) k[i] = x.w[i];
        } else {
            const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, key, 0, 0));
            k[0] = x.x;
            k[1] = x.y;
        }
        s = static_cast<uint32_t>(buf_load_i32(r, F::key_scale(m, g * (D / 4) / 32)));
    }
    // word i
    __device__ __forceinline__ void store(u32x4* page, int wave, int lane, int i) const {
        const float scale = scale_of(s >> (8 * wave) & 255u);
        page[(wave * kSteps + i) * 64 + lane] =
            u32x4{decode2<0>(k[i], scale), decode2<1>(k[i], scale), decode2<2>(k[i], scale), decode2<3>(k[i], scale)};
    }
    __device__ __forceinline__ void store(u32x4* page, int wave, int lane) const {
#pragma unroll
        for (int i = 0; i < kWords; ++i) store(page, wave, lane, i);
    }
};
template <int D>
struct RawValues {
    static constexpr int kSteps = D / 32, kPairs = 2 * kSteps / kWaves;
    uint32_t v[2][D / 32];

    __device__ __forceinline__ void load(buf_rsrc r, int wave, int m, int g) {
        using F = PageFormat<D>;
        const int u = wave * kPairs / kSteps;
#pragma unroll
        for (int b = 0; b < 2; ++b)
            load_codes<D, 0>(r, F::value_code(4 * g, m * F::kLaneDims) + (2 * u + b) * (F::value_code(16, 0) - F::kCodes), v[b]);
    }
    // pair kAt
    template <bool kHalf, int kAt>
    __device__ __forceinline__ void store(const uint32_t (&vs)[4], u32x4* page, int wave, int lane) const {
        const int u = wave * kPairs / kSteps, j0 = wave * kPairs % kSteps;
        float s[2][4];
        row_scales(u ? vs[2] : vs[0], u ? vs[3] : vs[1], s);
        uint32_t c[2][D / 32];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int i = 0; i < D / 32; ++i) c[b][i] = v[b][i] >> (8 * j0);
        u32x4 even, odd;
        value_pair<D, kHalf, kAt>(c[0], c[1], s, even, odd);
        u32x4* to = page + (4 * kSteps + (u * kSteps + j0 + kAt) * 2) * 64 + lane;
        to[0] = even;
        to[64] = odd;
    }
    template <bool kHalf>
    __device__ __forceinline__ void store(const uint32_t (&vs)[4], u32x4* page, int wave, int lane) const {
        each(std::make_integer_sequence<int, kPairs>(),
             [&](auto at) { store<kHalf, decltype(at)::value>(vs, page, wave, lane); });
    }
};
template <int D>
__device__ __forceinline__ void load_value_scales(buf_rsrc r, int m, int g, uint32_t (&s)[4]) {
    const vec16 x = buf_load16(r, PageFormat<D>::value_scale(4 * g, m * PageFormat<D>::kLaneDims / 32));
#pragma unroll
    for (int t = 0; t < 4; ++t) s[t] = x.w[t];
}

// Many columns of one group, kTiles tiles a wavefront, against run `split` of its pages.  The wavefronts decode a page once,
// a share each, into LDS.  A page's weights are formed beside the products of the next one's keys, and its values are
// multiplied beside the decoding of further pages, so that neither unit of a SIMD waits for the other: a wavefront issues
// some 64 products (1,024 cycles of the matrix unit), 170 vector instructions and 32 exponentials a page, two wavefronts a
// SIMD.  16 questions of 128 tokens after 16K: 814 us with each wavefront decoding for itself, 640 through LDS, 583 with what
// is rare outside the loop (its registers made the loop spill), 543 with the products beside the weights.  Four tiles a
// wavefront, one wavefront a SIMD: 1,777 (spills); eight wavefronts to a page: 607 (a barrier's phases meet).
// At d128 bf16 it holds 256 registers and spills 76 bytes a lane, none of which the loop over pages touches (but for its branch
// that raises a reference).
// Only for columns that see all of the run, and for a bf16 call values that fit f16 and references below kFar; false: they do
// not (looked at every 64 pages), nothing is stored.
template <typename T, int D, int kTiles>
__device__ __forceinline__ bool attend_wide(const PoolView& pool, const TokensView& tok, const PrefixView& px,
                                            const SharedArgs& a, const T* __restrict__ q, int64_t q_stride, float* smem, int h,
                                            int at_slot, int n_slots, int shared, int split) {
    using F = PageFormat<D>;
    constexpr int kSteps = D / 32, kFrags = 8 * kSteps, kTerms = Columns<T, D, kTiles>::kTerms, kParts = sizeof(T) == 4 ? 3 : 1;
    constexpr bool kHalf = sizeof(T) == 2;
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));  // log2(e) / sqrt(d)
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, m = lane & 15, g = lane >> 4;
    u32x4* const pages = reinterpret_cast<u32x4*>(smem);                // [2][kFrags][64]
    int* const s_of = reinterpret_cast<int*>(smem + 2 * kFrags * 256);  // [wave][2], then [wave]: no reason to stop
    const int columns = n_slots * a.ratio, c0 = wave * 16 * kTiles, heads = pool.n_kv * a.ratio;

    Columns<T, D, kTiles> col;
    load_columns<T, D, kTiles>(pool, tok, px, a.ratio, q, q_stride, h, at_slot, c0, columns, m, g, col);
    int s = 0, first = INT32_MAX;  // of the tokens that are some
#pragma unroll
    for (int i = 0; i < kTiles; ++i) first = min(first, col.pos[i] < 0 ? INT32_MAX : col.pos[i]);
    first = -1 - row_max(-1 - first);
    int* const s_fit = s_of + 2 * kWaves;
    if (lane == 0) {
        s_of[2 * wave] = col.s;
        s_of[2 * wave + 1] = first;
        s_fit[wave] = 1;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        s = max(s, s_of[2 * w]);
        first = min(first, s_of[2 * w + 1]);
    }
    s = __builtin_amdgcn_readfirstlane(s);
    first = __builtin_amdgcn_readfirstlane(first);
    PageRun run = page_run(split, shared, a.run[0], a.most[0]);
    if (first == INT32_MAX) run.b = run.a;  // no token: no row of the table either
    if (first < run.b * kPageRows - 1) return false;

    Acc<D, kTiles> acc;
    clear(acc);
    ScaleRange range;
    for (int e0 = run.a; e0 < run.b; e0 += 64) {
        // the next 64 pages, one a lane
        int id = -1;
        if (e0 + lane < run.b) id = tok.page_id(s, e0 + lane);
        uint64_t left = __builtin_amdgcn_ballot_w64(pool.has(id));
        if (!left) continue;
        // lane i's page; i -1: an empty one, whose loads return zeros
        const auto part = [&](int i) {
            return make_rsrc(pool.page(__builtin_amdgcn_readlane(id, max(i, 0))) + h * F::kBytes, i >= 0 ? F::kBytes : 0);
        };
        const auto pop = [&] {
            const int i = left ? static_cast<int>(__builtin_ctzll(left)) : -1;
            left &= left - 1;
            return i;
        };
        // A page is multiplied, next the keys of n1 (in LDS), whose values are decoded meanwhile with the keys of n2; the
        // buffers of a page are those of its number's last bit.
        int n1, n2, bit = 0;
        RawKeys<D> rk;
        RawValues<D> rv;
        uint32_t vs[4], vs_after[4];
        {
            const buf_rsrc r = part(pop());
            n1 = pop();
            n2 = pop();
            RawKeys<D> rk1;
            rk.load(r, wave, m, g);
            rv.load(r, wave, m, g);
            load_value_scales<D>(r, m, g, vs);
            rk1.load(part(n1), wave, m, g);
            rk.store(pages, wave, lane);
            range.add(vs);
            rv.template store<kHalf>(vs, pages, wave, lane);
            rk1.store(pages + kFrags * 64, wave, lane);
        }
        rk.load(part(n2), wave, m, g);
        rv.load(part(n1), wave, m, g);
        load_value_scales<D>(part(n1), m, g, vs);
        load_value_scales<D>(part(n2), m, g, vs_after);
        if (n1 < 0)
#pragma unroll
            for (int t = 0; t < 4; ++t) vs[t] = 0x7f7f7f7fu;  // (no page: it fits)
        __syncthreads();
        f32x4 sc[kTiles][4];
        float top[kTiles];
        const auto fetch = [&](const u32x4* keys, int tt, u32x4 (&kf)[kSteps]) {
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk) kf[kk] = keys[(tt * kSteps + kk) * 64 + lane];
        };
        // scores of 16 keys
        const auto scores = [&](const u32x4 (&kf)[kSteps], int tt) {
#pragma unroll
            for (int i = 0; i < kTiles; ++i) sc[i][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < kSteps; ++kk)
#pragma unroll
                for (int x = 0; x < kTerms; ++x)
#pragma unroll
                    for (int i = 0; i < kTiles; ++i) sc[i][tt] = mfma(kf[kk], col.qf[i][x][kk], sc[i][tt]);
        };
#pragma unroll
        for (int tt = 0; tt < 4; ++tt) {
            u32x4 kf[kSteps];
            fetch(pages, tt, kf);
            scores(kf, tt);
        }
        largest<kTiles>(sc, top);
        __syncthreads();
        for (bool more = true; more;) {
            u32x4* const page = pages + bit * kFrags * 64;
            u32x4* const other = pages + (bit ^ 1) * kFrags * 64;
            raise_reference<D, kTiles>(top, scale, acc, [&] { s_fit[wave] = 0; });
            u32x4 w[2][kTiles][kParts], kf[2][kSteps];
            float base[kTiles];
#pragma unroll
            for (int i = 0; i < kTiles; ++i) base[i] = acc.m[i] == -INFINITY ? 0.f : acc.m[i];
            fetch(other, 0, kf[0]);
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                if (tt > 0) fetch(other, tt, kf[tt % 2]);
#pragma unroll
                for (int i = 0; i < kTiles; ++i) {
                    float pv[4];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        pv[x] = __builtin_amdgcn_exp2f(fmaf(sc[i][tt][x], scale, -base[i]));
                        acc.l[i] += pv[x];
                    }
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        if constexpr (kHalf) {
                            w[tt / 2][i][0][2 * (tt % 2) + y] = pack2h(pv[2 * y], pv[2 * y + 1]);
                        } else {
                            uint32_t of[kParts];
                            split2<kParts>(pv[2 * y], pv[2 * y + 1], of);
#pragma unroll
                            for (int x = 0; x < kParts; ++x) w[tt / 2][i][x][2 * (tt % 2) + y] = of[x];
                        }
                    }
                }
                // the next page's scores take the registers of those that have just become weights
                if (tt > 0) scores(kf[(tt + 1) % 2], tt - 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            u32x4 vf[2][2];
            const auto fetch_values = [&](int i, u32x4 (&f)[2]) {
                f[0] = page[(4 * kSteps + 2 * i) * 64 + lane];
                f[1] = page[(4 * kSteps + 2 * i + 1) * 64 + lane];
            };
            fetch_values(0, vf[0]);
            scores(kf[1], 3);
            range.add(vs);
            __builtin_amdgcn_sched_barrier(0);
            each(std::make_integer_sequence<int, 2 * kSteps>(), [&](auto at) {
                constexpr int i = decltype(at)::value, u = i / kSteps, j = i % kSteps;
                if constexpr (i + 1 < 2 * kSteps) fetch_values(i + 1, vf[(i + 1) % 2]);
#pragma unroll
                for (int x = 0; x < kParts; ++x)
#pragma unroll
                    for (int y = 0; y < 2; ++y)
#pragma unroll
                        for (int t = 0; t < kTiles; ++t) {
                            f32x4& o = acc.o[t][2 * j + y];
                            o = kHalf ? mfma_f16(vf[i % 2][y], w[u][t][x], o) : mfma(vf[i % 2][y], w[u][t][x], o);
                        }
                // a share of the decoding: keys first
                if constexpr (i < kSteps)
                    rk.store(page, wave, lane, i);
                else if constexpr ((i - kSteps) % 2 == 0 || kSteps == 2)
                    if constexpr ((i - kSteps) / (kSteps / 2) < RawValues<D>::kPairs)
                        rv.template store<kHalf, (i - kSteps) / (kSteps / 2)>(vs, other, wave, lane);
                __builtin_amdgcn_sched_barrier(0);
            });
            largest<kTiles>(sc, top);
            more = n1 >= 0;
            const int n3 = pop();
            rk.load(part(n3), wave, m, g);
            rv.load(part(n2), wave, m, g);
#pragma unroll
            for (int t = 0; t < 4; ++t) vs[t] = vs_after[t];
            load_value_scales<D>(part(n3), m, g, vs_after);
            if (n2 < 0)
#pragma unroll
                for (int t = 0; t < 4; ++t) vs[t] = 0x7f7f7f7fu;
            n1 = n2;
            n2 = n3;
            bit ^= 1;
            __syncthreads();
        }
        if constexpr (kHalf) {
            if (__builtin_expect(!range.fits(), 0)) {
                // Zeros, perhaps: the pages' values once more, each wavefront a share of them (16 questions of 128 tokens after
                // 16K, a row of zeros in every page or every 64th: 573 and 565 us, by few columns 1,476 and 1,321, without such
                // rows 540; looked for page by page in the loop, that takes 561 without any).
                const uint64_t pages_here = __builtin_amdgcn_ballot_w64(pool.has(id));
                const int rank = __popcll(pages_here & ((uint64_t(1) << lane) - 1));
                for (uint64_t mine = __builtin_amdgcn_ballot_w64(pool.has(id) && rank % kWaves == wave); mine; mine &= mine - 1) {
                    Values<D> v;
                    load_values<D, 0>(part(static_cast<int>(__builtin_ctzll(mine))), m, g, v);
                    if (!zeros_fit<D>(v)) s_fit[wave] = 0;
                }
                range = ScaleRange();
                __syncthreads();
            }
            // (written again behind the next pages' first barrier at the earliest)
            int fit = 1;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) fit &= s_fit[w];
            if (!__builtin_amdgcn_readfirstlane(fit)) return false;
        }
    }
    // columns of no token saw the pages too
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
        if (col.pos[i] < 0) {
            acc.m[i] = -INFINITY;
            acc.l[i] = 0.f;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc.o[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    const int64_t rows = static_cast<int64_t>(tok.n_tokens) * heads;
    put_columns<T, D, kTiles>(a, static_cast<T*>(nullptr), acc, c0, columns, m, g, [&](int c, bool& whole) {
        whole = false;
        return split * rows + static_cast<int64_t>(at_slot + c / a.ratio) * heads + h * a.ratio + c % a.ratio;
    });
    return true;
}

// A unit of own pages, sequence by sequence.
template <typename T, int D, bool kAlone>
__device__ __forceinline__ void attend_own(const PoolView& pool, const TokensView& tok, const PrefixView& px,
                                           const SharedArgs& a, const T* __restrict__ q, int64_t q_stride, T* __restrict__ out,
                                           float* smem, int h, int unit, int split) {
    const int lane = threadIdx.x & 63;
    const int from = unit * a.slots[1], n = min(a.slots[1], tok.n_tokens - from);
    // a lane a slot: where a run of slots of one sequence and group begins
    const int t = px.token(from + min(lane, n - 1), tok.n_tokens), seq = t < 0 ? -1 : tok.seq[t];
    const SlotGroup in = slot_groups(px, tok, from, n);
    const int group = t < 0 ? -2 : in.g;  // no token: a run of its own
    const int seq_before = __shfl_up(seq, 1), group_before = __shfl_up(group, 1);
    const bool begins = lane == 0 || group == -2 || seq != seq_before || group != group_before;
    uint64_t left = __builtin_amdgcn_ballot_w64(lane < n && begins);
    while (left) {
        const int i = static_cast<int>(__builtin_ctzll(left));
        left &= left - 1;
        const int end = left ? static_cast<int>(__builtin_ctzll(left)) : n;
        attend_slots<T, D, true, kAlone>(pool, tok, px, a, q, q_stride, out, smem, h, from + i, end - i,
                                         __builtin_amdgcn_readlane(in.shared, i), split);
        if constexpr (!kAlone) __syncthreads();  // LDS is the next sequence's
    }
}

// Own pages and groups' pages in one launch; a unit's runs stand in the outer order.  Whose blocks stand first is a matter of
// which take longer: the tokens' own where the groups' are as short (12 groups of few columns: 24 us the other way round, 21
// so), the groups' where they are the long ones (16 questions: 559 and 552; drafts 27.6 and 25.9).
// kTiles 0: groups of few columns.
template <typename T, int D, int kTiles>
__global__ __launch_bounds__(kThreads, (D == 64 && kTiles == 0 ? 3 : 2)) void attend_shared_kernel(
    PoolView pool, TokensView tok, PrefixView px, SharedArgs a, const T* __restrict__ q, int64_t q_stride, T* __restrict__ out) {
    extern __shared__ __align__(16) float smem[];
    uint32_t block = linear_block<kThreads>();
    const uint32_t of_own = static_cast<uint32_t>(a.units[1]) * pool.n_kv;
    const uint32_t n_own = a.alone ? (of_own + kWaves - 1) / kWaves : of_own * a.most[1];
    const uint32_t of_group = static_cast<uint32_t>(a.units[0]) * pool.n_kv, n_group = of_group * a.most[0];
    constexpr bool kOwnFirst = kTiles == 0;
    const bool own = kOwnFirst ? block < n_own : block >= n_group;
    if (own != kOwnFirst) block -= kOwnFirst ? n_own : n_group;
    if (block >= (own ? n_own : n_group)) return;
    if (own) {
        if (a.alone) {
            // (one run a unit)
            const uint32_t item = block * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            if (item >= of_own) return;
            const TokenHead where = token_head(item, pool.n_kv);
            attend_own<T, D, true>(pool, tok, px, a, q, q_stride, out, smem, where.h, where.t, 0);
        } else {
            const TokenHead where = token_head(block % of_own, pool.n_kv);
            attend_own<T, D, false>(pool, tok, px, a, q, q_stride, out, smem, where.h, where.t,
                                    static_cast<int>(block / of_own));
        }
        return;
    }
    const int split = static_cast<int>(block / of_group);
    const TokenHead where = token_head(block % of_group, pool.n_kv);
    const GroupUnit u = group_unit(px, tok, a.slots[0], where.t);
    if (u.g < 0 || split >= runs_of(u.shared, a.run[0], a.most[0])) return;
    if constexpr (kTiles == 0) {
        attend_slots<T, D, false, false>(pool, tok, px, a, q, q_stride, out, smem, where.h, u.a, u.b - u.a, u.shared, split);
    } else if (!attend_wide<T, D, kTiles>(pool, tok, px, a, q, q_stride, smem, where.h, u.a, u.b - u.a, u.shared, split)) {
        // 16 columns at a time
        const int slots = 16 / a.ratio;
        for (int at = u.a; at < u.b; at += slots) {
            __syncthreads();  // LDS is the next columns'
            attend_slots<T, D, false, false>(pool, tok, px, a, q, q_stride, out, smem, where.h, at, min(slots, u.b - at),
                                             u.shared, split);
        }
    }
}

// Joins the partial results of a slot's query head, in a fixed order.  Its D / 4 columns of four dimensions are a thread
// each; kTeams of them take parts in turns.
template <typename T, int D, int kTeams>
__global__ __launch_bounds__(256) void join_shared_kernel(int n_tokens, int heads, PrefixView px, SharedArgs a,
                                                          T* __restrict__ out) {
    constexpr int kCols = D / 4, kRows = 256 / kCols / kTeams;
    __shared__ float4 s_o[kTeams][kRows][kCols];
    __shared__ float s_l[kTeams][kRows], s_m[kTeams][kRows];
    const int col = threadIdx.x % kCols, sub = threadIdx.x / kCols % kRows, team = threadIdx.x / kCols / kRows;
    const int64_t row = static_cast<int64_t>(linear_block<256>()) * kRows + sub, rows = static_cast<int64_t>(n_tokens) * heads;
    const bool real = row < rows;
    const int slot = real ? static_cast<int>(row / heads) : 0, head = static_cast<int>(row % heads);
    const int t = real ? px.token(slot, n_tokens) : -1;
    const int of_group = a.counts[2 * slot], of_own = a.counts[2 * slot + 1];
    // (the result of a single run of own pages is there)
    const int parts = t < 0 || (of_group == 0 && of_own <= 1) ? 0 : of_group + of_own;
    float m = -INFINITY, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int w0 = team; w0 < parts; w0 += 4 * kTeams) {
        float2 ml[4];
        float4 x[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const int w = min(w0 + y * kTeams, parts - 1);
            const int64_t at = (w < of_group ? w : a.most[0] + w - of_group) * rows + row;
            ml[y] = reinterpret_cast<const float2*>(a.part_ml)[at];
            x[y] = reinterpret_cast<const float4*>(a.part)[at * kCols + col];
        }
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            if (w0 + y * kTeams >= parts) break;
            const float top = fmaxf(m, ml[y].x), ref = top == -INFINITY ? 0.f : top;
            const float f = part_weight(m, ref), e = part_weight(ml[y].x, ref);
            m = top;
            l = l * f + ml[y].y * e;
            o = make_float4(o.x * f, o.y * f, o.z * f, o.w * f);
            add_scaled(o, e, x[y]);
        }
    }
    if constexpr (kTeams > 1) {
        s_o[team][sub][col] = o;
        if (col == 0) {
            s_m[team][sub] = m;
            s_l[team][sub] = l;
        }
        __syncthreads();
        if (team > 0) return;
        m = s_m[0][sub];
#pragma unroll
        for (int w = 1; w < kTeams; ++w) m = fmaxf(m, s_m[w][sub]);
        const float ref = m == -INFINITY ? 0.f : m;
        o = make_float4(0.f, 0.f, 0.f, 0.f);
        l = 0.f;
#pragma unroll
        for (int w = 0; w < kTeams; ++w) {
            const float f = part_weight(s_m[w][sub], ref);
            l += f * s_l[w][sub];
            add_scaled(o, f, s_o[w][sub][col]);
        }
    }
    if (parts == 0) return;
    put4<T, D>(a, out, true, static_cast<int64_t>(t) * heads + head, 4 * col, o, m, l);
}

// How a call is cut: slots of a unit, pages of a run and runs of a unit at most, units; [0] the groups'
// pages, [1] the tokens' own.
struct Cut {
    int tiles;  // of a wavefront of a group's unit; 0: the unit is one tile, for few columns
    int slots[2], run[2], most[2], units[2];
    bool alone;
    int64_t part, part_ml, bytes;  // the workspace, in bytes from its start
};

int64_t pad16(int64_t n) { return (n + 15) / 16 * 16; }

// Tiles of a wavefront of a group's unit; 0: a tile a workgroup, which needs a shorter start and finds more workgroups to run
// beside it.  Several where a group has the columns (on average) and all tiles have pages to multiply for some 70 us: us with
// one tile and with several, 32/4 heads d128 bf16: 32K tile pages (64 samples of 256 pages) 50 and 62, 65K 66 and 67, 131K 123
// and 102, 524K 406 and 289 (16 questions of 128 tokens after 256: 808 and 535); 8/8 heads d64 bf16, 32K 44 and 49, 131K 114
// and 81; 16/4 d64 fp32, 65K 84 and 85, 262K 290 and 188; 16/4 d128 fp32, 32K 58 and 61, 131K 177 and 171.  Groups of 32 and
// 64 columns, 32K tile pages: 26 and 31, 33 and 41.
int tiles_of(const hga_plan& plan, int n_tokens, int n_groups, int shared_pages) {
    const int64_t columns = static_cast<int64_t>(n_tokens) * (plan.p.n_q_heads / plan.p.n_kv_heads);
    if (columns <= 64 * static_cast<int64_t>(n_groups) || columns / 16 * plan.p.n_kv_heads * shared_pages < 3 << 15) return 0;
    return plan.p.dtype == HGA_F32 && plan.p.head_dim == 128 ? 1 : 2;
}
// Slots of a tile of one sequence.
int own_slots(const hga_plan& plan, int n_tokens, int n_seqs) {
    const int64_t per_seq = (static_cast<int64_t>(n_tokens) + n_seqs - 1) / std::max(n_seqs, 1);
    return static_cast<int>(std::clamp<int64_t>(per_seq, 1, 16 / (plan.p.n_q_heads / plan.p.n_kv_heads)));
}

Cut cut_call(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups, int shared_hint, int own_hint,
             int64_t ws_bytes) {
    const int ratio = plan.p.n_q_heads / plan.p.n_kv_heads, kv = plan.p.n_kv_heads;
    const int64_t rows = static_cast<int64_t>(n_tokens) * plan.p.n_q_heads;
    const int64_t pages[2] = {std::clamp(shared_hint, 1, std::max(max_pages, 1)), std::clamp(own_hint, 1, std::max(max_pages, 1))};
    const int64_t cus = plan.n_cu;
    const auto up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    Cut c{};
    c.tiles = tiles_of(plan, n_tokens, n_groups, static_cast<int>(pages[0]));
    c.slots[0] = 16 * (c.tiles ? c.tiles * kWaves : 1) / ratio;
    c.slots[1] = own_slots(plan, n_tokens, n_seqs);
    // a group's last unit may be a small one
    c.units[0] = n_groups ? static_cast<int>(std::min<int64_t>(n_tokens, n_tokens / c.slots[0] + static_cast<int64_t>(n_groups))) : 0;
    c.units[1] = static_cast<int>(up(n_tokens, c.slots[1]));
    for (int i = 0; i < 2; ++i) {
        const int64_t units = kv * (i ? c.units[1] : std::max(up(n_tokens, c.slots[0]), static_cast<int64_t>(n_groups)));
        c.run[i] = static_cast<int>(pages[i]);
        c.most[i] = 1;
        if (c.units[i] == 0 || units >= 2 * cus) continue;
        const int64_t run = std::max<int64_t>(i ? 16 : 8, up(units * pages[i], 2 * cus));
        c.most[i] = static_cast<int>(up(pages[i], run));
        c.run[i] = static_cast<int>(up(pages[i], c.most[i]));
    }
    // Own pages by a wavefront or a workgroup: what a round of workgroups takes, in pages, about five of them for what comes
    // before the first (256 tokens of 8 heads d64 with 20 own pages: 59 us a call by wavefronts, 73 by workgroups; 64 sequences
    // of four tokens and 8 pages, 4 heads: 45 and 40).
    const int64_t own = static_cast<int64_t>(c.units[1]) * kv;
    c.alone = c.most[1] == 1 && up(own, 2 * kWaves * cus) * (5 + pages[1]) <= up(own, 2 * cus) * (5 + up(pages[1], kWaves));
    const int64_t counts = pad16(static_cast<int64_t>(n_tokens) * 8);
    // fewer runs where the workspace holds no more
    const int64_t run_bytes = rows * (plan.p.head_dim + 2) * 4;
    const int64_t room = ws_bytes < counts ? 0 : (ws_bytes - counts) / run_bytes;
    while (c.most[0] + c.most[1] > room && (c.most[0] > 1 || c.most[1] > 1)) {
        const int i = c.most[0] >= c.most[1] ? 0 : 1;
        c.run[i] = static_cast<int>(up(pages[i], --c.most[i]));
    }
    c.part = counts;
    c.part_ml = c.part + (c.most[0] + c.most[1]) * rows * plan.p.head_dim * 4;
    c.bytes = c.part_ml + (c.most[0] + c.most[1]) * rows * 8;
    return c;
}

template <typename T, int D, int kTiles>
hipError_t run(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const PrefixView& px, const SharedArgs& a,
               const void* q, int64_t q_stride, void* out, hipStream_t stream) {
    constexpr size_t kJoin = sizeof(float) * kWaves * 16 * (D + 4 + 2);
    constexpr size_t kPages = kTiles ? 2 * (D / 4) * 1024 + 3 * kWaves * 4 : 0;
    constexpr size_t lds = std::max(kJoin, kPages);
    const auto kernel = attend_shared_kernel<T, D, kTiles>;
    hipError_t e;
    if constexpr (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        e = once_per_device(done, plan.device, [=] {
            return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize,
                                       static_cast<int>(lds));
        });
        if (e != hipSuccess) return e;
    }
    const int64_t own = static_cast<int64_t>(pool.n_kv) * a.units[1];
    const int64_t n = static_cast<int64_t>(pool.n_kv) * a.units[0] * a.most[0] +
                      (a.alone ? (own + kWaves - 1) / kWaves : own * a.most[1]);
    kernel<<<grid_of(n, kThreads), kThreads, lds, stream>>>(pool, tok, px, a, static_cast<const T*>(q), q_stride,
                                                            static_cast<T*>(out));
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int heads = pool.n_kv * a.ratio;
    const int64_t rows = static_cast<int64_t>(tok.n_tokens) * heads;
    constexpr int kRows = 256 / (D / 4);
    if (a.most[0] + a.most[1] <= 4)
        join_shared_kernel<T, D, 1><<<grid_of((rows + kRows - 1) / kRows, 256), 256, 0, stream>>>(tok.n_tokens, heads, px, a,
                                                                                                  static_cast<T*>(out));
    else
        join_shared_kernel<T, D, kRows><<<grid_of(rows, 256), 256, 0, stream>>>(tok.n_tokens, heads, px, a, static_cast<T*>(out));
    return hipGetLastError();
}

}  // namespace

int64_t attend_shared_bytes(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups, int shared_hint,
                            int own_hint, bool must) {
    if (n_tokens == 0) return 0;
    return cut_call(plan, n_tokens, n_seqs, max_pages, n_groups, shared_hint, own_hint, must ? 0 : INT64_MAX).bytes;
}

// Whether reading shared pages once is worth a second kernel: by the pages that tiles of single sequences would multiply, each
// as much as prefixes of up to 128 pages are long.  Measured over 1 and 8 groups of 2 to 128 sequences after 8 to 384 pages
// (32/4 heads d128 and 8/8 d64 bf16, 16/4 d128 and 8/4 d64 fp32; 1 and 4 tokens each), us shared and not: 512 tile pages of
// prefixes of 8 pages 8.9 and 6.1, 4,096 of 8 19.0 and 13.0, 2,048 of 32 12.1 and 11.5, 4,096 of 32 13.8 and 15.5, 16,384 of 8
// 14.2 and 22.3, 4,096 of 128 14.2 and 16.4, 16,384 of 128 22.6 and 29.8, 65,536 of 32 20.4 and 51.3.  Own pages are not in the
// rule, though what they take grows with the tokens: above the border drafts of four after 32 pages take longer shared, 8
// groups of 32 sequences 94.7 and 82.1 (32/4 heads d128 bf16; one token each 30.7 and 41.1, after 128 pages 164 and 221), 67.8
// and 62.9 (16/4 d128 fp32), one group of 128 41.5 and 34.4.
bool attend_shared_pays(const hga_plan& plan, int n_tokens, int n_seqs, int max_pages, int n_groups, int shared_hint) {
    if (n_groups == 0 || std::min(n_seqs, n_tokens) < 2 * static_cast<int64_t>(n_groups)) return false;
    const int64_t tiles = (static_cast<int64_t>(n_tokens) + own_slots(plan, n_tokens, n_seqs) - 1) / own_slots(plan, n_tokens, n_seqs);
    const int64_t pages = std::min(shared_hint, max_pages);
    const int64_t least = 1 << 17;
    return tiles * plan.p.n_kv_heads * pages * std::min<int64_t>(pages, 128) >= least;
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
    a.alone = c.alone;
    a.lse = lse;
    char* w = static_cast<char*>(ws);
    a.counts = reinterpret_cast<int32_t*>(w);
    a.part = reinterpret_cast<float*>(w + c.part);
    a.part_ml = reinterpret_cast<float*>(w + c.part_ml);
    const auto go = [&](auto zero, auto dim) {
        using T = decltype(zero);
        constexpr int D = decltype(dim)::value, kMost = sizeof(T) == 4 && D == 128 ? 1 : 2;
        const auto f = c.tiles ? run<T, D, kMost> : run<T, D, 0>;
        return f(plan, pool, tok, px, a, q, q_stride, out, stream);
    };
    const bool f32 = plan.p.dtype == HGA_F32;
    if (plan.p.head_dim == 128)
        return f32 ? go(0.f, std::integral_constant<int, 128>()) : go(bf16_t(0), std::integral_constant<int, 128>());
    return f32 ? go(0.f, std::integral_constant<int, 64>()) : go(bf16_t(0), std::integral_constant<int, 64>());
}

}  // namespace hga

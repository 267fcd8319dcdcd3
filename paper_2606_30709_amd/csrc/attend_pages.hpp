// Building blocks of attention over the paged 4-bit cache: a wavefront's steps over one page, shared by the kernels that
// attend single tokens and batches with shared prefixes.  Columns of a tile are query heads; the operands' layout is that
// of a page (tokens.hpp).
#pragma once

#include "hga_device.hpp"
#include "tokens.hpp"

namespace hga {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0,
                                                   0);
}

// Two floats as a pair of bf16, rounded to nearest even.
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
}

// kTerms words whose bf16 pairs add up to (a, b): the rounded values, then what rounding left.  The first of three terms is
// cut off instead, which leaves no more than the other two hold: rounded, the largest floats would become infinite.
template <int kTerms>
__device__ __forceinline__ void split2(float a, float b, uint32_t (&w)[kTerms]) {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) {
        w[i] = kTerms == 3 && i == 0 ? __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u)
                                     : pack2(a, b);
        if (i + 1 == kTerms) break;
        a -= __uint_as_float(w[i] << 16);
        b -= __uint_as_float(w[i] & 0xffff0000u);
    }
}

// The term of a value that column m holds in the spread form: bits 0-7, 8-15 and 16-23 of the significand, counted from the
// top, each exact in bf16; the fourth column of a head holds zeros.
struct TermMask {
    uint32_t hi, lo;
};
__device__ __forceinline__ TermMask term_mask(int m) {
    const uint32_t cut[4] = {0u, 0xffff0000u, 0xffffff00u, 0xffffffffu};
    const int x = m & 3;
    return TermMask{x == 0 ? cut[1] : x == 1 ? cut[2] : cut[3], x == 0 ? cut[0] : x == 1 ? cut[1] : x == 2 ? cut[2] : cut[3]};
}
__device__ __forceinline__ float term_of(float x, const TermMask& k) {
    return __uint_as_float(__float_as_uint(x) & k.hi) - __uint_as_float(__float_as_uint(x) & k.lo);
}
// Sum over a head's four columns (the lanes of a quad).
__device__ __forceinline__ float quad_sum(float x) {
    x += __uint_as_float(static_cast<uint32_t>(
        __builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(x)), 0xB1, 0xf, 0xf, true)));
    return x + __uint_as_float(static_cast<uint32_t>(
                   __builtin_amdgcn_mov_dpp(static_cast<int>(__float_as_uint(x)), 0x4E, 0xf, 0xf, true)));
}

// A lane's share of a page's keys and of its values.
template <int D>
struct Keys {
    uint32_t c[4][D / 32];
    uint32_t s;
};
template <int D>
struct Values {
    uint32_t c[4][D / 32];
    uint32_t s[4];
};

// One head's part of a page as a buffer: no address arithmetic per lane but a fixed offset, and an empty buffer's loads
// touch no memory, so that the loop below needs no branch around its last loads.
// Codes are loaded past the caches (kNt): histories of a decode step are read once (400 of 32 pages: 91 us cached, 83 so;
// 64 of 31 listed pages 17.9 and 16.6; 32 of 128 pages on average 61 either way), and prompts, whose units share pages, take
// the same time either way.
constexpr int kNt = 2;
template <int D, int kAux = kNt>
__device__ __forceinline__ void load_codes(buf_rsrc r, uint32_t offset, uint32_t (&w)[D / 32]) {
    if constexpr (D == 128) {
        const vec16 x = __builtin_bit_cast(vec16, __builtin_amdgcn_raw_buffer_load_b128(r, offset, 0, kAux));
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x.w[i];
    } else {
        const uint2 x = __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(r, offset, 0, kAux));
        w[0] = x.x;
        w[1] = x.y;
    }
}
template <int D, int kAux = kNt>
__device__ __forceinline__ void load_keys(buf_rsrc r, int m, int g, Keys<D>& k) {
    using F = PageFormat<D>;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_codes<D, kAux>(r, F::key_code(m, g * (D / 4)) + t * F::key_code(16, 0), k.c[t]);
    k.s = static_cast<uint32_t>(buf_load_i32(r, F::key_scale(m, g * (D / 4) / 32)));
}
template <int D, int kAux = kNt>
__device__ __forceinline__ void load_values(buf_rsrc r, int m, int g, Values<D>& v) {
    using F = PageFormat<D>;
#pragma unroll
    for (int t = 0; t < 4; ++t)
        load_codes<D, kAux>(r, F::value_code(4 * g, m * F::kLaneDims) + t * (F::value_code(16, 0) - F::kCodes), v.c[t]);
    const vec16 x = buf_load16(r, F::value_scale(4 * g, m * F::kLaneDims / 32));
#pragma unroll
    for (int t = 0; t < 4; ++t) v.s[t] = x.w[t];
}

// The maximum (sum) of the four lanes that share a column, in all of them.
__device__ __forceinline__ float max_groups(float x) {
    const uint32_t u = __float_as_uint(x);
    const auto a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    x = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const uint32_t v = __float_as_uint(x);
    const auto b = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float sum_groups(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A reference below the maximum by this (log2) stays: weights reach 2^kSlack, exact in fp32 and within bf16's range.
constexpr float kSlack = 8.0f;

// What a wavefront holds of its columns.
template <int D, int kTiles>
struct Acc {
    f32x4 o[kTiles][D / 16];
    float m[kTiles], l[kTiles];
};

// A page's scores.
template <int D, int kTerms, int kTiles>
__device__ __forceinline__ void page_scores(const Keys<D>& k, const u32x4 (&qf)[kTiles][kTerms][D / 32],
                                            f32x4 (&sc)[kTiles][4]) {
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
        const float ks = scale_of(k.s >> (8 * tt) & 255u);
#pragma unroll
        for (int i = 0; i < kTiles; ++i) sc[i][tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            const uint32_t c = k.c[tt][kk];
            const u32x4 kf = {decode2<0>(c, ks), decode2<1>(c, ks), decode2<2>(c, ks), decode2<3>(c, ks)};
#pragma unroll
            for (int i = 0; i < kTiles; ++i)
#pragma unroll
                for (int x = 0; x < kTerms; ++x) sc[i][tt] = mfma(kf, qf[i][x][kk], sc[i][tt]);
        }
    }
}

// The running reference of every column, raised where a page's scores exceed it by more than the slack.
template <int D, int kTiles>
__device__ __forceinline__ void page_reference(const f32x4 (&sc)[kTiles][4], float scale, Acc<D, kTiles>& acc) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i) {
        float top = sc[i][0][0];
#pragma unroll
        for (int tt = 0; tt < 4; ++tt)
#pragma unroll
            for (int x = 0; x < 4; ++x) top = fmaxf(top, sc[i][tt][x]);
        top = max_groups(top) * scale;
        const bool grow = top > acc.m[i] + kSlack;
        if (__builtin_amdgcn_ballot_w64(grow)) {
            const float alpha = grow ? __builtin_amdgcn_exp2f(acc.m[i] - top) : 1.f;
            if (grow) acc.m[i] = top;
            acc.l[i] *= alpha;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc.o[i][j] *= alpha;
        }
    }
}

// The weights of half a page (32 keys, tiles 2 u and 2 u + 1) under the reference, four keys of a tile as two words.
template <int D, int kParts, int kTiles>
__device__ __forceinline__ void half_weights(int u, const f32x4 (&sc)[kTiles][4], float scale, Acc<D, kTiles>& acc,
                                             u32x4 (&w)[kTiles][kParts], const TermMask* mask) {
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
            if (mask) {
#pragma unroll
                for (int x = 0; x < 4; ++x) pv[x] = term_of(pv[x], *mask);
                // exact in bf16: the high halves
                w[i][0][2 * b] = __builtin_amdgcn_perm(__float_as_uint(pv[1]), __float_as_uint(pv[0]), 0x07060302u);
                w[i][0][2 * b + 1] = __builtin_amdgcn_perm(__float_as_uint(pv[3]), __float_as_uint(pv[2]), 0x07060302u);
            } else {
                uint32_t lo[kParts], hi[kParts];
                split2<kParts>(pv[0], pv[1], lo);
                split2<kParts>(pv[2], pv[3], hi);
#pragma unroll
                for (int x = 0; x < kParts; ++x) {
                    w[i][x][2 * b] = lo[x];
                    w[i][x][2 * b + 1] = hi[x];
                }
            }
        }
    }
}

// Its weighted values: the rows of a quad decoded two dimensions at a time, then paired by row.
template <int D, int kParts, int kTiles>
__device__ __forceinline__ void half_values(int u, const Values<D>& v, const u32x4 (&w)[kTiles][kParts],
                                            Acc<D, kTiles>& acc) {
    constexpr int DL = D / 16;
    uint32_t vf[DL][4];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int tt = 2 * u + b;
#pragma unroll
        for (int r2 = 0; r2 < 2; ++r2) {
            uint32_t lo[DL / 2], hi[DL / 2];
            const float s0 = scale_of(v.s[tt] >> (16 * r2) & 255u);
            const float s1 = scale_of(v.s[tt] >> (16 * r2 + 8) & 255u);
            if constexpr (DL == 8) {
                const uint32_t c0 = v.c[tt][2 * r2], c1 = v.c[tt][2 * r2 + 1];
                lo[0] = decode2<0>(c0, s0);
                lo[1] = decode2<1>(c0, s0);
                lo[2] = decode2<2>(c0, s0);
                lo[3] = decode2<3>(c0, s0);
                hi[0] = decode2<0>(c1, s1);
                hi[1] = decode2<1>(c1, s1);
                hi[2] = decode2<2>(c1, s1);
                hi[3] = decode2<3>(c1, s1);
            } else {
                const uint32_t c = v.c[tt][r2];
                lo[0] = decode2<0>(c, s0);
                lo[1] = decode2<1>(c, s0);
                hi[0] = decode2<2>(c, s1);
                hi[1] = decode2<3>(c, s1);
            }
#pragma unroll
            for (int j = 0; j < DL / 2; ++j) {
                vf[2 * j][2 * b + r2] = __builtin_amdgcn_perm(hi[j], lo[j], 0x05040100u);
                vf[2 * j + 1][2 * b + r2] = __builtin_amdgcn_perm(hi[j], lo[j], 0x07060302u);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int x = 0; x < kParts; ++x)
#pragma unroll
            for (int j = 0; j < DL; ++j)
                acc.o[i][j] = mfma(u32x4{vf[j][0], vf[j][1], vf[j][2], vf[j][3]}, w[i][x], acc.o[i][j]);
}

// Bit 7 of each byte that is 255.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & w & 0x80808080u; }

// Value blocks of a page that stand for NaN, where some columns see a row and others do not: 0 * NaN would reach those too.
// They count as some number from here on, and the columns that see them are to become NaN (the block's dimensions): column
// 16 i + m sees the page's rows up to seen[i]; bit i of the result: it does, in the lane's dimensions (a block's:
// (4 g + x) DL + j, x < 4, j < DL).
template <int D, int kTiles>
__device__ __forceinline__ uint32_t nan_reached(Values<D>& v, int m, int g, const int (&seen)[kTiles]) {
    constexpr int DL = D / 16;
    uint32_t any = 0;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) any |= nan_bytes(v.s[tt]);
    if (!__builtin_amdgcn_ballot_w64(any != 0)) return 0;
    uint32_t reached = 0;
#pragma unroll
    for (int tt = 0; tt < 4; ++tt) {
        const uint32_t is = nan_bytes(v.s[tt]);
        for (int x = 0; x < 4; ++x) {
            // one lane for a block's: those of its first dimensions
            uint64_t lanes = __builtin_amdgcn_ballot_w64((is >> (8 * x) & 0x80u) != 0 && m * DL % 32 == 0);
            for (; lanes; lanes &= lanes - 1) {
                const int at = static_cast<int>(__builtin_ctzll(lanes)), row = 16 * tt + 4 * (at >> 4) + x;
                if ((at & 15) * DL / 32 != 4 * g * DL / 32) continue;
#pragma unroll
                for (int i = 0; i < kTiles; ++i) reached |= row <= seen[i] ? 1u << i : 0u;
            }
        }
        v.s[tt] ^= is;  // 127, a scale of 1
    }
    return reached;
}
template <int D, int kTiles>
__device__ __forceinline__ void set_nan(uint32_t reached, Acc<D, kTiles>& acc) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
        if (reached >> i & 1)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) acc.o[i][j] = f32x4{NAN, NAN, NAN, NAN};
}
template <int D, int kTiles>
__device__ __forceinline__ void take_out_nan(Values<D>& v, int m, int g, const int (&seen)[kTiles], Acc<D, kTiles>& acc) {
    set_nan<D, kTiles>(nan_reached<D, kTiles>(v, m, g, seen), acc);
}

// The weight of a partial result with reference m under the reference `base`.  One without a reference has seen nothing
// (zeros) or only what is not a number: that stays.
__device__ __forceinline__ float part_weight(float m, float base) {
    return m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - base);
}
__device__ __forceinline__ float natural_lse(float base, float l) {
    return l == 0.f ? -INFINITY : base * 0.6931471805599453f + logf(l);
}

}  // namespace
}  // namespace hga

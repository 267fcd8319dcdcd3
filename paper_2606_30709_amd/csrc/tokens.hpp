// The paged 4-bit cache: how a page is laid out, and how a batch of tokens finds its pages.
//
// A page holds the keys and values of 64 consecutive positions of one sequence (one chunk) for every KV head.  A row of
// d values is stored as d/32 blocks that each share a power-of-two scale 2^(e - 127) (one byte e; 255 marks a block that
// holds NaN) and 4-bit codes of {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign: the element, block and scale formats of the
// OCP Microscaling specification.  Scale and product are exact in bf16, so attention multiplies what is stored exactly.
//
// One head's part of a page is laid out for the matrix instruction's operands, a wavefront reading each kilobyte with
// one 16-byte load a lane (lane l: m = l % 16, g = l / 16; 16-key tile t of the page):
//   key codes    [64 rows][d/2]: lane (m, g) reads d/8 bytes of row 16 t + m, its quarter of the row, whose dimensions are
//                the reduction indices it owns -- the order of the reduction is free as long as q has the same;
//   value codes  [16 quads][16][4][d/32]: lane (m, g) reads, of rows 16 t + 4 g .. + 3, dimensions m d/16 .. + d/16 - 1;
//   key scales   [16][d/32][4]: row 16 t + m at [m][block][t], one word for a lane's four tiles;
//   value scales [4][d/32][4][4]: row 16 t + 4 g + i at [g][block][t][i], 16 bytes for a lane's sixteen rows.
#pragma once

#include "hga_device.hpp"

namespace hga {

constexpr int kPageRows = 64;
// Most pages of a sequence: as many chunks as the routing takes (16.7 M tokens).
constexpr int kMaxSeqPages = 1 << 18;

template <int D>
struct PageFormat {
    static constexpr int kCodes = kPageRows * D / 2;  // bytes of the keys' (the values') codes
    static constexpr int kBlocks = D / 32;            // scales of a row
    static constexpr int kKeyScales = 2 * kCodes;
    static constexpr int kValueScales = kKeyScales + kPageRows * kBlocks;
    static constexpr int kBytes = kValueScales + kPageRows * kBlocks;
    static constexpr int kLaneDims = D / 16;          // dimensions of a value lane

    // Byte of dimension `dim` (even: the low half of the byte) of a row.
    __host__ __device__ static constexpr int key_code(int row, int dim) {
        return row * (D / 2) + dim / 2;
    }
    __host__ __device__ static constexpr int value_code(int row, int dim) {
        return kCodes + ((row / 4) * 16 + dim / kLaneDims) * (2 * kLaneDims) +
               (row % 4) * (kLaneDims / 2) + dim % kLaneDims / 2;
    }
    __host__ __device__ static constexpr int key_scale(int row, int block) {
        return kKeyScales + ((row % 16) * kBlocks + block) * 4 + row / 16;
    }
    __host__ __device__ static constexpr int value_scale(int row, int block) {
        return kValueScales + (((row / 4 % 4) * kBlocks + block) * 4 + row / 16) * 4 + row % 4;
    }
};

__host__ __device__ constexpr int page_head_bytes(int d) { return kPageRows * (d + d / 16); }

// One layer of a pool.  Page ids below n_hot lie in device memory, those from n_hot to n_hot + n_cold in the cold tier
// (pinned host memory, by its device address); any other id is an absent page.
struct PoolView {
    unsigned char* hot;
    unsigned char* cold;
    float* sum;  // [n_hot + n_cold][n_kv][d]
    int n_hot, n_cold, n_kv;
    int64_t page_bytes;

    __host__ __device__ bool has(int id) const {
        return static_cast<uint32_t>(id) < static_cast<uint32_t>(n_hot) + static_cast<uint32_t>(n_cold);
    }
    __host__ __device__ unsigned char* page(int id) const {
        return id < n_hot ? hot + id * page_bytes : cold + static_cast<int64_t>(id - n_hot) * page_bytes;
    }
};

// A call's tokens: token t is position pos[t] of sequence seq[t], whose chunk c lies in page table[seq[t]][c].
struct TokensView {
    const int32_t* seq;
    const int32_t* pos;
    const int32_t* table;  // [n_seqs][max_pages]
    int n_tokens, n_seqs, max_pages;

    // Whether token t is one (its sequence and position inside the table), and which.
    __host__ __device__ bool at(int t, int& s, int& p) const {
        s = seq[t];
        p = pos[t];
        return static_cast<uint32_t>(s) < static_cast<uint32_t>(n_seqs) && p >= 0 && p / kPageRows < max_pages;
    }
    // The page of chunk c (0 <= c < max_pages) of sequence s, by the table's word.
    __host__ __device__ int page_id(int s, int c) const {
        return table[static_cast<int64_t>(s) * max_pages + c];
    }
};

// Token and head of a call's unit (or item) number, below 2^31: a division of 32-bit words.
struct TokenHead {
    int t, h;
};
__host__ __device__ inline TokenHead token_head(uint32_t unit, int n_kv) {
    const uint32_t t = unit / static_cast<uint32_t>(n_kv);
    return TokenHead{static_cast<int>(t), static_cast<int>(unit - t * static_cast<uint32_t>(n_kv))};
}

// An entry of a token's list of chunks, as a page and how many of its rows the token at position p sees (0: none).
// Entries may hold anything.
struct SeenPage {
    int id, rows;
};
__host__ __device__ inline SeenPage seen_page(const PoolView& pool, const TokensView& tok, int s, int p, int c) {
    SeenPage r{-1, 0};
    const int own = p / kPageRows;
    if (c < 0 || c > own) return r;
    const int id = tok.page_id(s, c);
    if (!pool.has(id)) return r;
    r.id = id;
    r.rows = c < own ? kPageRows : p % kPageRows + 1;
    return r;
}

#if defined(__HIP_DEVICE_COMPILE__) || defined(__HIPCC__)

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

// 2^(e - 127); the conversions below make NaN of e = 255.
__device__ __forceinline__ float scale_of(uint32_t e) { return __uint_as_float(e << 23); }

// The two values of byte kByte of `codes` times a power of two, exact in bf16: low half first.
template <int kByte>
__device__ __forceinline__ uint32_t decode2(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, kByte));
}

// The block's shared exponent byte from the largest magnitude's bits: the smallest 2^s with amax <= 6 * 2^s -- 6 = 1.5 * 4,
// so s is amax's exponent less two, one more above a fraction of 1.5 -- kept where every value is a normal bf16.
__device__ __forceinline__ uint32_t block_scale(uint32_t amax_bits) {
    const uint32_t e = (amax_bits >> 23) + ((amax_bits & 0x7fffffu) > 0x400000u ? 1u : 0u);
    if (amax_bits >= 0x7f800000u) return 255u;  // NaN or infinity in the block
    return e < 4u ? 2u : e - 2u;
}

// Codes of eight values of a block with exponent byte e, rounded to nearest (ties to the even code).
__device__ __forceinline__ uint32_t encode8(const float* x, uint32_t e) {
    if (e == 255u) return 0u;
    const float s = scale_of(e);
    // at the largest scale 4 * 2^126 would pass the largest float: 3 * 2^126 at most
    const float top = e == 253u ? 3.0f * s : __uint_as_float(0x7f7fffffu);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = __builtin_amdgcn_fmed3f(x[i], -top, top);
    uint32_t r = 0;
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[0], y[1], s, 0);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[2], y[3], s, 1);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[4], y[5], s, 2);
    r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, y[6], y[7], s, 3);
    return r;
}

// 16 bytes read or written once: not kept in the caches.
__device__ __forceinline__ vec16 load16_once(const void* p) {
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(vec16, __builtin_nontemporal_load(static_cast<const u32x4_t*>(p)));
}
__device__ __forceinline__ void store16_once(void* p, const vec16& v) {
    typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
    __builtin_nontemporal_store(__builtin_bit_cast(u32x4_t, v), static_cast<u32x4_t*>(p));
}

// Eight consecutive elements of a row, 16-byte loads; _once: of a row read once.
__device__ __forceinline__ void load8(const float* p, float* x) {
    elem<float>::unpack(load16(p), x);
    elem<float>::unpack(load16(p + 4), x + 4);
}
__device__ __forceinline__ void load8(const bf16_t* p, float* x) { elem<bf16_t>::unpack(load16(p), x); }
__device__ __forceinline__ void load8_once(const float* p, float* x) {
    elem<float>::unpack(load16_once(p), x);
    elem<float>::unpack(load16_once(p + 4), x + 4);
}
__device__ __forceinline__ void load8_once(const bf16_t* p, float* x) { elem<bf16_t>::unpack(load16_once(p), x); }

#endif

}  // namespace hga

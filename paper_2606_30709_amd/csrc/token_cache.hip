// The paged 4-bit cache: appending tokens, reading rows back, copying pages.
//
// Append and read move a row of a head with D/8 lanes, eight dimensions each: the four lanes of a 32-dimension block find
// the block's largest magnitude among themselves, and a lane's eight codes are one word of the page.  Both are bound by
// their bytes (a token of 4 heads of d128: 2 KiB of bf16 in, 544 bytes out).
#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr int kThreads = 256;

// Largest of the four lanes of a quad.
__device__ __forceinline__ uint32_t quad_max(uint32_t x) {
    uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0xB1, 0xf, 0xf, true));
    x = o > x ? o : x;
    o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(x), 0x4E, 0xf, 0xf, true));
    return o > x ? o : x;
}

__device__ __forceinline__ uint32_t bits_of(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// The values of four codes of a block with exponent byte e.
__device__ __forceinline__ void decode4(uint32_t codes, uint32_t e, float* x) {
    const uint32_t lo = decode2<0>(codes, scale_of(e)), hi = decode2<1>(codes, scale_of(e));
    x[0] = __uint_as_float(lo << 16);
    x[1] = __uint_as_float(lo & 0xffff0000u);
    x[2] = __uint_as_float(hi << 16);
    x[3] = __uint_as_float(hi & 0xffff0000u);
}

// Stores a lane's eight dimensions of a row of a (token, head): lanes 0 .. D/8 - 1 the keys', the next the values'.
template <typename T, int D>
__device__ __forceinline__ void store_piece(const PoolView& pool, const TokensView& tok, int t, int h, int lane,
                                            const T* __restrict__ k, int64_t k_stride, const T* __restrict__ v,
                                            int64_t v_stride) {
    using F = PageFormat<D>;
    const bool key = lane < D / 8;
    const int dim = lane % (D / 8) * 8;
    float x[8];  // fetched before the page is known
    load8_once((key ? k + t * k_stride : v + t * v_stride) + h * D + dim, x);
    int s, p;
    if (!tok.at(t, s, p)) return;
    const int id = tok.page_id(s, p / kPageRows), row = p % kPageRows;
    if (!pool.has(id)) return;
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, bits_of(x[j]));
    const uint32_t e = block_scale(quad_max(m));
    const uint32_t codes = encode8(x, e);
    unsigned char* head = pool.page(id) + h * F::kBytes;
    if (key) {
        *reinterpret_cast<uint32_t*>(head + F::key_code(row, dim)) = codes;
        if (dim % 32 == 0) head[F::key_scale(row, dim / 32)] = static_cast<unsigned char>(e);
    } else {
        if constexpr (F::kLaneDims == 8) {
            *reinterpret_cast<uint32_t*>(head + F::value_code(row, dim)) = codes;
        } else {
            *reinterpret_cast<uint16_t*>(head + F::value_code(row, dim)) = static_cast<uint16_t>(codes);
            *reinterpret_cast<uint16_t*>(head + F::value_code(row, dim + 4)) = static_cast<uint16_t>(codes >> 16);
        }
        if (dim % 32 == 0) head[F::value_scale(row, dim / 32)] = static_cast<unsigned char>(e);
    }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void append_kernel(PoolView pool, TokensView tok, const T* __restrict__ k,
                                                          int64_t k_stride, const T* __restrict__ v,
                                                          int64_t v_stride) {
    constexpr int kLanes = 2 * D / 8;  // lanes of a (token, head): keys, then values
    const auto [t, h] = token_head(linear_block<kThreads>() * (kThreads / kLanes) + threadIdx.x / kLanes, pool.n_kv);
    if (t < tok.n_tokens) store_piece<T, D>(pool, tok, t, h, threadIdx.x % kLanes, k, k_stride, v, v_stride);
}

// A wavefront forms the summary of a page of one head: the mean over the stored keys turned to the page's middle, as the
// chunk summaries are.  A lane holds four pairs of dimensions of every kAtOnce-th row.
template <int D>
__device__ __forceinline__ void summarise(const unsigned char* head, const float* __restrict__ phase, float* out) {
    using F = PageFormat<D>;
    constexpr int HALF = D / 2;
    constexpr int kRow = HALF / 4;      // lanes of a row
    constexpr int kAtOnce = 64 / kRow;  // rows
    constexpr int kBatch = 4;           // ... times this are fetched at once
    const int lane = threadIdx.x & 63, dim = lane % kRow * 4, slot = lane / kRow;
    float sa[4] = {}, sb[4] = {};
#pragma unroll
    for (int r0 = 0; r0 < kPageRows; r0 += kBatch * kAtOnce) {
        uint32_t ca[kBatch], cb[kBatch], ea[kBatch], eb[kBatch];
        float4 c[kBatch], sn[kBatch];
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            const int row = r0 + y * kAtOnce + slot;
            ca[y] = *reinterpret_cast<const uint16_t*>(head + F::key_code(row, dim));
            cb[y] = *reinterpret_cast<const uint16_t*>(head + F::key_code(row, dim + HALF));
            ea[y] = head[F::key_scale(row, dim / 32)];
            eb[y] = head[F::key_scale(row, (dim + HALF) / 32)];
            c[y] = *reinterpret_cast<const float4*>(phase + row * HALF + dim);
            sn[y] = *reinterpret_cast<const float4*>(phase + (kPageRows + row) * HALF + dim);
        }
#pragma unroll
        for (int y = 0; y < kBatch; ++y) {
            float a[4], b[4];
            decode4(ca[y], ea[y], a);
            decode4(cb[y], eb[y], b);
            const float cy[4] = {c[y].x, c[y].y, c[y].z, c[y].w}, sy[4] = {sn[y].x, sn[y].y, sn[y].z, sn[y].w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                sa[j] += a[j] * cy[j] - b[j] * sy[j];
                sb[j] += a[j] * sy[j] + b[j] * cy[j];
            }
        }
    }
#pragma unroll
    for (int m = kRow; m < 64; m *= 2)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sa[j] += __shfl_xor(sa[j], m);
            sb[j] += __shfl_xor(sb[j], m);
        }
    if (slot == 0) {
        constexpr float f = 1.f / kPageRows;
        *reinterpret_cast<float4*>(out + dim) = make_float4(sa[0] * f, sa[1] * f, sa[2] * f, sa[3] * f);
        *reinterpret_cast<float4*>(out + dim + HALF) = make_float4(sb[0] * f, sb[1] * f, sb[2] * f, sb[3] * f);
    }
}

// Summaries of the pages that the call's tokens fill (those at a page's last row), once all their rows are stored: a
// workgroup looks at 64 tokens of a head (of a prompt one of them, of a decode step few but all of them at times), its
// wavefronts take every kCloseWaves-th page.  Kept apart from the kernel before: with its registers that one, bound by
// memory, had a third of the wavefronts it needs (23 K tokens of 8 heads of d64: 103 us together, 28 and 9 us apart).
constexpr int kCloseWaves = 4;
template <int D, int kOf>
__device__ __forceinline__ void close_pages(const PoolView& pool, const TokensView& tok, int64_t t0, int h,
                                            const float* __restrict__ phase) {
    using F = PageFormat<D>;
    const int64_t t = t0 + (threadIdx.x & 63);
    int s = 0, p = 0, id = -1;
    if (t < tok.n_tokens && tok.at(static_cast<int>(t), s, p) && p % kPageRows == kPageRows - 1)
        id = tok.page_id(s, p / kPageRows);
    int n = 0;
    for (uint64_t left = __builtin_amdgcn_ballot_w64(id >= 0 && pool.has(id)); left; left &= left - 1) {
        if (n++ % kOf != static_cast<int>(threadIdx.x >> 6)) continue;
        const int page = __builtin_amdgcn_readlane(id, static_cast<int>(__builtin_ctzll(left)));
        summarise<D>(pool.page(page) + h * F::kBytes, phase,
                     pool.sum + (static_cast<int64_t>(page) * pool.n_kv + h) * D);
    }
}
template <int D>
__global__ __launch_bounds__(64 * kCloseWaves) void close_kernel(PoolView pool, TokensView tok,
                                                                 const float* __restrict__ phase) {
    const auto [t64, h] = token_head(linear_block<64 * kCloseWaves>(), pool.n_kv);
    close_pages<D, kCloseWaves>(pool, tok, static_cast<int64_t>(t64) * 64, h, phase);
}

// Both in one launch, for calls of at most kFewTokens tokens: a workgroup stores every row of a head, and so knows them
// stored when it looks for the pages they fill.  4 heads of d128, a call in a graph (and on the host): 1 token 4.5 us (6.4)
// against 5.8 (9.1) in two launches, 32 tokens 5.5 against 6.1, 64 tokens 7.0 against 6.2.
constexpr int kFewTokens = 32, kFewWaves = 8;
template <typename T, int D>
__global__ __launch_bounds__(64 * kFewWaves) void append_few_kernel(PoolView pool, TokensView tok,
                                                                    const T* __restrict__ k, int64_t k_stride,
                                                                    const T* __restrict__ v, int64_t v_stride,
                                                                    const float* __restrict__ phase) {
    constexpr int kLanes = 2 * D / 8, kAtOnce = 64 * kFewWaves / kLanes;
    const int h = static_cast<int>(linear_block<64 * kFewWaves>());
    if (h >= pool.n_kv) return;
#pragma unroll 4
    for (int t = threadIdx.x / kLanes; t < tok.n_tokens; t += kAtOnce)
        store_piece<T, D>(pool, tok, t, h, threadIdx.x % kLanes, k, k_stride, v, v_stride);
    __syncthreads();
    for (int t = 0; t < tok.n_tokens; t += 64) close_pages<D, kFewWaves>(pool, tok, t, h, phase);
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void read_kernel(PoolView pool, TokensView tok, T* __restrict__ k,
                                                        T* __restrict__ v) {
    using F = PageFormat<D>;
    constexpr int kLanes = 2 * D / 8;
    const uint32_t item = linear_block<kThreads>() * (kThreads / kLanes) + threadIdx.x / kLanes;
    const auto [t, h] = token_head(item, pool.n_kv);
    if (t >= tok.n_tokens) return;
    const int lane = threadIdx.x % kLanes;
    const bool key = lane < D / 8;
    const int dim = lane % (D / 8) * 8;
    int s, p;
    const bool in = tok.at(t, s, p);
    const int id = in ? tok.page_id(s, p / kPageRows) : -1;
    uint32_t codes = 0;
    uint32_t e = 127;
    if (in && pool.has(id)) {
        const int row = p % kPageRows;
        const unsigned char* head = pool.page(id) + h * F::kBytes;
        if (key) {
            codes = *reinterpret_cast<const uint32_t*>(head + F::key_code(row, dim));
        } else if constexpr (F::kLaneDims == 8) {
            codes = *reinterpret_cast<const uint32_t*>(head + F::value_code(row, dim));
        } else {
            codes = *reinterpret_cast<const uint16_t*>(head + F::value_code(row, dim)) |
                    static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(head + F::value_code(row, dim + 4))) << 16;
        }
        e = head[key ? F::key_scale(row, dim / 32) : F::value_scale(row, dim / 32)];
    }
    const float sc = scale_of(e);
    vec16 b;
    b.w[0] = decode2<0>(codes, sc);
    b.w[1] = decode2<1>(codes, sc);
    b.w[2] = decode2<2>(codes, sc);
    b.w[3] = decode2<3>(codes, sc);
    T* out = (key ? k : v) + static_cast<int64_t>(item) * D + dim;
    if constexpr (sizeof(T) == 2) {
        store16(out, b);
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            vec16 w;
            w.w[0] = b.w[2 * i] << 16;
            w.w[1] = b.w[2 * i] & 0xffff0000u;
            w.w[2] = b.w[2 * i + 1] << 16;
            w.w[3] = b.w[2 * i + 1] & 0xffff0000u;
            store16(out + 4 * i, w);
        }
    }
}

// Copies page src[i] over page dst[i] in every layer, summaries too: a workgroup a page of a layer, kBatch 16-byte loads a
// thread in flight (a page of 4 heads of d128 is 8.5 times what its threads load at once), past the caches (256 pages of 48
// layers: 190 us in equal 16 KiB pieces, 180 a page a workgroup, 164 past the caches).
struct CopyArgs {
    unsigned char *hot, *cold;
    float* sum;
    int n_hot, n_cold, n_layers;
    int64_t page_bytes, sum_bytes;  // of one page in one layer
};

__device__ __forceinline__ void copy_bytes(const unsigned char* from, unsigned char* to, int64_t bytes) {
    constexpr int kBatch = 9, kStep = kThreads * 16;
    for (int64_t b0 = threadIdx.x * 16; b0 < bytes; b0 += kBatch * kStep) {
        vec16 x[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (b0 + j * kStep < bytes) x[j] = load16_once(from + b0 + j * kStep);
#pragma unroll
        for (int j = 0; j < kBatch; ++j)
            if (b0 + j * kStep < bytes) store16_once(to + b0 + j * kStep, x[j]);
    }
}

__global__ __launch_bounds__(kThreads) void copy_kernel(CopyArgs a, const int32_t* __restrict__ src,
                                                        const int32_t* __restrict__ dst, int n) {
    const uint32_t block = linear_block<kThreads>();
    const int layer = static_cast<int>(block / static_cast<uint32_t>(n)), i = static_cast<int>(block % static_cast<uint32_t>(n));
    if (layer >= a.n_layers) return;
    const int from = src[i], to = dst[i];
    const uint32_t ids = static_cast<uint32_t>(a.n_hot) + static_cast<uint32_t>(a.n_cold);
    if (static_cast<uint32_t>(from) >= ids || static_cast<uint32_t>(to) >= ids || from == to) return;
    const auto page = [&](int id) {
        return id < a.n_hot ? a.hot + (static_cast<int64_t>(layer) * a.n_hot + id) * a.page_bytes
                            : a.cold + (static_cast<int64_t>(layer) * a.n_cold + id - a.n_hot) * a.page_bytes;
    };
    const auto sum = [&](int id) {
        return reinterpret_cast<unsigned char*>(a.sum) + (static_cast<int64_t>(layer) * ids + id) * a.sum_bytes;
    };
    copy_bytes(page(from), page(to), a.page_bytes);
    copy_bytes(sum(from), sum(to), a.sum_bytes);
}

int64_t items(const hga_plan& plan, const TokensView& tok) {
    return static_cast<int64_t>(tok.n_tokens) * plan.p.n_kv_heads;
}

template <typename T, int D>
hipError_t append_t(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* k, int64_t k_stride,
                    const void* v, int64_t v_stride, hipStream_t stream) {
    if (tok.n_tokens <= kFewTokens) {
        append_few_kernel<T, D><<<grid_of(plan.p.n_kv_heads, 64 * kFewWaves), 64 * kFewWaves, 0, stream>>>(
            pool, tok, static_cast<const T*>(k), k_stride, static_cast<const T*>(v), v_stride, phase_chunk(plan));
        return hipGetLastError();
    }
    constexpr int per = kThreads / (2 * D / 8);
    append_kernel<T, D><<<grid_of((items(plan, tok) + per - 1) / per, kThreads), kThreads, 0, stream>>>(
        pool, tok, static_cast<const T*>(k), k_stride, static_cast<const T*>(v), v_stride);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int64_t blocks = (static_cast<int64_t>(tok.n_tokens) + 63) / 64 * plan.p.n_kv_heads;
    close_kernel<D><<<grid_of(blocks, 64 * kCloseWaves), 64 * kCloseWaves, 0, stream>>>(pool, tok, phase_chunk(plan));
    return hipGetLastError();
}

template <typename T, int D>
hipError_t read_t(const hga_plan& plan, const PoolView& pool, const TokensView& tok, void* k, void* v,
                  hipStream_t stream) {
    constexpr int per = kThreads / (2 * D / 8);
    read_kernel<T, D><<<grid_of((items(plan, tok) + per - 1) / per, kThreads), kThreads, 0, stream>>>(
        pool, tok, static_cast<T*>(k), static_cast<T*>(v));
    return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* k,
                               int64_t k_stride, const void* v, int64_t v_stride, hipStream_t stream) {
    const bool f32 = plan.p.dtype == HGA_F32;
    const auto f = plan.p.head_dim == 128 ? (f32 ? append_t<float, 128> : append_t<bf16_t, 128>)
                                          : (f32 ? append_t<float, 64> : append_t<bf16_t, 64>);
    return f(plan, pool, tok, k, k_stride, v, v_stride, stream);
}

hipError_t launch_cache_read(const hga_plan& plan, const PoolView& pool, const TokensView& tok, void* k, void* v,
                             hipStream_t stream) {
    const bool f32 = plan.p.dtype == HGA_F32;
    const auto f = plan.p.head_dim == 128 ? (f32 ? read_t<float, 128> : read_t<bf16_t, 128>)
                                          : (f32 ? read_t<float, 64> : read_t<bf16_t, 64>);
    return f(plan, pool, tok, k, v, stream);
}

hipError_t launch_copy_pages(const hga_plan& plan, const hga_pool& pool, void* cold, const int32_t* src,
                             const int32_t* dst, int n, hipStream_t stream) {
    CopyArgs a;
    a.hot = static_cast<unsigned char*>(pool.pages);
    a.cold = static_cast<unsigned char*>(cold);
    a.sum = pool.page_sum;
    a.n_hot = pool.n_pages;
    a.n_cold = pool.n_cold;
    a.n_layers = pool.n_layers;
    a.page_bytes = static_cast<int64_t>(plan.p.n_kv_heads) * page_head_bytes(plan.p.head_dim);
    a.sum_bytes = static_cast<int64_t>(plan.p.n_kv_heads) * plan.p.head_dim * 4;
    const int64_t blocks = static_cast<int64_t>(n) * a.n_layers;
    copy_kernel<<<grid_of(blocks, kThreads), kThreads, 0, stream>>>(a, src, dst, n);
    return hipGetLastError();
}

}  // namespace hga

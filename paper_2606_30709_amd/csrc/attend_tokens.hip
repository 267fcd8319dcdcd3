// Attention of single tokens over the paged 4-bit cache (Sec. 3.4 at the token's grain, every query head of a KV head in
// one tile).
//
// A unit is (token, KV head).  Its query heads are the columns of a 16-column tile:
//   S^T [16 keys x 16 heads] = K~ [16 x d] q^T      (d/32 instructions of 16x16x32)
//   O^T [16 dims x 16 heads] += V~^T [16 x 32] P^T  (a 32-key half page, d/16 instructions)
// Codes become bf16 in registers, two an instruction with their scale.  The layout of a page (tokens.hpp) is that of these
// operands, so codes go straight from memory to the lane that multiplies them.  A lane of S^T holds keys 4 g .. 4 g + 3 of
// its tile, and takes those as its reduction indices of the second product: P never leaves the lane.  One pass over the
// keys with the running maximum and sum (in log2 units) of each head.
//
// fp32 queries and weights enter the matrix instructions as three bf16 terms each (24 bits); the stored keys and values are
// exact in bf16.
#include "hga_device.hpp"
#include "hga_internal.hpp"
#include "tokens.hpp"

namespace hga {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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
__device__ __forceinline__ float low_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// kTerms words whose bf16 pairs add up to (a, b): the rounded values, then what rounding left.
template <int kTerms>
__device__ __forceinline__ void split2(float a, float b, uint32_t* w) {
#pragma unroll
    for (int i = 0; i < kTerms; ++i) {
        w[i] = pack2(a, b);
        a -= low_f32(w[i]);
        b -= high_f32(w[i]);
    }
}

template <int D>
struct Page {  // a lane's share of a page
    uint32_t k[4][D / 32];
    uint32_t v[4][D / 32];
    uint32_t ks;
    uint32_t vs[4];
};

template <int D>
__device__ __forceinline__ void load_codes(const unsigned char* p, uint32_t* w) {
    if constexpr (D == 128) {
        const vec16 x = load16(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = x.w[i];
    } else {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        w[0] = x.x;
        w[1] = x.y;
    }
}

template <int D>
__device__ __forceinline__ void load_page(const unsigned char* head, int m, int g, Page<D>& pg) {
    using F = PageFormat<D>;
#pragma unroll
    for (int t = 0; t < 4; ++t) load_codes<D>(head + F::key_code(16 * t + m, g * (D / 4)), pg.k[t]);
    pg.ks = *reinterpret_cast<const uint32_t*>(head + F::key_scale(m, g * (D / 4) / 32));
#pragma unroll
    for (int t = 0; t < 4; ++t) load_codes<D>(head + F::value_code(16 * t + 4 * g, m * F::kLaneDims), pg.v[t]);
    const vec16 x = load16(head + F::value_scale(4 * g, m * F::kLaneDims / 32));
#pragma unroll
    for (int t = 0; t < 4; ++t) pg.vs[t] = x.w[t];
}

__device__ __forceinline__ float max_groups(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_groups(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

struct AttendArgs {
    const int32_t* list;  // NULL: every chunk
    int n_list, ratio;
    float* lse;
};

// A workgroup per unit; its wavefronts take every fourth page each and are joined in LDS.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void attend_tokens_kernel(PoolView pool, TokensView tok, AttendArgs a,
                                                                 const T* __restrict__ q, int64_t q_stride,
                                                                 T* __restrict__ out) {
    using F = PageFormat<D>;
    constexpr int kTerms = sizeof(T) == 4 ? 3 : 1;
    constexpr int DL = F::kLaneDims;
    constexpr int kSteps = D / 32;
    const float scale = 1.4426950408889634f / sqrtf(static_cast<float>(D));  // log2(e) / sqrt(d)
    __shared__ float s_o[kWaves][16][D + 4];
    __shared__ float s_m[kWaves][16], s_l[kWaves][16];
    const int64_t unit = linear_block<kThreads>();
    const int t = static_cast<int>(unit / pool.n_kv), h = static_cast<int>(unit % pool.n_kv);
    if (t >= tok.n_tokens) return;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, m = lane & 15, g = lane >> 4;
    int s = 0, p = 0;
    const bool in = tok.at(t, s, p);
    const int n_entries = !in ? 0 : a.list ? a.n_list : p / kPageRows + 1;
    const int32_t* list = a.list ? a.list + unit * a.n_list : nullptr;

    // column m: query head m of the KV head's (zeros past the last)
    u32x4 qf[kTerms][kSteps];
    {
        const T* row = q + t * q_stride + (static_cast<int64_t>(h) * a.ratio + m) * D + g * (D / 4);
#pragma unroll
        for (int kk = 0; kk < kSteps; ++kk) {
            float x[8] = {};
            if (in && m < a.ratio) load8(row + 8 * kk, x);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t w[kTerms];
                split2<kTerms>(x[2 * i], x[2 * i + 1], w);
#pragma unroll
                for (int e = 0; e < kTerms; ++e) qf[e][kk][i] = w[e];
            }
        }
    }
    f32x4 o[DL];
#pragma unroll
    for (int j = 0; j < DL; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_run = -INFINITY, l_run = 0.f;

    for (int e0 = wave; e0 < n_entries; e0 += 64 * kWaves) {
        // the next 64 entries of this wavefront, one a lane
        SeenPage mine{-1, 0};
        const int e = e0 + lane * kWaves;
        if (e < n_entries) mine = seen_page(pool, tok, s, p, list ? list[e] : e);
        const int batch = min(64, (n_entries - e0 + kWaves - 1) / kWaves);
        for (int i = 0; i < batch; ++i) {
            const int rows = __builtin_amdgcn_readlane(mine.rows, i);
            if (rows == 0) continue;
            const unsigned char* head = pool.page(__builtin_amdgcn_readlane(mine.id, i)) + h * F::kBytes;
            Page<D> pg;
            load_page<D>(head, m, g, pg);

            f32x4 sc[4];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                const float ks = scale_of(pg.ks >> (8 * tt) & 255u);
                sc[tt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < kSteps; ++kk) {
                    const uint32_t c = pg.k[tt][kk];
                    const u32x4 kf = {decode2<0>(c, ks), decode2<1>(c, ks), decode2<2>(c, ks), decode2<3>(c, ks)};
#pragma unroll
                    for (int x = 0; x < kTerms; ++x) sc[tt] = mfma(kf, qf[x][kk], sc[tt]);
                }
            }
            if (rows < kPageRows) {  // the token's own page: rows behind it hold anything
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (16 * tt + 4 * g + x >= rows) {
                            sc[tt][x] = -INFINITY;
                            pg.vs[tt] = (pg.vs[tt] & ~(255u << (8 * x))) | 127u << (8 * x);
                        }
                // codes of an unseen row: zeros, as its weight is (a scale of NaN went above)
            }
            float top = sc[0][0];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                for (int x = 0; x < 4; ++x) top = fmaxf(top, sc[tt][x]);
            const float m_new = fmaxf(m_run, max_groups(top) * scale);
            const float m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_use);
            m_run = m_new;
            l_run *= alpha;
#pragma unroll
            for (int j = 0; j < DL; ++j) o[j] *= alpha;
            // weights, four keys of a tile as two words: half page u is tiles 2u, 2u + 1
            uint32_t w[4][2][kTerms];
#pragma unroll
            for (int tt = 0; tt < 4; ++tt) {
                float pv[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    pv[x] = __builtin_amdgcn_exp2f(fmaf(sc[tt][x], scale, -m_use));
                    l_run += pv[x];
                }
                split2<kTerms>(pv[0], pv[1], w[tt][0]);
                split2<kTerms>(pv[2], pv[3], w[tt][1]);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                u32x4 pf[kTerms];
#pragma unroll
                for (int x = 0; x < kTerms; ++x)
                    pf[x] = u32x4{w[2 * u][0][x], w[2 * u][1][x], w[2 * u + 1][0][x], w[2 * u + 1][1][x]};
                // rows of a quad decoded two dimensions at a time, then paired by row
                uint32_t vf[DL][4];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int tt = 2 * u + b;
#pragma unroll
                    for (int r2 = 0; r2 < 2; ++r2) {
                        uint32_t lo[DL / 2], hi[DL / 2];
                        const float s0 = scale_of(pg.vs[tt] >> (16 * r2) & 255u);
                        const float s1 = scale_of(pg.vs[tt] >> (16 * r2 + 8) & 255u);
                        if constexpr (DL == 8) {
                            const uint32_t c0 = pg.v[tt][2 * r2], c1 = pg.v[tt][2 * r2 + 1];
                            lo[0] = decode2<0>(c0, s0);
                            lo[1] = decode2<1>(c0, s0);
                            lo[2] = decode2<2>(c0, s0);
                            lo[3] = decode2<3>(c0, s0);
                            hi[0] = decode2<0>(c1, s1);
                            hi[1] = decode2<1>(c1, s1);
                            hi[2] = decode2<2>(c1, s1);
                            hi[3] = decode2<3>(c1, s1);
                        } else {
                            const uint32_t c = pg.v[tt][r2];
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
                for (int j = 0; j < DL; ++j) {
                    const u32x4 va = {vf[j][0], vf[j][1], vf[j][2], vf[j][3]};
#pragma unroll
                    for (int x = 0; x < kTerms; ++x) o[j] = mfma(va, pf[x], o[j]);
                }
            }
        }
    }

    // join the wavefronts: lane (m, g) holds head m, dimensions (4 g + x) DL + j
    l_run = sum_groups(l_run);
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int j = 0; j < DL; ++j) s_o[wave][m][(4 * g + x) * DL + j] = o[j][x];
    if (g == 0) {
        s_m[wave][m] = m_run;
        s_l[wave][m] = l_run;
    }
    __syncthreads();
    for (int i = tid; i < a.ratio * D; i += kThreads) {
        const int r = i / D, c = i % D;
        float top = s_m[0][r];
        for (int w = 1; w < kWaves; ++w) top = fmaxf(top, s_m[w][r]);
        const float base = top == -INFINITY ? 0.f : top;
        float l = 0.f, acc = 0.f;
        for (int w = 0; w < kWaves; ++w) {
            // a wavefront without a maximum has seen nothing (zeros) or only what is not a number
            const float f = s_m[w][r] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(s_m[w][r] - base);
            l += f * s_l[w][r];
            acc += f * s_o[w][r][c];
        }
        const int64_t row = static_cast<int64_t>(t) * pool.n_kv * a.ratio + h * a.ratio + r;
        out[row * D + c] = elem<T>::from_f32(l == 0.f ? 0.f : acc / l);
        if (a.lse && c == 0) a.lse[row] = l == 0.f ? -INFINITY : base * 0.6931471805599453f + logf(l);
    }
}

template <typename T, int D>
hipError_t run(const PoolView& pool, const TokensView& tok, const AttendArgs& a, const void* q, int64_t q_stride,
               void* out, hipStream_t stream) {
    const int64_t n = static_cast<int64_t>(tok.n_tokens) * pool.n_kv;
    attend_tokens_kernel<T, D><<<grid_of(n, kThreads), kThreads, 0, stream>>>(
        pool, tok, a, static_cast<const T*>(q), q_stride, static_cast<T*>(out));
    return hipGetLastError();
}

}  // namespace

int64_t attend_tokens_bytes(const hga_plan&, int, int, int, int) { return 0; }

hipError_t launch_attend_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                                int64_t q_stride, const int32_t* list, int n_list, void* out, float* lse, void*, int64_t,
                                hipStream_t stream) {
    AttendArgs a;
    a.list = list;
    a.n_list = n_list;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.lse = lse;
    const bool f32 = plan.p.dtype == HGA_F32;
    const auto f = plan.p.head_dim == 128 ? (f32 ? run<float, 128> : run<bf16_t, 128>)
                                          : (f32 ? run<float, 64> : run<bf16_t, 64>);
    return f(pool, tok, a, q, q_stride, out, stream);
}

}  // namespace hga

// Routing of single tokens to pages (Sec. 3.3 at the token's grain): the chunks a token sees are its own, the
// deterministic ones (the first keep_first, the window before its own) and, of the middle ones, the topk_chunks whose
// page summaries have the largest products with the mean of the token's query heads.
//
// Scores are sums of 64-bit products: an fp32 score's error exceeds the gap at the border of the selection once in some
// tens of thousands of selections, a 64-bit one's practically never, and the fp64 rate of the vector unit equals its fp32
// rate, so a decode step stays bound by the summaries' bytes.  (The mean is taken as the sum: the order is the same.)  A
// score becomes a 64-bit key that orders as the score does.
//
// A unit is (token, KV head).  Three forms, the same lists:
//   a wavefront a unit    many units of short histories (prompts): keys in registers, no barrier
//   a workgroup a unit    keys in LDS
//   two kernels           few units of long histories: their scores by workgroups of kSlice rows each, keys in the
//                         workspace; then the choice, a workgroup a unit; as many tokens at a time as the workspace holds
#include <algorithm>

#include "hga_device.hpp"
#include "tokens_internal.hpp"

namespace hga {
namespace {

constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kLanes = 8;  // lanes of a summary row
// Pages of a sequence up to which a unit's keys lie in LDS (128 of its 160 KiB).
constexpr int kLdsPages = 1 << 14;
// Pages of a sequence up to which a wavefront takes a unit: keys a lane.
constexpr int kLaneKeys = 4;
constexpr int kSlice = 128;  // rows of a scoring workgroup of the two-kernel form
// Bytes of keys that the two-kernel form asks for, or one token's: a call of more tokens takes them in parts.  (A page
// table may be wide for the sake of one sequence: 4,096 tokens of 4 heads at 2^18 pages would have 32 GiB of keys.)
constexpr int64_t kKeyBytes = int64_t(1) << 28;

// A key that orders as the score: 0 is no candidate, 1 a score that is not a number.
__device__ __forceinline__ uint64_t score_key(double s) {
    if (s != s) return 1;
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(s + 0.0));
    return u >> 63 ? ~u : u | (uint64_t(1) << 63);
}
__device__ __forceinline__ double key_score(uint64_t k) {
    return __longlong_as_double(static_cast<long long>(k >> 63 ? k ^ (uint64_t(1) << 63) : ~k));
}

struct RouteArgs {
    int first, window, topk, ratio, n_list;
};

// The middle chunks [lo, hi) of a token whose own chunk is `own`.
__device__ __forceinline__ void middle(const RouteArgs& a, int own, int& lo, int& hi) {
    lo = min(a.first, own);
    hi = max(lo, own - a.window);
}

template <int kCtrl>
__device__ __forceinline__ double add_dpp_f64(double x) {
    const uint64_t u = static_cast<uint64_t>(__double_as_longlong(x));
    const uint32_t lo = static_cast<uint32_t>(
        __builtin_amdgcn_mov_dpp(static_cast<int>(static_cast<uint32_t>(u)), kCtrl, 0xf, 0xf, true));
    const uint32_t hi =
        static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(u >> 32), kCtrl, 0xf, 0xf, true));
    return x + __longlong_as_double(static_cast<long long>(static_cast<uint64_t>(hi) << 32 | lo));
}

// The sum over a row's eight lanes, in all of them: within pairs, within quads, then the quads of the half row.
__device__ __forceinline__ double row_sum(double x) {
    x = add_dpp_f64<0xB1>(x);   // quad_perm 1 0 3 2
    x = add_dpp_f64<0x4E>(x);   // quad_perm 2 3 0 1
    return add_dpp_f64<0x141>(x);  // row_half_mirror
}

// Dimension `dim` of the token's summed query heads.
template <typename T, int D>
__device__ __forceinline__ double head_sum(const T* qt, int dim, int ratio) {
    double s = 0.0;
#pragma unroll 4
    for (int r = 0; r < ratio; ++r) s += static_cast<double>(elem<T>::to_f32(qt[r * D + dim]));
    return s;
}

// The lane's dimensions of a row (16-byte pieces, eight lanes side by side) from the D sums in LDS.
template <int D>
__device__ __forceinline__ void load_query(const double* s_q, int sub, double (&q)[D / kLanes]) {
#pragma unroll
    for (int x = 0; x < D / 32; ++x)
#pragma unroll
        for (int j = 0; j < 4; ++j) q[4 * x + j] = s_q[(x * kLanes + sub) * 4 + j];
}

// Keys of kRows rows of a lane group, all their loads issued before the first is used; id < 0: no candidate.
template <int D, int kRows>
__device__ __forceinline__ void score_rows(const PoolView& pool, int h, const int (&id)[kRows], int sub,
                                           const double (&q)[D / kLanes], uint64_t (&key)[kRows]) {
    float4 w[kRows][D / 32];
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        const float* row = pool.sum + (static_cast<int64_t>(max(id[y], 0)) * pool.n_kv + h) * D;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) w[y][x] = *reinterpret_cast<const float4*>(row + (x * kLanes + sub) * 4);
    }
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        double acc = 0.0;
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            acc = fma(q[4 * x], static_cast<double>(w[y][x].x), acc);
            acc = fma(q[4 * x + 1], static_cast<double>(w[y][x].y), acc);
            acc = fma(q[4 * x + 2], static_cast<double>(w[y][x].z), acc);
            acc = fma(q[4 * x + 3], static_cast<double>(w[y][x].w), acc);
        }
        acc = row_sum(acc);
        key[y] = id[y] >= 0 ? score_key(acc) : 0;
    }
}

// The page of a middle chunk, -1 if absent (its row is read as page 0's, which a pool that the kernels see has).
__device__ __forceinline__ int page_or_none(const PoolView& pool, const TokensView& tok, int s, int c) {
    const int id = tok.page_id(s, c);
    return pool.has(id) ? id : -1;
}

// ------------------------------------------------------------ a workgroup a unit ---

__device__ __forceinline__ int block_scan(int x, int* s_w, int& total) {  // exclusive
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int incl = wave_incl_scan_add(x);
    if (lane == 63) s_w[wave] = incl;
    __syncthreads();
    int before = incl - x;
    total = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int n = s_w[w];
        if (w < wave) before += n;
        total += n;
    }
    __syncthreads();
    return before;
}

// The border of a selection: keys above `key` (under `mask`) are taken, of those equal to it the first `ties` (all: there
// are no more of them).
struct Border {
    uint64_t key, mask;
    int ties;
    bool all;
};

struct ChooseLds {
    uint32_t hist[2048];
    uint64_t cand[kThreads];
    int cand_at[kThreads];
    uint64_t lo[kWaves], hi[kWaves];
    int scan[kWaves];
    int bin, above, n_cand;
    uint64_t border;
    int ties;
    bool all;
};

// By counting, from the most significant byte down: any keys.
__device__ __forceinline__ Border border_by_bytes(const uint64_t* keys, int n, int k, ChooseLds& s) {
    const int tid = threadIdx.x;
    Border b{0, 0, k, false};
    for (int shift = 56; shift >= 0; shift -= 8) {
        if (tid < 256) s.hist[tid] = 0;
        __syncthreads();
        for (int i = tid; i < n; i += kThreads) {
            const uint64_t v = keys[i];
            if (v != 0 && (v & b.mask) == b.key) atomicAdd(&s.hist[v >> shift & 255], 1u);
        }
        __syncthreads();
        // every thread walks down from the top bin to the one that holds the border
        int bin = 255, above = 0;
        while (bin > 0 && above + static_cast<int>(s.hist[bin]) < b.ties) above += static_cast<int>(s.hist[bin--]);
        const int in = static_cast<int>(s.hist[bin]);
        b.key |= static_cast<uint64_t>(bin) << shift;
        b.mask |= uint64_t(255) << shift;
        b.ties -= above;
        __syncthreads();
        if (in == b.ties) {  // all of the bin
            b.all = true;
            break;
        }
    }
    return b;
}

// By one count over 2048 equal steps between the least and the largest score (monotonic in the score, each step of the
// computation being so), which spreads the counts over the bins as the scores are spread, and the few keys of the border's
// bin ranked one by one.  Scores that are not finite, or a bin of more than a key a thread: by bytes.
__device__ __forceinline__ Border find_border(const uint64_t* keys, int n, int k, uint64_t least, uint64_t most,
                                              ChooseLds& s) {
    const int tid = threadIdx.x;
    const double lo = key_score(least), hi = key_score(most), width = hi - lo;
    if (least == 1 || !(width > 0.0) || !(width < 1.7e308) || !(2048.0 / width < 1.7e308))
        return border_by_bytes(keys, n, k, s);
    const double step = 2047.0 / width;
    const auto bin_of = [&](uint64_t v) { return min(2047, static_cast<int>((key_score(v) - lo) * step)); };
#pragma unroll
    for (int i = 0; i < 2048 / kThreads; ++i) s.hist[i * kThreads + tid] = 0;
    if (tid == 0) s.n_cand = 0;
    __syncthreads();
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t v = keys[i];
        if (v != 0) atomicAdd(&s.hist[bin_of(v)], 1u);
    }
    __syncthreads();
    // thread i counts bins 2047 - 4 i .. 2044 - 4 i: those before it are above
    constexpr int kBins = 2048 / kThreads;
    int mine = 0, total;
#pragma unroll
    for (int i = 0; i < kBins; ++i) mine += static_cast<int>(s.hist[2047 - tid * kBins - i]);
    int above = block_scan(mine, s.scan, total);
    if (above < k && above + mine >= k) {
        int bin = 2047 - tid * kBins;
        while (above + static_cast<int>(s.hist[bin]) < k) above += static_cast<int>(s.hist[bin--]);
        s.bin = bin;
        s.above = above;
    }
    __syncthreads();
    const int bin = s.bin, need = k - s.above, in = static_cast<int>(s.hist[bin]);
    if (in > kThreads) {
        __syncthreads();  // every thread has read its count before the counts are cleared for bytes
        return border_by_bytes(keys, n, k, s);
    }
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t v = keys[i];
        if (v != 0 && bin_of(v) == bin) {
            const int at = atomicAdd(&s.n_cand, 1);
            s.cand[at] = v;
            s.cand_at[at] = i;
        }
    }
    __syncthreads();
    if (tid < in) {
        const uint64_t v = s.cand[tid];
        int rank = 0, upto = 1, equal = 0;  // keys before this one; equal ones up to it, and in all
        for (int i = 0; i < in; ++i) {
            const bool same = s.cand[i] == v, tie = same && s.cand_at[i] < s.cand_at[tid];
            rank += s.cand[i] > v || tie;
            upto += tie;
            equal += same;
        }
        if (rank == need - 1) {
            s.border = v;
            s.ties = upto;
            s.all = upto == equal;
        }
    }
    __syncthreads();
    return Border{s.border, ~uint64_t(0), s.ties, s.all};
}

// A unit's list from its keys[0..n) of middle chunks lo .. lo + n - 1.
__device__ __forceinline__ void choose(const PoolView& pool, const TokensView& tok, const RouteArgs& a, int s, int own,
                                       int lo, int n, const uint64_t* keys, int32_t* out, ChooseLds& lds) {
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    int found = 0, total;
    uint64_t least = ~uint64_t(0), most = 0;
    for (int i = tid; i < n; i += kThreads) {
        const uint64_t v = keys[i];
        if (v == 0) continue;
        ++found;
        least = v < least ? v : least;
        most = v > most ? v : most;
    }
    // least as the largest complement
    most = wave_max_u64(most);
    least = ~wave_max_u64(~least);
    if (lane == 0) {
        lds.lo[wave] = least;
        lds.hi[wave] = most;
    }
    block_scan(found, lds.scan, total);
    Border b{0, 0, 0, true};
    if (total > a.topk) {  // more candidates than are taken
        for (int w = 0; w < kWaves; ++w) {
            least = lds.lo[w] < least ? lds.lo[w] : least;
            most = lds.hi[w] > most ? lds.hi[w] : most;
        }
        b = find_border(keys, n, a.topk, least, most, lds);
    }
    // thread i takes a run of chunks; their ranks from a scan of the chosen, and one of the ties where some are left out
    const int per = own / kThreads + 1, c0 = min(tid * per, own + 1), c1 = min(c0 + per, own + 1);
    const auto key = [&](int c) { return keys[c - lo]; };
    int ties0 = 0;
    if (!b.all) {
        int ties = 0;
        for (int c = max(c0, lo); c < min(c1, lo + n); ++c) ties += key(c) != 0 && (key(c) & b.mask) == b.key;
        ties0 = block_scan(ties, lds.scan, total);
    }
    const auto pick = [&](int c, int& tie) {
        if (c < lo || c >= lo + n) return pool.has(tok.page_id(s, c));
        const uint64_t v = key(c) & b.mask;
        if (key(c) == 0 || v < b.key) return false;
        return b.all || v != b.key || tie++ < b.ties;
    };
    if (per <= 64) {  // a run's choices fit a word: made once
        uint64_t picked = 0;
        for (int c = c0; c < c1; ++c)
            if (pick(c, ties0)) picked |= uint64_t(1) << (c - c0);
        int rank = block_scan(__popcll(picked), lds.scan, total);
        for (; picked; picked &= picked - 1, ++rank)
            if (rank < a.n_list) out[rank] = c0 + static_cast<int>(__builtin_ctzll(picked));
    } else {
        int count = 0, tie = ties0;
        for (int c = c0; c < c1; ++c) count += pick(c, tie);
        int rank = block_scan(count, lds.scan, total);
        tie = ties0;
        for (int c = c0; c < c1; ++c)
            if (pick(c, tie) && rank < a.n_list) out[rank++] = c;
    }
    for (int i = total + tid; i < a.n_list; i += kThreads) out[i] = -1;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void route_block_kernel(PoolView pool, TokensView tok, RouteArgs a,
                                                               const T* __restrict__ q, int64_t q_stride,
                                                               int32_t* __restrict__ list) {
    extern __shared__ __align__(16) uint64_t keys[];
    __shared__ ChooseLds lds;
    __shared__ double s_q[D];
    const int64_t unit = linear_block<kThreads>();
    const auto [t, h] = token_head(static_cast<uint32_t>(unit), pool.n_kv);
    if (t >= tok.n_tokens) return;
    const int tid = threadIdx.x, sub = tid % kLanes;
    int32_t* out = list + unit * a.n_list;
    int s, p;
    if (!tok.at(t, s, p)) {
        for (int i = tid; i < a.n_list; i += kThreads) out[i] = -1;
        return;
    }
    const int own = p / kPageRows;
    int lo, hi;
    middle(a, own, lo, hi);
    const int n = hi - lo;
    if (tid < D) s_q[tid] = head_sum<T, D>(q + t * q_stride + static_cast<int64_t>(h) * a.ratio * D, tid, a.ratio);
    // pages first, where their keys will be
    for (int i = tid; i < n; i += kThreads) keys[i] = static_cast<uint64_t>(page_or_none(pool, tok, s, lo + i));
    __syncthreads();
    double qd[D / kLanes];
    load_query<D>(s_q, sub, qd);
    constexpr int kRows = 4, kGroups = kThreads / kLanes;
    for (int i0 = tid / kLanes; i0 < n; i0 += kRows * kGroups) {
        int id[kRows];
        uint64_t k[kRows];
#pragma unroll
        for (int y = 0; y < kRows; ++y) id[y] = i0 + y * kGroups < n ? static_cast<int>(keys[i0 + y * kGroups]) : -1;
        score_rows<D, kRows>(pool, h, id, sub, qd, k);
        __builtin_amdgcn_wave_barrier();  // a row's lanes have read its page before one of them overwrites it
#pragma unroll
        for (int y = 0; y < kRows; ++y)
            if (sub == 0 && i0 + y * kGroups < n) keys[i0 + y * kGroups] = k[y];
    }
    __syncthreads();
    choose(pool, tok, a, s, own, lo, n, keys, out, lds);
}

// ------------------------------------------------------------------- two kernels ---

// Keys of middle chunks [slice kSlice, ...) of a unit into ws[unit][max_pages].
template <typename T, int D>
__global__ __launch_bounds__(256) void score_slices_kernel(PoolView pool, TokensView tok, RouteArgs a, int slices,
                                                           const T* __restrict__ q, int64_t q_stride,
                                                           uint64_t* __restrict__ ws) {
    __shared__ double s_q[D];
    const uint32_t block = linear_block<256>();
    const int64_t unit = block / static_cast<uint32_t>(slices);
    const auto [t, h] = token_head(static_cast<uint32_t>(unit), pool.n_kv);
    if (t >= tok.n_tokens) return;
    int s, p;
    if (!tok.at(t, s, p)) return;
    int lo, hi;
    middle(a, p / kPageRows, lo, hi);
    const int n = hi - lo, i0 = static_cast<int>(block % static_cast<uint32_t>(slices)) * kSlice;
    if (i0 >= n) return;
    const int tid = threadIdx.x, sub = tid % kLanes;
    constexpr int kGroups = 256 / kLanes, kRows = kSlice / kGroups;
    int id[kRows];
    uint64_t k[kRows];
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        const int i = i0 + y * kGroups + tid / kLanes;
        id[y] = i < n ? page_or_none(pool, tok, s, lo + i) : -1;
    }
    if (tid < D) s_q[tid] = head_sum<T, D>(q + t * q_stride + static_cast<int64_t>(h) * a.ratio * D, tid, a.ratio);
    __syncthreads();
    double qd[D / kLanes];
    load_query<D>(s_q, sub, qd);
    score_rows<D, kRows>(pool, h, id, sub, qd, k);
#pragma unroll
    for (int y = 0; y < kRows; ++y) {
        const int i = i0 + y * kGroups + tid / kLanes;
        if (sub == 0 && i < n) ws[unit * tok.max_pages + i] = k[y];
    }
}

__global__ __launch_bounds__(kThreads) void choose_kernel(PoolView pool, TokensView tok, RouteArgs a,
                                                          const uint64_t* __restrict__ ws, int32_t* __restrict__ list) {
    __shared__ ChooseLds lds;
    const int64_t unit = linear_block<kThreads>();
    const int t = token_head(static_cast<uint32_t>(unit), pool.n_kv).t;
    if (t >= tok.n_tokens) return;
    int32_t* out = list + unit * a.n_list;
    int s, p;
    if (!tok.at(t, s, p)) {
        for (int i = threadIdx.x; i < a.n_list; i += kThreads) out[i] = -1;
        return;
    }
    int lo, hi;
    middle(a, p / kPageRows, lo, hi);
    choose(pool, tok, a, s, p / kPageRows, lo, hi - lo, ws + unit * tok.max_pages, out, lds);
}

// ------------------------------------------------------------- a wavefront a unit ---

// Middle chunk lo + 64 j + i is key j of lane i.  The K_c-th largest is found bit by bit, by ballots.
template <typename T, int D, int kKeys>
__global__ __launch_bounds__(256) void route_wave_kernel(PoolView pool, TokensView tok, RouteArgs a,
                                                         const T* __restrict__ q, int64_t q_stride,
                                                         int32_t* __restrict__ list) {
    __shared__ double s_q[4][D];
    __shared__ uint64_t s_k[4][64 * kKeys];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, sub = lane % kLanes;
    const int64_t unit = static_cast<int64_t>(linear_block<256>()) * 4 + wave;
    const auto [t, h] = token_head(static_cast<uint32_t>(unit), pool.n_kv);
    if (t >= tok.n_tokens) return;
    int32_t* out = list + unit * a.n_list;
    int s, p;
    if (!tok.at(t, s, p)) {
        for (int i = lane; i < a.n_list; i += 64) out[i] = -1;
        return;
    }
    const int own = p / kPageRows;
    int lo, hi;
    middle(a, own, lo, hi);
    const int n = hi - lo;
    const T* qt = q + t * q_stride + static_cast<int64_t>(h) * a.ratio * D;
#pragma unroll
    for (int i = 0; i < D; i += 64) s_q[wave][i + lane] = head_sum<T, D>(qt, i + lane, a.ratio);
    int id[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; ++j) id[j] = 64 * j + lane < n ? page_or_none(pool, tok, s, lo + 64 * j + lane) : -1;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    double qd[D / kLanes];
    load_query<D>(s_q[wave], sub, qd);
    uint64_t key[kKeys];
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
        key[j] = 0;
        if (64 * j >= n) continue;
        // eight rows a step, four steps at once
        for (int r0 = 0; r0 < 64; r0 += 32) {
            int rid[4];
            uint64_t k[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) rid[y] = __shfl(id[j], r0 + 8 * y + lane / kLanes);
            score_rows<D, 4>(pool, h, rid, sub, qd, k);
#pragma unroll
            for (int y = 0; y < 4; ++y)
                if (sub == 0) s_k[wave][64 * j + r0 + 8 * y + lane / kLanes] = k[y];
        }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    int found = 0;
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
        if (64 * j < n) key[j] = s_k[wave][64 * j + lane];
        found += __popcll(__builtin_amdgcn_ballot_w64(key[j] != 0));
    }
    uint64_t border = 1;  // every candidate
    int ties = 64 * kKeys;
    if (found > a.topk) {
        border = 0;
        int count = found;  // keys >= border
        for (int b = 63; b >= 0 && count != a.topk; --b) {
            const uint64_t next = border | uint64_t(1) << b;
            int c = 0;
#pragma unroll
            for (int j = 0; j < kKeys; ++j) c += __popcll(__builtin_amdgcn_ballot_w64(key[j] >= next));
            if (c >= a.topk) {
                border = next;
                count = c;
            }
        }
        // as many keys as are taken reach the border, or more do: then it is their common value
        int above = 0;
#pragma unroll
        for (int j = 0; j < kKeys; ++j) above += __popcll(__builtin_amdgcn_ballot_w64(key[j] > border));
        if (count != a.topk) ties = a.topk - above;
    }
    // chunks in order: the first ones, the middle ones, the window and the token's own
    const uint64_t below = (uint64_t(1) << lane) - 1;
    int base = 0, tied = 0;
    const auto put = [&](bool pick, int c) {
        const uint64_t m = __builtin_amdgcn_ballot_w64(pick);
        const int rank = base + __popcll(m & below);
        if (pick && rank < a.n_list) out[rank] = c;
        base += __popcll(m);
    };
    for (int c = 0; c < lo; c += 64) put(c + lane < lo && pool.has(tok.page_id(s, c + lane)), c + lane);
#pragma unroll
    for (int j = 0; j < kKeys; ++j) {
        if (64 * j >= n) continue;
        const bool tie = key[j] == border;
        const uint64_t m = __builtin_amdgcn_ballot_w64(tie);
        put(key[j] > border || (tie && tied + __popcll(m & below) < ties), lo + 64 * j + lane);
        tied += __popcll(m);
    }
    for (int c = hi; c <= own; c += 64) put(c + lane <= own && pool.has(tok.page_id(s, c + lane)), c + lane);
    for (int i = base + lane; i < a.n_list; i += 64) out[i] = -1;
}

// Few units of long histories take two kernels: where a workgroup a unit would leave most of the device idle for the
// time that one takes over its summaries (128K tokens: 1 MiB at 512 bytes a chunk). 4 heads of d128, in two and in one: 1
// token at 32K 9.3 and 8.6 us, at 128K 11.9 and 17.1; 16 sequences at 64K 13.8 and 13.9.
bool few_and_long(const hga_plan& plan, int64_t units, int max_pages) {
    return max_pages > kLdsPages || (max_pages >= 8 * kSlice && units * 4 <= plan.n_cu);
}

template <typename T, int D>
hipError_t run(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const RouteArgs& a, const void* q,
               int64_t q_stride, int32_t* list, uint64_t* ws, int64_t ws_tokens, hipStream_t stream) {
    const int64_t units = static_cast<int64_t>(tok.n_tokens) * pool.n_kv;
    const T* qt = static_cast<const T*>(q);
    if (ws) {
        const int slices = (tok.max_pages + kSlice - 1) / kSlice;
        const int64_t part = std::min(ws_tokens, (int64_t(1) << 30) / (static_cast<int64_t>(slices) * pool.n_kv));
        for (int64_t t = 0; t < tok.n_tokens; t += part) {
            TokensView some = tok;
            some.seq += t;
            some.pos += t;
            some.n_tokens = static_cast<int>(std::min(part, tok.n_tokens - t));
            const int64_t n = static_cast<int64_t>(some.n_tokens) * pool.n_kv;
            score_slices_kernel<T, D><<<grid_of(n * slices, 256), 256, 0, stream>>>(pool, some, a, slices,
                                                                                   qt + t * q_stride, q_stride, ws);
            hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            choose_kernel<<<grid_of(n, kThreads), kThreads, 0, stream>>>(pool, some, a, ws,
                                                                         list + t * pool.n_kv * a.n_list);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    // A wavefront a unit: up to 64 chunks, a key a lane, at any count (3 heads of d64 at 4K, 1 token: 4.9 us, 6.6 with a
    // workgroup; 330 tokens: 5.7 and 12.5); up to four keys a lane where the units fill the device (1 token at 8K: 7.1 and
    // 6.7 us, 330: 8.4 and 12.7; 256 tokens at 16K: 10.8 and 10.3, 400: 12.9 and 15.0).
    if (tok.max_pages <= 64 || (tok.max_pages <= 64 * kLaneKeys && units >= 4 * plan.n_cu)) {
        // a key a lane or four: 4,096 tokens of 3 heads at 4K 16 and 19.5 us
        const auto kernel = tok.max_pages <= 64 ? route_wave_kernel<T, D, 1> : route_wave_kernel<T, D, kLaneKeys>;
        kernel<<<grid_of((units + 3) / 4, 256), 256, 0, stream>>>(pool, tok, a, qt, q_stride, list);
        return hipGetLastError();
    }
    static std::atomic<uint64_t> done{0};
    const hipError_t e = once_per_device(done, plan.device, [] {
        return hipFuncSetAttribute(reinterpret_cast<const void*>(route_block_kernel<T, D>),
                                   hipFuncAttributeMaxDynamicSharedMemorySize,
                                   static_cast<int>(sizeof(uint64_t) * kLdsPages));
    });
    if (e != hipSuccess) return e;
    route_block_kernel<T, D><<<grid_of(units, kThreads), kThreads, sizeof(uint64_t) * tok.max_pages, stream>>>(
        pool, tok, a, qt, q_stride, list);
    return hipGetLastError();
}

}  // namespace

// Bytes of a token's keys in the two-kernel form.
static int64_t token_key_bytes(const hga_plan& plan, int max_pages) {
    return static_cast<int64_t>(plan.p.n_kv_heads) * max_pages * static_cast<int64_t>(sizeof(uint64_t));
}

int64_t route_tokens_bytes(const hga_plan& plan, int n_tokens, int max_pages, bool must) {
    const int64_t units = static_cast<int64_t>(n_tokens) * plan.p.n_kv_heads;
    if (must ? max_pages <= kLdsPages : !few_and_long(plan, units, max_pages)) return 0;
    const int64_t one = token_key_bytes(plan, max_pages);
    return std::min<int64_t>(n_tokens, std::max<int64_t>(1, kKeyBytes / one)) * one;
}

hipError_t launch_route_tokens(const hga_plan& plan, const PoolView& pool, const TokensView& tok, const void* q,
                               int64_t q_stride, int32_t* list, int n_list, void* ws, int64_t ws_bytes,
                               hipStream_t stream) {
    RouteArgs a;
    a.first = plan.p.keep_first;
    a.window = recent_window(plan.p);
    a.topk = plan.p.topk_chunks;
    a.ratio = plan.p.n_q_heads / plan.p.n_kv_heads;
    a.n_list = n_list;
    const int64_t want = route_tokens_bytes(plan, tok.n_tokens, tok.max_pages, false);
    uint64_t* keys = want > 0 && ws_bytes >= want ? static_cast<uint64_t*>(ws) : nullptr;
    const bool f32 = plan.p.dtype == HGA_F32;
    const auto f = plan.p.head_dim == 128 ? (f32 ? run<float, 128> : run<bf16_t, 128>)
                                          : (f32 ? run<float, 64> : run<bf16_t, 64>);
    return f(plan, pool, tok, a, q, q_stride, list, keys, keys ? ws_bytes / token_key_bytes(plan, tok.max_pages) : 0,
             stream);
}

}  // namespace hga

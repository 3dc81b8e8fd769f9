// Actions drawn from logits [R, A] with temperature, top-k, min-p and top-p, one given uniform a row.
//
// All choices go by whole weights w_j = floor(2^31 exp((l_j - max) / T) + 1/2): their sums are exact in 64-bit integers,
// so the drawn action does not depend on how a row is split over threads, and every comparison of the filters is
// made between the same numbers on every run.
//
// The floor is one read of the logits (256 x 131072 bfloat16: 10 us).  An exact weight is about 24 instructions, of which expf is 9: 22 us
// of the 63 without filters, were they issued without a pause; with a cut the histograms are waited for (1.8 of 4 instructions a cycle).
// Measured: 1 x 131072 bfloat16 with top-k and top-p 14 us, 256 x 131072 without filters 63, top-k 50 54, top-p 0.9 182, mixed
// settings 117; 262144 x 18 fp32 without filters 14 (73 instructions a logit with the walks in shared memory).
#include <cooperative_groups.h>

#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_pair.cuh"
#include "rlcs_weights.cuh"

namespace {

using namespace rlcs_pair;
using namespace rlcs_rows;

constexpr int64_t kMostBlocks = (int64_t(1) << 31) - 1;

template <typename T> struct SampleParams {
    const T* logits;
    int64_t ld;
    const float* uniforms;
    const float* temperature;
    const int32_t* top_k;
    const float* top_p;
    const float* min_p;
    float temperature_all, top_p_all, min_p_all;
    int32_t top_k_all;
    int32_t* actions;
    float* log_probs;
    float* kept_log_probs;
    int64_t R;
    int A;
};

// Unsigned key in the order of the floats, and back.  bfloat16 values have 16 bits of key.
template <typename T> struct Key {
    static constexpr int kDown = sizeof(T) == 2 ? 16 : 0;
    static __device__ __forceinline__ uint32_t of(float f) {
        const uint32_t u = __float_as_uint(f);
        return (u ^ (((int32_t)u >> 31) | 0x80000000u)) >> kDown;
    }
    static __device__ __forceinline__ float value(uint32_t key) {
        const uint32_t u = key << kDown;
        return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~(u | (kDown ? 0xffffu : 0u)));
    }
};

// A row's settings, with the cases that leave one candidate folded into limit = 1.
struct Rules {
    float inv_t, p, low;
    int limit;
};

template <typename T> __device__ __forceinline__ Rules rules_of(const SampleParams<T>& P, int64_t row) {
    const float t = P.temperature != nullptr ? P.temperature[row] : P.temperature_all;
    const int k = P.top_k != nullptr ? P.top_k[row] : P.top_k_all;
    Rules r;
    r.p = P.top_p != nullptr ? P.top_p[row] : P.top_p_all;
    r.low = P.min_p != nullptr ? P.min_p[row] : P.min_p_all;
    const bool greedy = !(t > 0.f);
    r.inv_t = inverse_of(t);
    r.limit = k > 0 && k < P.A ? k : P.A;
    if (greedy || r.p <= 0.f || r.low > 1.f) r.limit = 1;
    if (!(r.low > 0.f) || r.low > 1.f) r.low = 0.f;
    if (!(r.p < 1.f)) r.p = 1.f;
    return r;
}

__device__ __forceinline__ uint32_t weight_at(float x, float m, const Rules& r) {
    const float e = expf(scaled(x, m, r.inv_t));
    return e >= r.low ? weight_of(e) : 0u;
}

// How many of equally weighted candidates stay when `above` lies before them: the least n with above + n w >= enough.
__device__ __forceinline__ int ties_until(double enough, u64 above, uint32_t w) {
    if (w == 0) return 1;
    int n = (int)((enough - (double)above) / (double)w);
    while (n > 0 && (double)(above + (u64)(n - 1) * w) >= enough) --n;
    while ((double)(above + (u64)n * w) < enough) ++n;
    return n;
}

// `all`: the softmax's sum, 1 for the most likely action
template <typename T>
__device__ __forceinline__ void write_row(const SampleParams<T>& P, int64_t row, int action, float x, float m, float inv_t, double all, u64 kept) {
    const double d = (double)scaled(x, m, inv_t);
    P.actions[row] = action;
    P.log_probs[row] = (float)(d - log(all));
    P.kept_log_probs[row] = (float)(d - log((double)kept * 0x1p-31));
}

template <typename T> __device__ __forceinline__ void write_none(const SampleParams<T>& P, int64_t row) {
    P.actions[row] = -1;
    P.log_probs[row] = -INFINITY;
    P.kept_log_probs[row] = -INFINITY;
}

// ---------------------------------------------------------------------------------------------- up to 64 actions
// One thread a row.  The block copies its rows to shared memory (coalesced; an odd row stride keeps the threads' walks
// in different banks); a thread then walks its row, and takes candidates one by one where there are filters.
constexpr int kSmallRows = 128, kSmallA = 64;

template <typename T>
__global__ void __launch_bounds__(kSmallRows) sample_small_kernel(const __grid_constant__ SampleParams<T> P, uint32_t a_mul) {
    extern __shared__ float tile[];
    const int A = P.A, stride = A | 1;
    const int64_t row0 = (int64_t)blockIdx.x * kSmallRows, row = row0 + threadIdx.x;
    const int rows = P.R - row0 < kSmallRows ? (int)(P.R - row0) : kSmallRows;
    const T* from = P.logits + row0 * P.ld;
    if (P.ld == A && A % 2 == 0 && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {      // whole vectors; neighbours of an even place share a row
        constexpr int N = Vec<T>::N;
#pragma unroll 4
        for (int i = threadIdx.x * N; i < rows * A - N + 1; i += kSmallRows * N) {
            float f[N];
            Vec<T>::unpack(*reinterpret_cast<const uint4*>(from + i), f);
#pragma unroll
            for (int k = 0; k < N; k += 2) {
                const int at = i + k + (int)__umulhi((uint32_t)(i + k), a_mul);
                tile[at] = clean(f[k]);
                tile[at + 1] = clean(f[k + 1]);
            }
        }
        for (int i = rows * A / N * N + threadIdx.x; i < rows * A; i += kSmallRows)
            tile[i + (int)__umulhi((uint32_t)i, a_mul)] = clean(Vec<T>::load(from + i));
    } else {
#pragma unroll 4
        for (int i = threadIdx.x; i < rows * A; i += kSmallRows) {
            const int r = a_mul != 0 ? (int)__umulhi((uint32_t)i, a_mul) : i, j = i - r * A;
            tile[r * stride + j] = clean(Vec<T>::load(from + r * P.ld + j));
        }
    }
    __syncthreads();
    if (row >= P.R) return;
    float* x = tile + threadIdx.x * stride;
    const Rules r = rules_of(P, row);
    float m = -INFINITY;
    for (int j = 0; j < A; ++j) m = fmaxf(m, x[j]);
    if (m == -INFINITY) return write_none(P, row);
    u64 all = 0, kept = 0, stay = 0;
    if (r.limit == A && r.p >= 1.f && r.low == 0.f) {          // no filter: the weights take the logits' places
#pragma unroll 2
        for (int j = 0; j < A; ++j) {
            const uint32_t w = weight_of(expf(scaled(x[j], m, r.inv_t)));
            x[j] = __uint_as_float(w);
            all += w;
        }
        const u64 target = target_of(P.uniforms[row], all);
        u64 sum = 0;
        int a = 0;
        for (; a < A - 1; ++a) {
            sum += __float_as_uint(x[a]);
            if (sum > target) break;
        }
        return write_row(P, row, a, clean(Vec<T>::load(from + threadIdx.x * P.ld + a)), m, r.inv_t, (double)all * 0x1p-31, all);
    }
    for (int j = 0; j < A; ++j) {
        const float e = expf(scaled(x[j], m, r.inv_t));
        const uint32_t w = weight_of(e);
        all += w;
        if (e >= r.low) { kept += w; stay |= 1ull << j; }
    }
    // the first candidate behind (value, index) in order
    auto next = [&](float v, int at, u64 among) {
        float best = -INFINITY;
        int where = -1;
        for (int j = 0; j < A; ++j)
            if ((among >> j & 1) && (x[j] < v || (x[j] == v && j > at)) && (where < 0 || x[j] > best)) { best = x[j]; where = j; }
        return where;
    };
    if (r.limit < A) {
        u64 some = 0;
        kept = 0;
        float v = INFINITY;
        int at = -1;
        for (int n = 0; n < r.limit; ++n) {
            at = next(v, at, ~0ull);
            v = x[at];
            if (!(stay >> at & 1)) continue;
            some |= 1ull << at;
            kept += weight_at(v, m, r);
        }
        stay = some;
    }
    if (r.p < 1.f && r.limit > 1) {
        const double enough = (double)r.p * (double)kept;
        u64 some = 0;
        kept = 0;
        float v = INFINITY;
        int at = -1;
        do {
            at = next(v, at, stay);
            v = x[at];
            some |= 1ull << at;
            kept += weight_at(v, m, r);
        } while ((double)kept < enough && some != stay);
        stay = some;
    }
    const u64 target = target_of(P.uniforms[row], kept);
    u64 sum = 0;
    for (int j = 0; j < A; ++j) {
        if (!(stay >> j & 1)) continue;
        sum += weight_at(x[j], m, r);
        if (sum > target) return write_row(P, row, j, x[j], m, r.inv_t, (double)all * 0x1p-31, kept);
    }
}

// ---------------------------------------------------------------------------------------------- up to 1024 actions
// A 64-bit sum over the warp of values below 2^40: two hardware sums.
__device__ __forceinline__ u64 redux_sum(u64 v) {
    return (u64)__reduce_add_sync(~0u, (uint32_t)v & 0xfffffu) + ((u64)__reduce_add_sync(~0u, (uint32_t)(v >> 20)) << 20);
}

// One warp a row, the row's keys and weights in registers (lane l holds elements l, l + 32, ...).  A cut is found bit by
// bit from the top: 32 (16) rounds of a comparison and an addition an element.
template <typename T, int PER>
__global__ void __launch_bounds__(256) sample_warp_kernel(const __grid_constant__ SampleParams<T> P) {
    typedef Key<T> K;
    const int lane = threadIdx.x & 31, A = P.A;
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    if (row >= P.R) return;
    const T* x = P.logits + row * P.ld;
    const Rules r = rules_of(P, row);
    uint32_t key[PER], w[PER];
    uint32_t top_key = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int j = i * 32 + lane;
        key[i] = j < A ? K::of(clean(Vec<T>::load(x + j))) : 0u;          // 0: below every logit
    }
#pragma unroll
    for (int i = 0; i < PER; ++i) top_key = max(top_key, key[i]);
    top_key = warp_max(top_key);
    const float m = K::value(top_key);
    if (m == -INFINITY) {
        if (lane == 0) write_none(P, row);
        return;
    }
    u64 all = 0, kept = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const float e = key[i] ? expf(scaled(K::value(key[i]), m, r.inv_t)) : 0.f;
        w[i] = weight_of(e);
        all += w[i];
        if (!(e >= r.low)) w[i] = 0;
        kept += w[i];
    }
    all = redux_sum(all);
    kept = r.low > 0.f ? redux_sum(kept) : all;
    uint32_t cut = 0;
    int ties = A;
    if (r.limit == 1) {
        cut = top_key;
        ties = 1;
        kept = 0x80000000u;
    } else if (r.limit < A) {
        for (int b = 31 - K::kDown; b >= 0; --b) {
            const uint32_t next = cut | (1u << b);
            int n = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) n += key[i] >= next;
            if (__reduce_add_sync(~0u, n) >= r.limit) cut = next;
        }
        int n = 0;
        kept = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            n += key[i] > cut;
            kept += key[i] > cut ? w[i] : 0u;
        }
        ties = r.limit - __reduce_add_sync(~0u, n);
        kept = redux_sum(kept) + (u64)ties * weight_at(K::value(cut), m, r);
    }
    if (r.p < 1.f && r.limit > 1) {
        const double enough = (double)r.p * (double)kept;
        uint32_t c = cut;                                        // everything from the cut up weighs enough
        for (int b = 31 - K::kDown; b >= 0; --b) {
            const uint32_t next = (c & ~((2u << b) - 1)) | (c & (1u << b)) | (1u << b);
            if (next <= c) continue;                             // the bit is set already
            u64 n = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) n += key[i] >= next ? w[i] : 0u;
            if ((double)redux_sum(n) >= enough) c = next;
        }
        u64 above = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) above += key[i] > c ? w[i] : 0u;
        above = redux_sum(above);
        const uint32_t at = weight_at(K::value(c), m, r);
        const int more = ties_until(enough, above, at);
        if (c > cut || more < ties) ties = more;
        cut = c;
        kept = above + (u64)ties * at;
    }
    const u64 target = target_of(P.uniforms[row], kept);
    u64 sum = 0;
    int seen = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const bool tied = key[i] == cut;
        const unsigned tie_lanes = __ballot_sync(~0u, tied);
        const bool in = key[i] > cut || (tied && seen + __popc(tie_lanes & ((1u << lane) - 1)) < ties);
        seen += __popc(tie_lanes);
        const u64 mine = in ? w[i] : 0u;
        const u64 step = redux_sum(mine);
        if (sum + step > target) {
            u64 run = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 v = __shfl_up_sync(~0u, run, o);
                run += lane >= o ? v : 0;
            }
            const unsigned past = __ballot_sync(~0u, sum + run > target);
            if (lane == __ffs(past) - 1) write_row(P, row, i * 32 + lane, K::value(key[i]), m, r.inv_t, (double)all * 0x1p-31, kept);
            return;
        }
        sum += step;
    }
}

// ---------------------------------------------------------------------------------------------- more actions
// One cluster of 1 to 8 blocks a row, each with a part of it that its passes find in L1 or L2 again; every warp has a
// contiguous range, so that sums in index order are sums over warps in order.
//   no cut (no top-k, no top-p):  maximum; weights by warp; one warp walks the range that holds the target.
//   top-k up to 192: the k-th largest of the threads' own maxima bounds the k-th largest logit from below, so that few
//     candidates pass it (about 200 of 131072 for k = 192 and 2048 threads); one block sorts them and does the rest.
//   otherwise a histogram of weights and counts over 24 steps of (l - max) / T, one column a lane and so without atomics (48 KB: four
//     blocks a multiprocessor, 117 us for 256 x 131072 with mixed settings; 32 steps and three blocks: 133),
//     finds the step that holds a cut; histograms over the keys of that step alone narrow it to one key.
constexpr int kT = 256, kW = kT / 32, kCoarse = 24, kFine = 1024, kList = 2048, kListLimit = 192, kMaxCluster = 8;
constexpr u64 kCountOne = 1ull << 48;                        // a column's entry: count above, weight below bit 48

struct Shared {
    union {
        u64 column[kW][kCoarse][32];
        struct {
            uint32_t count[kFine], low[kFine], high[kFine];      // weight in two words
        } fine;
        struct {
            u64 list[kList];                                 // (key, ~index)
            uint32_t maxima[kMaxCluster * kT];
            uint32_t digit[256];
        };
    };
    u64 trade[2][kW], near[kW];
    double whole[kW];                                        // each warp's part of sum_j e_j
    uint32_t trade_ties[2][kW], near_ties[kW];
    u64 coarse_weight[kCoarse];
    uint32_t coarse_count[kCoarse];
    u64 scan_weight[kW];
    uint32_t scan_count[kW];
    u64 found_weight;
    uint32_t found_count, found_bin, listed, bound;
};

struct Range {
    int v0, v1;                                              // vectors of the row
    bool head, tail;                                         // and the elements before the first, behind the last
};

// Where a target lies among parts in order: which part, and the weight and ties before it.
struct Located {
    int part;
    u64 before, total;
    uint32_t ties_before;
};

template <typename T> struct ClusterRow {
    typedef Key<T> K;
    const T* x;
    Shared& sh;
    int A, lane, warp, rank, ranks, turn;
    Span sp;
    Range mine;                                              // this warp's

    // Part `i` of `n` equal ones of a range: its vectors, and the single elements before and behind the row's if it is the
    // first or the last.
    static __device__ __forceinline__ Range part_of(const Range& r, int i, int n) {
        const int per = (r.v1 - r.v0 + n - 1) / n, at = min(r.v0 + i * per, r.v1);
        return Range{at, min(at + per, r.v1), r.head && i == 0, r.tail && i == n - 1};
    }
    __device__ __forceinline__ Range all() const { return Range{0, sp.vecs, true, true}; }
    __device__ __forceinline__ void sync() {
        if (ranks > 1) cooperative_groups::this_cluster().sync(); else __syncthreads();
    }
    __device__ __forceinline__ Shared& other(int rank_) {
        return ranks > 1 ? *cooperative_groups::this_cluster().map_shared_rank(&sh, rank_) : sh;
    }
    __device__ __forceinline__ int tail_at() const { return sp.head + sp.vecs * Vec<T>::N; }

    // f(logit, index) for every element of a range, four vectors of a lane in flight; places behind the range hold -inf.
    // Logits come as they are: NaN compares false and -0 equal to 0.  `then` is called after every vector.
    struct Nothing {
        __device__ __forceinline__ void operator()() const {}
    };
    template <typename F, typename G = Nothing> __device__ __forceinline__ void each(const Range& r, F f, G then = G()) const {
        constexpr int N = Vec<T>::N, kAhead = 4;
        const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
        const uint4 nothing = make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
        uint4 g[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) g[q] = r.v0 + lane + 32 * q < r.v1 ? __ldg(body + r.v0 + lane + 32 * q) : nothing;
#pragma unroll 1
        for (int v = r.v0 + lane; v - lane < r.v1; v += 32) {      // one copy of f's code a vector: the kernel has many such passes
            float e[N];
            Vec<T>::unpack(g[0], e);
#pragma unroll
            for (int q = 0; q + 1 < kAhead; ++q) g[q] = g[q + 1];
            g[kAhead - 1] = v + 32 * kAhead < r.v1 ? __ldg(body + v + 32 * kAhead) : nothing;
#pragma unroll
            for (int k = 0; k < N; ++k) f(e[k], sp.head + v * N + k);
            then();
        }
        const int singles = r.head ? sp.head : 0, ends = r.tail ? A - tail_at() : 0;
        if (lane < singles + ends) {
            const int j = lane < singles ? lane : tail_at() + lane - singles;
            f(Vec<T>::load(x + j), j);
            then();
        }
    }
    // The softmax's sum: parts left by every warp ahead of a barrier of the cluster, added up by a warp behind it.
    __device__ __forceinline__ void leave_whole(double part) {
        part = warp_sum(part);
        if (lane == 0) sh.whole[warp] = part;
    }
    __device__ __forceinline__ double whole() {
        double total = 0.;
        for (int i = lane; i < ranks * kW; i += 32) total += other(i / kW).whole[i % kW];
        return warp_sum(total);
    }
    // the largest logit of the lane's elements
    __device__ __forceinline__ float most() const {
        constexpr int kAhead = 8;
        uint32_t top = Vec<T>::kNothing;
        const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
        for (int v = mine.v0 + lane; v < mine.v1; v += 32 * kAhead) {
            uint4 g[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                g[q] = v + 32 * q < mine.v1 ? __ldg(body + v + 32 * q) : make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                top = Vec<T>::most_number(top, Vec<T>::most_number(Vec<T>::most_number(g[q].x, g[q].y), Vec<T>::most_number(g[q].z, g[q].w)));
        }
        float f = Vec<T>::most_number_of(top);
        if (mine.head && lane < sp.head) f = fmaxf(f, Vec<T>::load(x + lane));
        if (mine.tail && tail_at() + lane < A) f = fmaxf(f, Vec<T>::load(x + tail_at() + lane));
        return f + 0.f;
    }
    // over the cluster: the sum of all warps' values
    __device__ __forceinline__ u64 gather(u64 v) {
        v = warp_sum(v);
        turn ^= 1;
        if (lane == 0) sh.trade[turn][warp] = v;
        sync();
        u64 total = 0;
        for (int i = lane; i < ranks * kW; i += 32) total += other(i / kW).trade[turn][i % kW];
        return warp_sum(total);
    }
    __device__ __forceinline__ u64 gather_max(u64 v) {
        v = warp_max(v);
        turn ^= 1;
        if (lane == 0) sh.trade[turn][warp] = v;
        sync();
        u64 top = 0;
        for (int i = lane; i < ranks * kW; i += 32) { const u64 u = other(i / kW).trade[turn][i % kW]; top = u > top ? u : top; }
        return warp_max(top);
    }
    // Kept are all above the cut (their weights are in the parts' sums) and the first `ties` that equal it, of weight `each_tie`.
    // Parts in order, two a lane: which one holds the target, a share `uniform` of all kept weight (or that very target, where given).
    template <typename Entry>
    __device__ __forceinline__ Located locate(int n, Entry entry, u64 ties, uint32_t each_tie, float uniform, const u64* given) const {
        u64 w[2] = {0, 0};
        uint32_t t[2] = {0, 0};
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (2 * lane + h < n) entry(2 * lane + h, &w[h], &t[h]);
        uint32_t t_run = t[0] + t[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(~0u, t_run, o);
            t_run += lane >= o ? u : 0;
        }
        const uint32_t t0 = t_run - t[0] - t[1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const u64 at = h == 0 ? t0 : t0 + t[0], left = at < ties ? ties - at : 0;
            w[h] += (left < t[h] ? left : t[h]) * each_tie;
        }
        u64 run = w[0] + w[1];
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const u64 u = __shfl_up_sync(~0u, run, o);
            run += lane >= o ? u : 0;
        }
        Located r;
        r.total = __shfl_sync(~0u, run, 31);
        const u64 target = given != nullptr ? *given : target_of(uniform, r.total), before = run - w[0] - w[1];
        const unsigned past = __ballot_sync(~0u, run > target);
        const int src = past ? __ffs(past) - 1 : 31;
        const bool second = !(before + w[0] > target);
        r.part = 2 * src + __shfl_sync(~0u, (int)second, src);
        r.before = __shfl_sync(~0u, second ? before + w[0] : before, src);
        r.ties_before = __shfl_sync(~0u, second ? t0 + t[0] : t0, src);
        return r;
    }
    // A range in index order, by one warp: the element at which the running kept weight passes the target.
    template <typename F>
    __device__ __forceinline__ int walk(const Range& r, float cut, u64 ties, uint32_t each_tie, u64 target, F weight) const {
        constexpr int N = Vec<T>::N;
        int found = -1;
        u64 sum = 0, seen = 0;
        auto step = [&](const float* g, int n, int at) {     // n elements a lane, lane after lane
            u64 w = 0;
            uint32_t t = 0;
            u64 each_w[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                each_w[k] = k < n && g[k] > cut ? weight(g[k]) : 0u;
                w += each_w[k];
                t += k < n && g[k] == cut;
            }
            uint32_t t_run = t;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t u = __shfl_up_sync(~0u, t_run, o);
                t_run += lane >= o ? u : 0;
            }
            const u64 rank_ = seen + t_run - t, left = rank_ < ties ? ties - rank_ : 0;
            const u64 mine_ = w + (left < t ? left : t) * each_tie;
            u64 run = mine_;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const u64 u = __shfl_up_sync(~0u, run, o);
                run += lane >= o ? u : 0;
            }
            const unsigned past = __ballot_sync(~0u, sum + run > target);
            if (past) {
                u64 s_ = sum + run - mine_, q = rank_;
                int hit = -1;
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (k < n) {
                        s_ += each_w[k];
                        if (g[k] == cut && q++ < ties) s_ += each_tie;
                        if (hit < 0 && s_ > target) hit = at + k;
                    }
                found = __shfl_sync(~0u, hit, __ffs(past) - 1);
            }
            sum += __shfl_sync(~0u, run, 31);
            seen += __shfl_sync(~0u, t_run, 31);
        };
        const int singles = r.head ? sp.head : 0, ends = r.tail ? A - tail_at() : 0;
#pragma unroll 1
        for (int base = singles ? r.v0 - 32 : r.v0; base < (ends ? r.v1 + 32 : r.v1) && found < 0; base += 32) {
            // one step of the single elements before, steps of vectors, one of those behind
            float g[N];
            int n = 0, at = 0;
            if (base < r.v0) {
                at = lane;
                n = lane < singles;
            } else if (base < r.v1) {
                at = sp.head + (base + lane) * N;
                n = base + lane < r.v1 ? N : 0;
            } else {
                at = tail_at() + lane;
                n = lane < ends;
            }
#pragma unroll
            for (int k = 0; k < N; ++k) g[k] = -INFINITY;
            if (n == N) Vec<T>::unpack(__ldg(reinterpret_cast<const uint4*>(x + at)), g);
            else if (n == 1) g[0] = Vec<T>::load(x + at);
            step(g, n, at);
            if (base < r.v1 && base + 32 >= r.v1 && base >= r.v0) base = r.v1 - 32;      // the step behind the vectors starts at their end
        }
        return found;
    }
    // The action: the warps' sums (weights above the cut, ties) find the warp, its block's warps its part, one of them the element.
    // `done(element, kept weight)` is called by that warp.
    template <typename F, typename G>
    __device__ __forceinline__ void pick(u64 w, uint32_t t, float cut, u64 ties, uint32_t each_tie, float uniform, F weight, G done) {
        w = warp_sum(w);
        t = __reduce_add_sync(~0u, t);
        turn ^= 1;
        if (lane == 0) { sh.trade[turn][warp] = w; sh.trade_ties[turn][warp] = t; }
        sync();
        const int trade_turn = turn;
        const Located far = locate(ranks * kW, [&](int i, u64* ew, uint32_t* et) {
            Shared& o = other(i / kW);
            *ew = o.trade[trade_turn][i % kW];
            *et = o.trade_ties[trade_turn][i % kW];
        }, ties, each_tie, uniform, nullptr);
        if (far.part / kW != rank) return;
        u64 target = target_of(uniform, far.total) - far.before;
        ties = far.ties_before < ties ? ties - far.ties_before : 0;
        const Range near = part_of(part_of(all(), far.part, ranks * kW), warp, kW);
        w = 0;
        t = 0;
        each(near, [&](float f, int) {
            if (f > cut) w += weight(f);
            t += f == cut;
        });
        w = warp_sum(w);
        t = __reduce_add_sync(~0u, t);
        if (lane == 0) { sh.near[warp] = w; sh.near_ties[warp] = t; }
        __syncthreads();
        const Located here = locate(kW, [&](int i, u64* ew, uint32_t* et) { *ew = sh.near[i]; *et = sh.near_ties[i]; }, ties, each_tie, 0.f, &target);
        if (here.part != warp) return;
        const int a = walk(near, cut, here.ties_before < ties ? ties - here.ties_before : 0, each_tie, target - here.before, weight);
        if (a >= 0) done(a, far.total);
    }
};

// A cut being narrowed: keys in [lo, hi] hold it; `above` sums what lies over hi.
struct Cut {
    uint32_t lo, hi, above_count;
    u64 above_weight;
};

template <typename T>
__global__ void __launch_bounds__(kT, 4) sample_cluster_kernel(const __grid_constant__ SampleParams<T> P) {
    typedef Key<T> K;
    extern __shared__ __align__(16) char raw[];
    Shared& sh = *reinterpret_cast<Shared*>(raw);
    const int ranks = (int)cooperative_groups::this_cluster().num_blocks(), rank = (int)cooperative_groups::this_cluster().block_rank();
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t row = blockIdx.x / ranks;
    const T* x = P.logits + row * P.ld;
    ClusterRow<T> row_ = {x, sh, P.A, lane, warp, rank, ranks, 0, span_of(x, P.A), {0, 0, false, false}};
    row_.mine = row_.part_of(row_.all(), rank * kW + warp, ranks * kW);
    const Rules r = rules_of(P, row);

    const uint32_t my_top = K::of(row_.most()), top_key = (uint32_t)row_.gather_max(my_top);
    const float m = K::value(top_key);
    const float exp2_t = fminf(r.inv_t * 1.4426950408889634f, 3.4028235e38f);
    // For a finite m.  A quick exponential where only its sum's logarithm counts (ex2.approx: 2^-22), not a choice;
    // far below the maximum, -inf and NaN: 0.
    // That sum: a vector's terms in 32 bits, vectors in 64.  In 32 bits the thousands of terms that a thread may have would
    // lose 1e-5 and more of it where their roundings have one sign; and the whole weights leave out what lies below 2^-32 of the
    // most likely action, a million of which hold 1e-4.
    auto quick = [&](float f) { return exp2_of(fmaxf((f - m) * exp2_t, -1000.f)); };
    auto relative = [&](float f) { return fmaxf((f - m) * r.inv_t, -1000.f); };
    auto weight = [&](float f) {
        const float e = expf(relative(f));
        return e >= r.low ? weight_of(e) : 0u;
    };
    float some = 0.f;                                        // of the vector's terms
    double part = 0.;
    auto vector_done = [&] { part += (double)some; some = 0.f; };
    const float uniform = P.uniforms[row];
    auto done = [&](int a, u64 kept) {
        const double all = row_.whole();
        if (lane == 0) write_row(P, row, a, clean(Vec<T>::load(x + a)), m, r.inv_t, all, kept);
    };

    if (m == -INFINITY) {
        if (rank == 0 && tid == 0) write_none(P, row);
    } else if (m == INFINITY) {                              // the infinite ones share the probability
        uint32_t mine = 0;
        row_.each(row_.mine, [&](float f, int) { mine += f == m; });
        row_.leave_whole((double)mine);
        const u64 there = row_.gather(mine);
        u64 ties = min(there, (u64)r.limit);
        if (r.p < 1.f) ties = min(ties, (u64)ties_until((double)r.p * (double)(ties << 31), 0, 0x80000000u));
        row_.pick(0, mine, m, ties, 0x80000000u, uniform, weight, done);
    } else if (r.limit == 1) {
        uint32_t first = 0;                                  // ~index, so that the lowest wins
        row_.each(row_.mine, [&](float f, int j) {
            some += quick(f);
            if (f == m) first = max(first, ~(uint32_t)j);
        }, vector_done);
        row_.leave_whole(part);
        const int a = (int)~(uint32_t)row_.gather_max(first);
        if (rank == 0 && warp == 0) {
            const double all = row_.whole();
            if (lane == 0) write_row(P, row, a, m, m, r.inv_t, all, 0x80000000ull);
        }
    } else if (r.limit == P.A && r.p >= 1.f) {
        u64 mine = 0;
        if (r.low > 0.f) {
            row_.each(row_.mine, [&](float f, int) {
                const float e = expf(relative(f));
                some += e;
                mine += e >= r.low ? weight_of(e) : 0u;
            }, vector_done);
        } else {
            row_.each(row_.mine, [&](float f, int) {
                const float e = expf(relative(f));
                some += e;
                mine += weight_of(e);
            }, vector_done);
        }
        row_.leave_whole(part);
        row_.pick(mine, 0, -INFINITY, 0, 0, uniform, weight, done);
    } else {
        bool listed_all = false;
        if (r.limit <= kListLimit) {
            Shared& lead = row_.other(0);
            lead.maxima[rank * kT + tid] = my_top;
            if (rank == 0 && tid == 0) sh.listed = 0;
            row_.sync();
            if (rank == 0) {
                // the limit-th largest of the maxima, its upper 16 bits
                uint32_t prefix = 0, want = r.limit;
                constexpr int kTop = 32 - K::kDown;
                for (int round = 0; round < 2; ++round) {
                    const int shift = kTop - 8 * (round + 1);
                    sh.digit[tid] = 0;
                    __syncthreads();
                    for (int i = tid; i < ranks * kT; i += kT)
                        if (round == 0 || sh.maxima[i] >> (shift + 8) == prefix) atomicAdd(&sh.digit[(sh.maxima[i] >> shift) & 255], 1u);
                    __syncthreads();
                    if (warp == 0) {                         // lane l: digits 255 - 8l down to 248 - 8l
                        uint32_t n[8], sum = 0;
                        for (int k = 0; k < 8; ++k) sum += n[k] = sh.digit[255 - 8 * lane - k];
                        uint32_t run = sum;
                        for (int o = 1; o < 32; o <<= 1) {
                            const uint32_t u = __shfl_up_sync(~0u, run, o);
                            run += lane >= o ? u : 0;
                        }
                        if (run >= want && run - sum < want) {
                            uint32_t s = run - sum;
                            int k = 0;
                            while (s + n[k] < want) s += n[k++];
                            sh.found_bin = prefix << 8 | (255 - 8 * lane - k);
                            sh.found_count = want - s;
                        }
                    }
                    __syncthreads();
                    prefix = sh.found_bin;
                    want = sh.found_count;
                }
                if (tid == 0) sh.bound = prefix << (kTop - 16);
            }
            row_.sync();
            const float bound = K::value(max(lead.bound, K::of(-INFINITY)));
            row_.each(row_.mine, [&](float f, int j) {
                some += quick(f);
                if (f >= bound && j < P.A) {
                    const uint32_t at = atomicAdd(&lead.listed, 1u);
                    if (at < kList) lead.list[at] = (u64)K::of(f + 0.f) << 32 | ~(uint32_t)j;
                }
            }, vector_done);
            row_.leave_whole(part);
            part = 0.;
            row_.sync();                                     // the list and the sum are complete
            const uint32_t listed = lead.listed;
            listed_all = listed <= kList;
            row_.sync();                                     // read by all before the room is used again
            if (listed_all && rank == 0) {
                const double all = row_.whole();
                int size = 32;
                while (size < (int)listed) size *= 2;
                for (int i = tid; i < size; i += kT) if (i >= (int)listed) sh.list[i] = 0;
                __syncthreads();
                for (int k = 2; k <= size; k *= 2)
                    for (int j = k / 2; j > 0; j /= 2) {
                        for (int i = tid; i < size / 2; i += kT) {
                            const int a = 2 * i - (i & (j - 1)), b = a + j;
                            const u64 u = sh.list[a], v = sh.list[b];
                            if ((u < v) == ((a & k) == 0)) { sh.list[a] = v; sh.list[b] = u; }
                        }
                        __syncthreads();
                    }
                // fewer than the limit where the rest of the row is NaN
                const int candidates = min(r.limit, (int)listed);
                const u64 entry = tid < candidates ? sh.list[tid] : 0;
                const int index = (int)~(uint32_t)entry;
                const float f = K::value((uint32_t)(entry >> 32));
                uint32_t w = tid < candidates ? weight(f) : 0u;
                u64 run = w;
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 u = __shfl_up_sync(~0u, run, o);
                    run += lane >= o ? u : 0;
                }
                if (lane == 31) sh.scan_weight[warp] = run;
                __syncthreads();
                u64 total = 0, ahead = 0;
                for (int k = 0; k < kW; ++k) { if (k < warp) ahead += sh.scan_weight[k]; total += sh.scan_weight[k]; }
                const double enough = (double)r.p * (double)total;
                if (r.p < 1.f && tid > 0 && !((double)(ahead + run - w) < enough)) w = 0;
                __syncthreads();
                sh.list[tid] = (u64)w;                       // weights and indices of the kept, in order
                sh.maxima[tid] = (uint32_t)index;
                const u64 part_kept = warp_sum((u64)w);
                if (lane == 0) sh.scan_weight[warp] = part_kept;
                __syncthreads();
                u64 kept = 0;
                for (int k = 0; k < kW; ++k) kept += sh.scan_weight[k];
                const u64 target = target_of(uniform, kept);
                if (w != 0) {
                    u64 upto = 0;
                    for (int k = 0; k < candidates; ++k) upto += sh.maxima[k] <= (uint32_t)index ? sh.list[k] : 0;
                    if (upto > target && upto - w <= target) write_row(P, row, index, f, m, r.inv_t, all, kept);
                }
            }
        }
        if (!listed_all) {
            constexpr float kSteps = kCoarse / 22.25f;       // weights are 0 from 22.18 below the maximum on
            auto bin_of = [&](float f) { return min((int)(relative(f) * -kSteps), kCoarse - 1); };
            for (int i = tid; i < kW * kCoarse * 32; i += kT) (&sh.column[0][0][0])[i] = 0;
            __syncthreads();
            u64* column = &sh.column[warp][0][lane];
            row_.each(row_.mine, [&](float f, int) {
                const float d = relative(f), e = expf(d);
                const uint32_t w = weight_of(e);
                some += e;
                if (w != 0) column[min((int)(d * -kSteps), kCoarse - 1) * 32] += kCountOne + (e >= r.low ? w : 0u);
            }, vector_done);
            row_.leave_whole(part);
            __syncthreads();
            for (int b = warp; b < kCoarse; b += kW) {
                u64 w = 0;
                uint32_t n = 0;
                for (int k = 0; k < kW; ++k) { const u64 u = sh.column[k][b][lane]; w += u & (kCountOne - 1); n += (uint32_t)(u >> 48); }
                w = warp_sum(w);
                n = warp_sum(n);
                if (lane == 0) { sh.coarse_weight[b] = w; sh.coarse_count[b] = n; }
            }
            row_.sync();
            u64 bin_weight = 0, to_weight;                   // lane = step: its own, and up to and with it
            uint32_t bin_count = 0, to_count;
            for (int k = 0; k < ranks && lane < kCoarse; ++k) { bin_weight += row_.other(k).coarse_weight[lane]; bin_count += row_.other(k).coarse_count[lane]; }
            to_weight = bin_weight;
            to_count = bin_count;
            for (int o = 1; o < 32; o <<= 1) {
                const u64 u = __shfl_up_sync(~0u, to_weight, o);
                const uint32_t n = __shfl_up_sync(~0u, to_count, o);
                if (lane >= o) { to_weight += u; to_count += n; }
            }
            const u64 weighed = __shfl_sync(~0u, to_weight, 31);
            const uint32_t counted = __shfl_sync(~0u, to_count, 31);
            // the cut where `want` candidates, or `enough` weight, are reached: first the step, then its keys by histograms
            auto narrow = [&](bool by_count, uint32_t want, double enough) {
                auto reached = [&](uint32_t n, u64 w) { return by_count ? n >= want : (double)w >= enough; };
                const int b = __ffs(__ballot_sync(~0u, reached(to_count, to_weight))) - 1;
                Cut c;
                c.above_weight = __shfl_sync(~0u, to_weight - bin_weight, b);
                c.above_count = __shfl_sync(~0u, to_count - bin_count, b);
                auto least_key = [&](auto holds) {           // the least key for which it holds (as for all above), 32 tried at once
                    uint32_t lo = K::of(-INFINITY), hi = top_key;
                    while (lo < hi) {
                        const uint32_t step = (hi - lo + 31) / 32, at = min(lo + lane * step, hi);
                        const unsigned yes = __ballot_sync(~0u, holds(K::value(at)));
                        const int first = yes ? __ffs(yes) - 1 : 32;
                        const uint32_t from = lo;
                        if (first < 32) hi = min(from + first * step, hi);
                        if (first > 0) lo = min(from + (first - 1) * step + 1, hi);
                        else hi = lo;
                    }
                    return lo;
                };
                // the last step also takes all that weighs nothing, which 16-bit keys, counted without their weights, must leave out
                c.lo = b == kCoarse - 1 ? least_key([&](float f) { return weight_of(expf(relative(f))) != 0; })
                                        : least_key([&](float f) { return bin_of(f) <= b; });
                c.hi = b == 0 ? top_key : least_key([&](float f) { return bin_of(f) <= b - 1; }) - 1;
                while (c.lo < c.hi) {
                    int shift = 0;
                    while ((c.hi - c.lo) >> shift >= kFine) ++shift;
                    row_.sync();                             // the room, and what others still read there
                    for (int i = tid; i < kFine; i += kT) { sh.fine.count[i] = 0; sh.fine.low[i] = 0; sh.fine.high[i] = 0; }
                    __syncthreads();
                    const float low_f = K::value(c.lo), high_f = K::value(c.hi);
                    row_.each(row_.mine, [&](float f, int) {
                        if (!(f >= low_f && f <= high_f)) return;
                        const uint32_t k = K::of(f + 0.f);
                        if (k < c.lo || k > c.hi) return;    // 0 and -0 compare equal
                        if (K::kDown && shift == 0) {
                            atomicAdd(&sh.fine.count[c.hi - k], 1u);
                            return;
                        }
                        const float e = expf(relative(f));
                        const uint32_t w = weight_of(e);
                        if (w == 0) return;
                        const uint32_t at = (c.hi - k) >> shift;
                        atomicAdd(&sh.fine.count[at], 1u);
                        if (shift > 0 && e >= r.low) {       // places of one key: their count gives their weight
                            const uint32_t was = atomicAdd(&sh.fine.low[at], w);
                            if (was + w < was) atomicAdd(&sh.fine.high[at], 1u);
                        }
                    });
                    row_.sync();
                    // every block adds up a stretch of the places over the cluster; the stretches' sums say which one holds the
                    // cut, and its block tells the others
                    const int stretch = kFine / ranks, per = stretch < kT ? 1 : stretch / kT, first = rank * stretch + tid * per;
                    u64 w[kFine / kT], sum_w = 0;
                    uint32_t n[kFine / kT], sum_n = 0;
#pragma unroll
                    for (int k = 0; k < kFine / kT; ++k) {
                        w[k] = 0;
                        n[k] = 0;
                        if (k >= per || tid * per >= stretch) continue;
                        for (int q = 0; q < ranks; ++q) {
                            const Shared& o = row_.other(q);
                            n[k] += o.fine.count[first + k];
                            if (shift > 0) w[k] += (u64)o.fine.high[first + k] << 32 | o.fine.low[first + k];
                        }
                        if (shift == 0 && n[k] != 0) w[k] = (u64)n[k] * weight(K::value(c.hi - (first + k)));
                        sum_w += w[k];
                        sum_n += n[k];
                    }
                    u64 run_w = sum_w;
                    uint32_t run_n = sum_n;
                    for (int o = 1; o < 32; o <<= 1) {
                        const u64 u = __shfl_up_sync(~0u, run_w, o);
                        const uint32_t v = __shfl_up_sync(~0u, run_n, o);
                        if (lane >= o) { run_w += u; run_n += v; }
                    }
                    row_.turn ^= 1;
                    if (lane == 31) { sh.trade[row_.turn][warp] = run_w; sh.trade_ties[row_.turn][warp] = run_n; }
                    row_.sync();
                    u64 aw = c.above_weight;
                    uint32_t an = c.above_count;
                    for (int k = 0; k < rank * kW + warp; ++k) {
                        const Shared& o = row_.other(k / kW);
                        aw += o.trade[row_.turn][k % kW];
                        an += o.trade_ties[row_.turn][k % kW];
                    }
                    aw += run_w - sum_w;
                    an += run_n - sum_n;
                    if (!reached(an, aw) && reached(an + sum_n, aw + sum_w)) {
                        int k = 0;
                        while (k < per - 1 && !reached(an + n[k], aw + w[k])) { an += n[k]; aw += w[k]; ++k; }
                        for (int q = 0; q < ranks; ++q) {
                            Shared& o = row_.other(q);
                            o.found_bin = first + k;
                            o.found_weight = aw;
                            o.found_count = an;
                        }
                    }
                    row_.sync();
                    c.above_weight = sh.found_weight;
                    c.above_count = sh.found_count;
                    c.hi -= sh.found_bin << shift;
                    const uint32_t width = (1u << shift) - 1;
                    c.lo = c.hi - c.lo > width ? c.hi - width : c.lo;
                }
                return c;
            };
            uint32_t cut = K::of(-INFINITY);                 // nothing cut: -inf weighs 0
            u64 ties = 0, kept = weighed;
            if ((uint32_t)r.limit < counted) {
                const Cut c = narrow(true, r.limit, 0.);
                cut = c.lo;
                ties = r.limit - c.above_count;
                kept = c.above_weight + ties * weight(K::value(cut));
            }
            if (r.p < 1.f) {
                const double enough = (double)r.p * (double)kept;
                const Cut c = narrow(false, 0, enough);
                const u64 more = (u64)ties_until(enough, c.above_weight, weight(K::value(c.lo)));
                if (c.lo > cut || more < ties) ties = more;
                cut = c.lo;
            }
            const float cut_f = K::value(cut);
            u64 mine = 0;
            uint32_t tied = 0;
            row_.each(row_.mine, [&](float f, int) {
                if (f > cut_f) mine += weight(f);
                tied += f == cut_f;
            });
            row_.pick(mine, tied, cut_f, ties, weight(cut_f), uniform, weight, done);
        }
    }
    row_.sync();                                             // no block ends while another may read its memory
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T>
int sample_run(const SampleParams<T>& P, int64_t A, void* stream) {
    if (P.R < 0 || A < 0 || A > (int64_t(1) << 22) || P.R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (P.R == 0) return RLCS_OK;
    if (A == 0 || P.ld < A || P.ld > (int64_t(1) << 40) / P.R) return RLCS_ERR_SIZE;
    if (P.temperature_all != P.temperature_all || P.top_p_all != P.top_p_all || P.min_p_all != P.min_p_all) return RLCS_ERR_ARG;
    if (P.logits == nullptr || P.uniforms == nullptr || P.actions == nullptr || P.log_probs == nullptr || P.kept_log_probs == nullptr)
        return RLCS_ERR_NULL;
    const void* words[] = {P.uniforms, P.temperature, P.top_k, P.top_p, P.min_p, P.actions, P.log_probs, P.kept_log_probs};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(P.logits, sizeof(T))) return RLCS_ERR_ALIGN;
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t warps = (P.R + 7) / 8;
    if (A <= kSmallA) {
        const int64_t blocks = (P.R + kSmallRows - 1) / kSmallRows;
        if (blocks > kMostBlocks) return RLCS_ERR_SIZE;
        const uint32_t mul = A > 1 ? (uint32_t)(((uint64_t(1) << 32) + A - 1) / A) : 0;
        sample_small_kernel<T><<<(unsigned)blocks, kSmallRows, kSmallRows * (A | 1) * sizeof(float), s>>>(P, mul);
    } else if (A <= 2048) {
        if (warps > kMostBlocks) return RLCS_ERR_SIZE;
        if (A <= 128) sample_warp_kernel<T, 4><<<(unsigned)warps, 256, 0, s>>>(P);
        else if (A <= 256) sample_warp_kernel<T, 8><<<(unsigned)warps, 256, 0, s>>>(P);
        else if (A <= 512) sample_warp_kernel<T, 16><<<(unsigned)warps, 256, 0, s>>>(P);
        else if (A <= 1024) sample_warp_kernel<T, 32><<<(unsigned)warps, 256, 0, s>>>(P);
        else sample_warp_kernel<T, 64><<<(unsigned)warps, 256, 0, s>>>(P);
    } else {
        // blocks a row: until the GPU has four a multiprocessor (256 x 131072 with mixed settings: 4 blocks a row 117 us, 2 173, 8 123; without
        // filters 63, 66, 71), or a part would fall below 4096 actions
        int ranks = 1;
        while (ranks < kMaxCluster && P.R * ranks < 4 * rlcs_device::limits().sms && A / (2 * ranks) >= 4096) ranks *= 2;
        if (P.R * ranks > kMostBlocks) return RLCS_ERR_SIZE;
        static bool granted[64];                             // room beyond 48 KB of shared memory, asked for once a device
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RLCS_ERR_CUDA;
        if (!granted[dev])
            granted[dev] = cudaFuncSetAttribute(sample_cluster_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Shared)) == cudaSuccess;
        if (!granted[dev]) return RLCS_ERR_CUDA;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(P.R * ranks));
        cfg.blockDim = dim3(kT);
        cfg.dynamicSmemBytes = sizeof(Shared);
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = ranks;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, sample_cluster_kernel<T>, P) != cudaSuccess) return RLCS_ERR_CUDA;
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_sample_actions(const float* logits, int64_t ld, const float* uniforms, const float* temperature, const int32_t* top_k,
                        const float* top_p, const float* min_p, float temperature_all, int32_t top_k_all, float top_p_all,
                        float min_p_all, int32_t* actions, float* log_probs, float* kept_log_probs, int64_t R, int64_t A,
                        void* cuda_stream) {
    return sample_run<float>({logits, ld, uniforms, temperature, top_k, top_p, min_p, temperature_all, top_p_all, min_p_all, top_k_all,
                              actions, log_probs, kept_log_probs, R, (int)A}, A, cuda_stream);
}

int rlcs_sample_actions_bf16(const uint16_t* logits, int64_t ld, const float* uniforms, const float* temperature,
                             const int32_t* top_k, const float* top_p, const float* min_p, float temperature_all, int32_t top_k_all,
                             float top_p_all, float min_p_all, int32_t* actions, float* log_probs, float* kept_log_probs, int64_t R,
                             int64_t A, void* cuda_stream) {
    return sample_run<bf16>({reinterpret_cast<const bf16*>(logits), ld, uniforms, temperature, top_k, top_p, min_p, temperature_all,
                             top_p_all, min_p_all, top_k_all, actions, log_probs, kept_log_probs, R, (int)A}, A, cuda_stream);
}

}  // extern "C"

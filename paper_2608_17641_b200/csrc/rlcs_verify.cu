// Drafted tokens kept or turned down against the target's probabilities, from given uniforms.
//
//   p, q: softmax of the target's and the draft policy's logits at the trajectory's temperature; x_i the i-th draft
//   x_i stays while u_i q_i(x_i) < p_i(x_i);  at the first that does not, the next token is drawn from max(0, p_i - q_i), and
//   after the last draft from p.  What is kept and drawn is then distributed as the target's own samples are.
//
// All choices go by whole weights w_j = floor(2^31 exp((l_j - max) / T) + 1/2), as action sampling's do: their sums are exact, so that
// neither verdict nor draw depends on how a row is split over threads.  A difference of two distributions is taken in units of
// 2^-40: floor(w_j P) - floor(v_j Q) with P = 2^40 / W, Q = 2^40 / V and the products rounded to 64-bit floats: a multiplication an entry instead of a
// division, and the same whole numbers in any program that rounds there.
//
// Two kernels.  The first reads every row once, at the rate of the memory, and leaves its maximum and the sum of its exponentials
// (the hardware's, summed in fp32 over 32 and in 64 bits beyond: within 2^-15 of the whole weights' sum, but for a weight an entry; derived below).  The
// second has a cluster a trajectory.  A draft whose verdict is the same anywhere within those bounds, nearly every one, needs no
// more; another row's weights are summed up exactly, and so are those of the row from which the next token is drawn.
//
// Measured: 128 trajectories of up to 7 drafts, 131072 entries in bfloat16, 132 us: 55 in the first kernel (0.75 of the copy bandwidth), in the
// second 26 for exact weights (18 instructions each, expf's among them), 10 for their differences and 42 of waiting: five rounds of
// clusters, each with a verdict and two sums over the cluster.  One trajectory: 18 us (7 + 11).  Not kept: exact weights of every row (585 us);
// clusters of eight with twice the share (168), 256 threads a block (137), 512 (137; kept where clusters do not queue: 384 make one
// trajectory's 20 us), dependent launch of the second kernel (0.4 us).
#include <cooperative_groups.h>

#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_pair.cuh"
#include "rlcs_weights.cuh"

namespace {

namespace cg = cooperative_groups;
using namespace rlcs_pair;
using namespace rlcs_rows;

constexpr double kShareOne = 0x1p40;      // a probability of 1 in a difference

// A part of a row of logits: its maximum, the first place that has it, the sum of exp((l - top) / T).
struct PartStat {
    double all;
    float top;
    int32_t best;
};

template <typename T> struct VerifyParams {
    const T* logits;
    const T* drafts;
    const int32_t* tokens;
    const int32_t* offsets;
    const float* uniforms;
    const float* draw_uniforms;
    const float* temperature;
    float temperature_all;
    int32_t* out;
    float* log_probs;
    int32_t* accepted;
    PartStat* stats;                      // [2][rows][parts]: of the target's rows, of the draft policy's
    float* picked;                        // [2][rows]: the draft's logit
    int64_t ld, ldd;
    int32_t rows, seqs, A, parts;
    int32_t share;                        // entries of a row that a block of the second kernel has
};

template <typename T> __device__ __forceinline__ float temperature_of(const VerifyParams<T>& P, int b) {
    return P.temperature != nullptr ? P.temperature[b] : P.temperature_all;
}

// exp((x - top) / T) as the weights are made of it; NaN, and what an infinite temperature makes of -inf, count nothing.
__device__ __forceinline__ float e_of(float x, float top, float inv) {
    const float e = expf(scaled(clean(x), top, inv));
    return e >= 0.f ? e : 0.f;
}

// The trajectory that row t belongs to, by a whole warp; -1 where there is none.  [begin, end): its rows.
template <typename T> __device__ __forceinline__ int seq_of(const VerifyParams<T>& P, int t, int lane, int* begin, int* end) {
    int lo = 0, n = P.seqs;                                  // the last trajectory that starts at or before t
    while (n > 1) {
        const int step = (n + 31) / 32, at = lo + lane * step;
        const unsigned some = __ballot_sync(~0u, lane * step < n && P.offsets[at] <= t);
        const int last = some == 0 ? 0 : 31 - __clz(some);
        n = min(step, n - last * step);
        lo += last * step;
    }
    *begin = max(P.offsets[lo], 0);
    *end = min(P.offsets[lo + 1], P.rows);
    return t >= *begin && t < *end ? lo : -1;
}

// ---------------------------------------------------------------------------------------------- every row once
// G threads a row (a warp, eight rows a block; or the block), which may be one of P.parts of it.
constexpr int kScan = 256, kAhead = 4;       // threads; 16-byte vectors of a row that a thread has at a time

// How far off a row's sum S = sum 2^-d_j may be, d_j = (max l - l_j) log2(e) / T.  A thread's base follows its maximum only when it is kBehind
// binary places behind: if it followed every time, a rising row would be rescaled by up to 1024 approximations in a row, whose errors add up.  An
// entry's exponential is a product of at most 3 + (d + 8) / 8 of the hardware's (2^-22 each): its own, one for each time that the base moved on, the
// thread's join and the part's.  Their exponents add up to d in pieces of at most d + 16 in all, each rounded five times (1 / T, log2(e) / T with its constant, difference, product:
// 4.5 * 2^-24 of it).  The mean of d over the row's probabilities is at most log2 A <= 22, so that the sum is off by
//   ln 2 (22 + 16) 4.5 * 2^-24 + (3 + 30 / 8) 2^-22  and  10 * 2^-24 of the fp32 sums of 32,  together 39 * 2^-22 = 9.2e-6 of itself:
// below the 1e-5 of log-probabilities.  The whole weights come from expf (2^-23) of an argument rounded twice, another 4 * 2^-22, and half a
// weight an entry: 43 * 2^-22 < 2^-15 and A / 2; entries beyond d = 32, whose share may be off by more, weigh nothing and are within the other A / 2.
constexpr float kBehind = 8.f;

template <typename T, int G>
__global__ void __launch_bounds__(kScan) verify_scan_kernel(const __grid_constant__ VerifyParams<T> P) {
    constexpr int N = Vec<T>::N;
    __shared__ double sums[kScan / 32];
    __shared__ float tops[kScan / 32];
    __shared__ int bests[kScan / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, me = tid % G;
    const int64_t item = G == 32 ? (int64_t)blockIdx.x * (kScan / 32) + warp : blockIdx.x;
    const int part = (int)(item % P.parts);
    const int64_t row = item / P.parts;
    const int which = row >= P.rows ? 1 : 0, t = (int)(row - (which ? P.rows : 0));
    if (t >= P.rows || (which == 1 && P.drafts == nullptr)) return;      // warps of the last block
    int begin, end;
    const int b = seq_of(P, t, lane, &begin, &end);
    const float temperature = b >= 0 ? temperature_of(P, b) : 0.f;
    if (b < 0 || (which == 1 && (t + 1 == end || !(temperature > 0.f)))) return;
    const float inv = inverse_of(temperature), k = inv * 1.4426950408889634f;
    const T* x = which ? P.drafts + t * P.ldd : P.logits + t * P.ld;
    const Span sp = span_of(x, P.A);
    const int per = (sp.vecs + P.parts - 1) / P.parts, v0 = min(part * per, sp.vecs), n = min(per, sp.vecs - v0);
    const int rest = sp.head + sp.vecs * N, singles = part == 0 ? sp.head + P.A - rest : 0;      // before and behind the vectors
    const uint4* body = reinterpret_cast<const uint4*>(x + sp.head) + v0;
    auto single = [&](int i) { return i < sp.head ? i : rest + i - sp.head; };

    float picked = -INFINITY;
    if (part == 0 && me == 0 && t + 1 < end) {
        const int token = P.tokens[t + 1];
        if (token >= 0 && token < P.A) picked = clean(Vec<T>::load(x + token));
    }
    float m = -INFINITY, base = -INFINITY;                   // the thread's maximum, and what its sum is relative to
    double all = 0.;
    int chunk = -1;                                          // where the thread's maximum came first: a chunk of vectors, or -2 - a single
    auto follow = [&] {
        if ((m - base) * k <= kBehind) return;
        all = base == -INFINITY ? 0. : all * (double)exp2_of((base - m) * k);
        base = m;
    };
    for (int i = me; i < singles; i += G) {
        const float f = Vec<T>::load(x + single(i));
        if (f > m) {
            m = f;
            chunk = -2 - i;
            follow();
        }
        if (m != -INFINITY) all += (double)exp2_of((f - base) * k);
    }
    auto take = [&](int c, auto whole) {
        uint4 v[kAhead];
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            const int i = (c * kAhead + q) * G + me;
            v[q] = whole() || i < n ? __ldcs(body + i) : make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
        }
        uint32_t most = Vec<T>::kNothing;
#pragma unroll
        for (int q = 0; q < kAhead; ++q)
            most = Vec<T>::most_number(most, Vec<T>::most_number(Vec<T>::most_number(v[q].x, v[q].y), Vec<T>::most_number(v[q].z, v[q].w)));
        const float top = Vec<T>::most_number_of(most);
        if (top > m || (top == m && chunk < -1)) {           // of equals a vector's place, unless a single's comes before: below
            m = top;
            chunk = c;
            follow();
        }
        if (m == -INFINITY) return;
        const float2 less = {-base, -base}, scale = {k, k};
        float2 s[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
        for (int q = 0; q < kAhead; ++q) {
            float f[N];
            Vec<T>::unpack(v[q], f);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 d = mul2(add2(make_float2(f[j], f[j + 1]), less), scale);
                s[j >> 1 & 1] = add2(s[j >> 1 & 1], make_float2(exp2_of(d.x), exp2_of(d.y)));
            }
        }
        all += (double)((s[0].x + s[1].x) + (s[0].y + s[1].y));
    };
    int c = 0;
    for (; (c + 1) * kAhead * G <= n; ++c) take(c, [] { return true; });
    if (c * kAhead * G < n) take(c, [] { return false; });

    // the row's maximum, and the first place that has it
    float top = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (G > 32) {
        if (lane == 0) tops[warp] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < G / 32; ++w) top = fmaxf(top, tops[w]);
    }
    int best = P.A;
    if (m == top && top != -INFINITY) {
        if (chunk < 0) {
            best = single(-2 - chunk);
        } else {
            for (int q = kAhead - 1; q >= 0; --q) {
                const int i = (chunk * kAhead + q) * G + me;
                for (int j = N - 1; j >= 0; --j)
                    if (i < n && Vec<T>::load(x + sp.head + (int64_t)(v0 + i) * N + j) == top) best = sp.head + (v0 + i) * N + j;
            }
        }
        for (int i = me; i < singles; i += G)                // a place among the singles may come before the chunk's
            if (Vec<T>::load(x + single(i)) == top) { best = min(best, single(i)); break; }
    }
    best = __reduce_min_sync(~0u, best);
    if (base != top) all = base == -INFINITY ? 0. : all * (double)exp2_of((base - top) * k);
    all = warp_sum(all);
    if (G > 32) {
        if (lane == 0) { sums[warp] = all; bests[warp] = best; }
        __syncthreads();
        all = 0.;
#pragma unroll
        for (int w = 0; w < G / 32; ++w) { all += sums[w]; best = min(best, bests[w]); }
    }
    if (!(all == all) || all > 1e300) {                      // NaN or +inf in the row, or a temperature next to 0 or infinite
        double sum = 0.;
        for (int i = me; i < n; i += G)
            for (int j = 0; j < N; ++j) sum += (double)e_of(Vec<T>::load(x + sp.head + (int64_t)(v0 + i) * N + j), top, inv);
        for (int i = me; i < singles; i += G) sum += (double)e_of(Vec<T>::load(x + single(i)), top, inv);
        all = warp_sum(sum);
        if (G > 32) {
            __syncthreads();
            if (lane == 0) sums[warp] = all;
            __syncthreads();
            all = 0.;
            for (int w = 0; w < G / 32; ++w) all += sums[w];
        }
    }
    if (me == 0) P.stats[row * P.parts + part] = PartStat{top == -INFINITY ? 0. : all, top, best};
    if (me == 0 && part == 0) P.picked[row] = picked;
}

// ---------------------------------------------------------------------------------------------- verdict and draw
// A row of logits: the parts joined.
struct RowStat {
    double all;
    float top, picked;
    int32_t best;
};

constexpr int kMostParts = 16;

// Both of row t's, by a warp: sixteen lanes each.  Lanes below 16 have the target's, the others the draft policy's (nothing without it).
template <typename T> __device__ __forceinline__ RowStat join_parts(const VerifyParams<T>& P, int t, bool both, float inv, int lane) {
    const int part = lane & 15, which = lane >> 4;
    const int64_t row = (int64_t)which * P.rows + t;
    const bool there = which == 0 || both;
    PartStat v = {0., -INFINITY, P.A};
    if (there && part < P.parts) v = P.stats[row * P.parts + part];
    RowStat r;
    r.picked = there ? P.picked[row] : -INFINITY;
    r.top = v.top;
#pragma unroll
    for (int o = 8; o; o >>= 1) r.top = fmaxf(r.top, __shfl_xor_sync(~0u, r.top, o));
    const float d = scaled(v.top, r.top, inv);
    r.all = v.top == -INFINITY || d != d ? 0. : v.all * (double)expf(d);
    r.best = v.top == r.top ? v.best : P.A;
#pragma unroll
    for (int o = 8; o; o >>= 1) {
        r.all += __shfl_xor_sync(~0u, r.all, o);
        r.best = min(r.best, __shfl_xor_sync(~0u, r.best, o));
    }
    return r;
}

// A row's part as a block weighs it: n entries from x on, their maximum finite; their weights go to `to` (16-byte aligned at the row's
// first vector).  An entry that equals the maximum is 0 away, and one of -inf or NaN ends as 0.
template <typename T> struct Weigher {
    static constexpr int N = Vec<T>::N;
    const T* x;
    uint32_t* to;
    Span sp;
    int n;
    float top, inv;

    __device__ __forceinline__ uint4 load(int i) const { return reinterpret_cast<const uint4*>(x + sp.head)[i]; }

    __device__ __forceinline__ u64 vector(int i, const uint4& v) const {
        uint4* const out = reinterpret_cast<uint4*>(to + sp.head) + i * (N / 4);
        // a vector of nothing but weights of 0 (exp below 2^-32): -inf counts among them, NaN is passed over
        const float best = Vec<T>::most_number_of(Vec<T>::most_number(Vec<T>::most_number(v.x, v.y), Vec<T>::most_number(v.z, v.w)));
        if ((best - top) * inv < -22.5f) {
#pragma unroll
            for (int j = 0; j < N; j += 4) out[j / 4] = make_uint4(0, 0, 0, 0);
            return 0;
        }
        float e[N];
        Vec<T>::unpack(v, e);
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            e[j] = expf((e[j] - top) * inv);
            most = max_nan(most, e[j]);
        }
        uint32_t w[N];
        u64 sum = 0;
        if (most < 0x1p-10f) {                               // nearly always: weight_of's short way, sums of 2^24 at most
            uint32_t all = 0;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                w[j] = (__float_as_uint(__fmaf_rd(e[j], 0x1p31f, 4194304.5f)) & 0x7fffffu) >> 1;
                all += w[j];
            }
            sum = all;
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) {
                w[j] = weight_of(e[j] >= 0.f ? e[j] : 0.f);
                sum += w[j];
            }
        }
#pragma unroll
        for (int j = 0; j < N; j += 4) out[j / 4] = make_uint4(w[j], w[j + 1], w[j + 2], w[j + 3]);
        return sum;
    }

    __device__ __forceinline__ u64 singles(int first, int step) const {
        u64 sum = 0;
        const int rest = sp.head + sp.vecs * N;
        for (int i = first; i < sp.head + n - rest; i += step) {
            const int j = i < sp.head ? i : rest + i - sp.head;
            const uint32_t w = weight_of(e_of(Vec<T>::load(x + j), top, inv));
            to[j] = w;
            sum += w;
        }
        return sum;
    }
};

// The sum over a warp of numbers below 2^60: three hardware sums.
__device__ __forceinline__ u64 redux_sum(u64 v) {
    const uint32_t a = __reduce_add_sync(~0u, (uint32_t)v & 0xfffffu), b = __reduce_add_sync(~0u, (uint32_t)(v >> 20) & 0xfffffu);
    return (u64)a + ((u64)b << 20) + ((u64)__reduce_add_sync(~0u, (uint32_t)(v >> 40)) << 40);
}

// 2^52 + floor(w unit), the product rounded to nearest before its floor, for floor(w unit) < 2^52, as the bits of a double: differences of two
// are those of the floors.  Conversions between integers and doubles, which this does without, have a quarter of the rate of 64-bit additions.
__device__ __forceinline__ long long shares_of(uint32_t w, double unit) {
    return __double_as_longlong(__dadd_rd((__hiloint2double(0x43300000, (int)w) - 0x1p52) * unit, 0x1p52));
}

// Log-probability of an entry under the whole softmax.
__device__ __noinline__ float score(double all, float x, float top, float inv) { return (float)((double)scaled(x, top, inv) - log(all)); }

// NT threads a block, a cluster a trajectory.  HELD: a block's weights of both rows stay in shared memory.
template <typename T, int NT, bool HELD>
__global__ void __launch_bounds__(NT, NT >= 384 ? 3 : NT == 256 ? 6 : 1) verify_draw_kernel(const __grid_constant__ VerifyParams<T> P) {
    extern __shared__ __align__(16) uint32_t held[];         // [2, or 1 without drafts' logits][share and up to a vector before it]
    __shared__ u64 part[2][NT / 32], sent[2][16][2], total_of[2];
    __shared__ RowStat stat[2];                              // of row r below
    __shared__ int stop;                                     // least 2 t + 1 of a row whose draft does not stay, 2 t where that is unclear
    const cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = blockIdx.x / ranks, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int begin = max(P.offsets[b], 0), end = min(P.offsets[b + 1], P.rows);
    if (begin >= end) {                                      // for all of the cluster alike
        if (rank == 0 && tid == 0) P.accepted[b] = 0;
        return;
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");      // this block runs
    const float temperature = temperature_of(P, b), inv = inverse_of(temperature);
    const bool greedy = !(temperature > 0.f);
    const int j0 = min(rank * P.share, P.A), j1 = min(j0 + P.share, P.A);

    // (x, y), the same for all lanes of a warp, summed over the cluster by the first warp; x stays in part[0].  Two sets of places, in turn.
    int turns = 0;
    auto cluster_sum = [&](u64* x, u64* y) {
        __syncthreads();
        if (lane == 0) { part[0][warp] = *x; part[1][warp] = *y; }
        __syncthreads();
        const int turn = turns++ & 1;
        if (ranks > 1 && turns == 1) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");      // all of the cluster's blocks run
        if (warp == 0) {
            const u64 a = redux_sum(lane < NT / 32 ? part[0][lane] : 0), c = redux_sum(lane < NT / 32 ? part[1][lane] : 0);
            if (lane < ranks) {
                u64* to = cluster.map_shared_rank(&sent[turn][rank][0], lane);
                to[0] = a;
                to[1] = c;
            }
        }
        if (ranks > 1) cluster.sync(); else __syncthreads();
        if (warp == 0) {
            const u64 a = redux_sum(lane < ranks ? sent[turn][lane][0] : 0), c = redux_sum(lane < ranks ? sent[turn][lane][1] : 0);
            if (lane == 0) { total_of[0] = a; total_of[1] = c; }
        }
        __syncthreads();
        *x = total_of[0];
        *y = total_of[1];
    };
    // does u (v W) < w V hold?
    auto decide = [&](int t, double w, double W, double v, double V) { return (double)P.uniforms[t] * (v * W) < w * V; };
    // a row's weights in shared memory begin where its vectors are aligned there too
    auto lead = [&](const T* x) { return (Vec<T>::N - span_of(x + j0, j1 - j0).head) % Vec<T>::N; };

    // Row r: the first whose draft does not stay, or the last; a warp a row.  Then the exact sums of its weights.
    int r, from = begin;
    bool turned, two;                                        // a draft was turned down; a difference is drawn from
    u64 sums[2];
    while (true) {
        __syncthreads();
        if (tid == 0) stop = INT32_MAX;
        __syncthreads();
        RowStat mine;
        int failed = -1;
        for (int t = from + warp; t < end && failed < 0; t += NT / 32) {
            const bool last = t == end - 1;
            mine = join_parts(P, t, P.drafts != nullptr && !last && !greedy, inv, lane);
            const int token = last ? -1 : P.tokens[t + 1];
            const float top = __shfl_sync(~0u, mine.top, 0), picked = __shfl_sync(~0u, mine.picked, 0);
            const double all = __shfl_sync(~0u, mine.all, 0), all_q = __shfl_sync(~0u, mine.all, 16);
            const double at = mine.top == -INFINITY ? 0. : (double)weight_of(e_of(mine.picked, mine.top, inv)), slack = P.A;
            const double w = __shfl_sync(~0u, at, 0), v_q = __shfl_sync(~0u, at, 16);
            bool yes = false, no = true;
            if (token >= 0 && token < P.A && top != -INFINITY) {
                if (greedy) {
                    yes = token == __shfl_sync(~0u, mine.best, 0);
                } else {                                     // the same verdict at both ends, moved apart by more than the products' roundings
                    constexpr double kLess = 0x1p31 * (1. - 0x1p-15), kMore = 0x1p31 * (1. + 0x1p-15);
                    const bool drawn = P.drafts != nullptr;
                    const double v = drawn ? v_q : 1., least_v = drawn ? fmax(all_q * kLess - slack, 0.) : 1., most_v = drawn ? all_q * kMore + slack : 1.;
                    yes = decide(t, w * (1. - 0x1p-40), all * kMore + slack, v, least_v);
                    no = !decide(t, w * (1. + 0x1p-40), fmax(all * kLess - slack, 0.), v, most_v);
                }
            }
            if (!yes) {
                failed = t;
                if (lane == 0) atomicMin(&stop, 2 * t + (no ? 1 : 0));
            } else if (rank == 0 && lane == 0) {             // unless a row before it fails: below
                P.out[t] = token;
                P.log_probs[t] = score(all, picked, top, inv);
            }
        }
        __syncthreads();
        r = stop >> 1;
        const bool clear = stop & 1;
        if (failed == r && (lane & 15) == 0) stat[lane >> 4] = mine;
        __syncthreads();
        turned = r + 1 < end;
        two = turned && P.drafts != nullptr;
        if (greedy || stat[0].top == -INFINITY) break;
        Weigher<T> of[2];
        bool quick[2];
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            of[which].x = (which ? P.drafts + r * P.ldd : P.logits + r * P.ld) + j0;
            of[which].n = j1 - j0;
            of[which].top = stat[which].top;
            of[which].inv = inv;
            quick[which] = HELD && (which == 0 || two) && stat[which].top != -INFINITY && stat[which].top < INFINITY;
            of[which].sp = quick[which] ? span_of(of[which].x, j1 - j0) : Span{0, 0};
            of[which].to = held + which * (P.share + 8) + (which == 0 || two ? lead(of[which].x - j0) : 0);
            sums[which] = 0;
        }
        // both rows' vectors are on the way together
        for (int i = tid; i < max(of[0].sp.vecs, of[1].sp.vecs); i += NT) {
            uint4 v[2];
#pragma unroll
            for (int which = 0; which < 2; ++which)
                if (i < of[which].sp.vecs) v[which] = of[which].load(i);
#pragma unroll
            for (int which = 0; which < 2; ++which)
                if (i < of[which].sp.vecs) sums[which] += of[which].vector(i, v[which]);
        }
#pragma unroll
        for (int which = 0; which < 2; ++which) {
            if (quick[which]) {
                sums[which] += of[which].singles(tid, NT);
            } else if (which == 0 || two) {
                for (int j = tid; j < j1 - j0; j += NT) {
                    const uint32_t w = of[which].top == -INFINITY ? 0 : weight_of(e_of(Vec<T>::load(of[which].x + j), of[which].top, inv));
                    if (HELD) of[which].to[j] = w;
                    sums[which] += w;
                }
            }
            sums[which] = redux_sum(sums[which]);
        }
        cluster_sum(&sums[0], &sums[1]);
        if (clear) break;
        const double w = weight_of(e_of(stat[0].picked, stat[0].top, inv));
        const double v = !two ? 1. : stat[1].top == -INFINITY ? 0. : (double)weight_of(e_of(stat[1].picked, stat[1].top, inv));
        if (!decide(r, w, (double)sums[0], v, two ? (double)sums[1] : 1.)) break;
        if (rank == 0 && tid == 0) {
            P.out[r] = P.tokens[r + 1];
            P.log_probs[r] = score(stat[0].all, stat[0].picked, stat[0].top, inv);
        }
        from = r + 1;
    }

    const float top = stat[0].top;
    if (rank == 0) {
        if (tid == 0) P.accepted[b] = r - begin;
        for (int t = r + tid; t < end; t += NT)
            if (t > r || top == -INFINITY) {
                P.out[t] = -1;
                P.log_probs[t] = -INFINITY;
            }
    }
    int drawn = -1;                                          // the token of row r, where this thread has it
    const T* const x = P.logits + r * P.ld;
    if (greedy || top == -INFINITY) {
        if (rank == 0 && tid == 0 && top != -INFINITY) drawn = max(0, min(stat[0].best, P.A - 1));      // rows of offsets that do not ascend may hold anything
        if (ranks > 1 && turns == 0) asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
    } else {
        const double p_unit = kShareOne / (double)sums[0], q_unit = sums[1] > 0 ? kShareOne / (double)sums[1] : 0.;
        const int given = turned && !two ? P.tokens[r + 1] : -1;
        bool plain = !turned || (!two && given < 0);
        const T* const y = two ? P.drafts + r * P.ldd : x;
        const uint32_t *my_w = held + lead(x) - j0, *my_v = held + P.share + 8 + lead(y) - j0;
        const float top_q = stat[1].top;
        auto weight = [&](int j) -> u64 {
            const uint32_t w = HELD ? my_w[j] : weight_of(e_of(Vec<T>::load(x + j), top, inv));
            if (plain) return w;
            if (!two) return j == given ? 0 : w;
            const uint32_t v = HELD ? my_v[j] : top_q == -INFINITY ? 0 : weight_of(e_of(Vec<T>::load(y + j), top_q, inv));
            const long long more = shares_of(w, p_unit) - shares_of(v, q_unit);
            return more > 0 ? (u64)more : 0;
        };
        // every warp has a stretch of the block's share, in order
        const int per = ((j1 - j0 + NT / 32 - 1) / (NT / 32) + 31) / 32 * 32, k0 = min(j0 + warp * per, j1), k1 = min(k0 + per, j1);
        u64 mine, total, none = 0;
        __syncthreads();
        while (true) {
            mine = 0;
#pragma unroll 4
            for (int j = k0 + lane; j < k1; j += 32) mine += weight(j);
            total = mine = redux_sum(mine);
            cluster_sum(&total, &none);
            if (total > 0 || plain) break;
            plain = true;                                     // nothing is left of the difference: the target's own probabilities
        }
        const u64 target = target_of(P.draw_uniforms[b], total);
        u64 before = lane < warp ? part[0][lane] : 0;
        if (lane < rank) before += sent[(turns - 1) & 1][lane][0];
        before = redux_sum(before);
        if (before <= target && target < before + mine) {
            for (int base = k0; base < k1; base += 32) {
                const int j = base + lane;
                const u64 w = j < k1 ? weight(j) : 0;
                u64 run = w;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const u64 up = __shfl_up_sync(~0u, run, o);
                    if (lane >= o) run += up;
                }
                const unsigned over = __ballot_sync(~0u, before + run > target);
                if (over) {
                    if (lane == __ffs(over) - 1) drawn = j;
                    break;
                }
                before += __shfl_sync(~0u, run, 31);
            }
        }
    }
    if (drawn >= 0) {
        P.out[r] = drawn;
        P.log_probs[r] = score(stat[0].all, clean(Vec<T>::load(x + drawn)), top, inv);
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int kMostShare = 28 * 1024, kMostRanks = 16;

// Rows are cut into parts only while all parts are fewer than four a multiprocessor.
size_t workspace_of(int64_t rows) { return (size_t)(2 * rows + 4 * rlcs_device::limits().sms) * sizeof(PartStat) + (size_t)(2 * rows) * sizeof(float); }

// One cluster a trajectory.  Room beyond 48 KB of shared memory is asked for once a device.
template <typename T, int NT, bool HELD> int launch_draw(const VerifyParams<T>& P, int ranks, cudaStream_t s) {
    const auto kernel = verify_draw_kernel<T, NT, HELD>;
    static bool granted[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RLCS_ERR_CUDA;
    if (!granted[dev]) {
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 8 * (kMostShare + 8)) != cudaSuccess ||
            cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)
            return RLCS_ERR_CUDA;
        granted[dev] = true;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(P.seqs * ranks));
    cfg.blockDim = dim3(NT);
    cfg.dynamicSmemBytes = HELD ? (P.drafts != nullptr ? 8 : 4) * (size_t)(P.share + 8) : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

template <typename T>
int verify_run(const T* logits, int64_t ld, const T* drafts, int64_t ldd, const int32_t* tokens, const int32_t* offsets, const float* uniforms,
               const float* draw_uniforms, const float* temperature, float temperature_all, int32_t* out, float* log_probs, int32_t* accepted,
               int64_t rows, int64_t seqs, int64_t A, void* workspace, size_t workspace_bytes, void* stream) {
    if (rows < 0 || seqs < 0 || A < 0 || A > (int64_t(1) << 22) || rows > (int64_t(1) << 24) || seqs > (int64_t(1) << 24)) return RLCS_ERR_SIZE;
    if (seqs == 0) return RLCS_OK;
    if (rows > 0 && (A == 0 || ld < A || (drafts != nullptr && ldd < A))) return RLCS_ERR_SIZE;
    if (rows > 0 && (ld > (int64_t(1) << 40) / rows || ldd > (int64_t(1) << 40) / rows)) return RLCS_ERR_SIZE;
    if (std::isnan(temperature_all)) return RLCS_ERR_ARG;
    if (offsets == nullptr || accepted == nullptr) return RLCS_ERR_NULL;
    if (rows > 0 && (logits == nullptr || tokens == nullptr || uniforms == nullptr || draw_uniforms == nullptr || out == nullptr || log_probs == nullptr))
        return RLCS_ERR_NULL;
    const void* words[] = {tokens, offsets, uniforms, draw_uniforms, temperature, out, log_probs, accepted};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(drafts, sizeof(T))) return RLCS_ERR_ALIGN;
    if (rows > 0 && (workspace == nullptr || workspace_bytes < workspace_of(rows))) return RLCS_ERR_WORKSPACE;
    if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    VerifyParams<T> P = {logits, drafts, tokens, offsets, uniforms, draw_uniforms, temperature, temperature_all, out, log_probs, accepted,
                         static_cast<PartStat*>(workspace),
                         reinterpret_cast<float*>(static_cast<PartStat*>(workspace) + 2 * rows + 4 * rlcs_device::limits().sms), ld, ldd, (int32_t)rows, (int32_t)seqs, (int32_t)A, 1, 0};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    const int64_t all = rows * (drafts != nullptr ? 2 : 1), sms = rlcs_device::limits().sms, vecs = A / Vec<T>::N;
    if (rows > 0) {
        if (vecs <= 512) {                                       // a warp's 16 loads at most
            verify_scan_kernel<T, 32><<<(unsigned)((all + kScan / 32 - 1) / (kScan / 32)), kScan, 0, s>>>(P);
        } else {
            // rows in parts while there are fewer than two blocks a multiprocessor and a thread keeps a round of loads
            while (P.parts < kMostParts && all * P.parts < 2 * sms && vecs / (2 * P.parts) >= kScan * kAhead) P.parts *= 2;
            verify_scan_kernel<T, kScan><<<(unsigned)(all * P.parts), kScan, 0, s>>>(P);
        }
    }
    // a block's share of a row: at most 8192 entries where sixteen blocks hold a row so (1000 rows of 50000: 283 us, 479 with shares of
    // half of that), less while there are fewer than two blocks a multiprocessor and a share keeps 2048; the weights of both rows (of one,
    // where the drafts have no logits) in shared memory up to 224 KB
    int ranks = 1;
    while (ranks < kMostRanks && ((A + ranks - 1) / ranks > 8192 || (seqs * ranks < 2 * sms && (A + ranks - 1) / ranks >= 4096))) ranks *= 2;
    P.share = (int32_t)(((A + ranks - 1) / ranks + 7) / 8 * 8);
    const bool hold = P.share <= kMostShare;
    // more than one round: where more than three shares fit into a multiprocessor half the threads, up to twice the blocks at once (1000
    // rows of 50000 198 us, 283 with 512 threads; 2000 of 9000 with the drafts' logits 161, 198); where three do, fewer warps to sum over
    // (300 of 150000 264 us, 284 with 512)
    const int64_t room = P.share * (drafts != nullptr ? 8 : 4);
    const bool queue = seqs * ranks > 3 * sms;
    const int st = A <= 1024 ? launch_draw<T, 128, true>(P, ranks, s) : queue && room <= 48 * 1024 ? launch_draw<T, 256, true>(P, ranks, s)
                   : queue && room <= 74 * 1024 ? launch_draw<T, 384, true>(P, ranks, s)
                   : hold ? launch_draw<T, 512, true>(P, ranks, s) : launch_draw<T, 512, false>(P, ranks, s);
    if (st != RLCS_OK) return st;
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t rlcs_verify_drafts_workspace_bytes(int64_t T, int64_t B) {
    return T <= 0 || B <= 0 || T > (int64_t(1) << 24) || B > (int64_t(1) << 24) ? 0 : workspace_of(T);
}

int rlcs_verify_drafts(const float* logits, int64_t ld, const float* draft_logits, int64_t ldd, const int32_t* tokens, const int32_t* offsets,
                       const float* uniforms, const float* draw_uniforms, const float* temperature, float temperature_all, int32_t* out_tokens,
                       float* log_probs, int32_t* accepted, int64_t T, int64_t B, int64_t A, void* workspace, size_t workspace_bytes,
                       void* cuda_stream) {
    return verify_run<float>(logits, ld, draft_logits, ldd, tokens, offsets, uniforms, draw_uniforms, temperature, temperature_all, out_tokens,
                             log_probs, accepted, T, B, A, workspace, workspace_bytes, cuda_stream);
}

int rlcs_verify_drafts_bf16(const uint16_t* logits, int64_t ld, const uint16_t* draft_logits, int64_t ldd, const int32_t* tokens,
                            const int32_t* offsets, const float* uniforms, const float* draw_uniforms, const float* temperature,
                            float temperature_all, int32_t* out_tokens, float* log_probs, int32_t* accepted, int64_t T, int64_t B, int64_t A,
                            void* workspace, size_t workspace_bytes, void* cuda_stream) {
    return verify_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, reinterpret_cast<const bf16*>(draft_logits), ldd, tokens, offsets, uniforms,
                            draw_uniforms, temperature, temperature_all, out_tokens, log_probs, accepted, T, B, A, workspace, workspace_bytes,
                            cuda_stream);
}

}  // extern "C"

// Policy loss of given actions from logits [R, A], and its gradient.
//
//   lp = log softmax(l / T),  p_j = exp(lp_j),  H = -sum_j p_j lp_j
//   gain = adv * lp_a,  or  min(rho adv, clip(rho, 1 - eps, 1 + eps) adv)  with rho = exp(lp_a - old)
//   loss = -scale * (gain + c H)
//   d loss / d l_j = scale / T * [ s (p_j - [j = a]) + c p_j (lp_j + H) ],   s = adv, or rho adv where unclipped, or 0
//
// With y_j = l_j - max l, S = sum exp(y_j / T) and U = sum exp(y_j / T) y_j:  lp_j = y_j / T - log S, H = log S - U / (S T),
// and the bracket is p_j (s + c (H - log S) + (c / T) y_j): one multiply-add a logit on top of its exponential.  The maximum is
// taken off before the division, so that a masked logit of the type's lowest value cannot overflow.
#include <cooperative_groups.h>

#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_pair.cuh"
#include "rlcs_rows.cuh"

namespace rlcs_hooks {
extern int g_wait_polls;      // rlcs_debug_set_wait_polls; defined in rlcs_api.cu
}

namespace {

using namespace rlcs_pair;
using namespace rlcs_rows;

template <typename T> struct PolicyParams {
    const T* logits;
    int64_t ld;
    const int32_t* actions;
    const uint8_t* mask;
    const float* advantages;
    const float* old_log_probs;
    float* loss;
    float* log_probs;
    float* entropy;
    T* dlogits;
    int64_t ldd;
    int64_t R;
    int A;
    float inv_t, exp2_t, clip, bonus, scale;       // 1 / T and log2(e) / T
    int polls;                                     // kPolls, or a test's
};

constexpr float kLowest = -1.0e30f;      // stands for y = -inf where y multiplies exp(y / T) = 0

// running maximum with the sums relative to it
struct Stat {
    float m, s, u;
};

// the sums of `a` relative to a maximum m that is not below its own
__device__ __forceinline__ Stat rebase(Stat a, float m, float exp2_t) {
    const float y = fmaxf(a.m - m, kLowest), f = exp2_of(y * exp2_t);
    // nothing is left of far lower logits, though their own sums may have overflowed (policy_block_kernel); a NaN stays in s
    return Stat{m, f == 0.f && a.s == a.s ? 0.f : a.s * f, f == 0.f ? 0.f : (a.u + a.s * y) * f};
}

__device__ __forceinline__ Stat join(Stat a, Stat b, float exp2_t) {
    const float m = fmaxf(a.m, b.m);
    if (m == -INFINITY) return Stat{m, a.s + b.s, 0.f};
    const Stat x = rebase(a, m, exp2_t), y = rebase(b, m, exp2_t);
    return Stat{m, x.s + y.s, x.u + y.u};
}

// What the gradient pass needs of a row.
struct RowGrad {
    float c0, c1, inv_s, m, hit;          // dl_j = exp(y / T) * inv_s * (c0 + c1 y), minus `hit` at the action
                                          // (y times `unit` is y / T)
    bool live;
};

__device__ __forceinline__ float grad_of(float x, const RowGrad& g, float exp2_t) {
    const float y = x - g.m;
    return exp2_of(y * exp2_t) * g.inv_s * fmaf(g.c1, fmaxf(y, kLowest), g.c0);
}

// `d`: (l_a - max) / T; `unit`: what turns the unit of U into that of d.
// Loaded ahead of the sums: a row's advantage and acting log-probability.
struct Given {
    float advantage, old_log_prob;
};

template <typename T> __device__ __forceinline__ Given given_of(const PolicyParams<T>& P, int64_t row, bool live) {
    return Given{live && P.advantages != nullptr ? P.advantages[row] : 0.f, live && P.old_log_probs != nullptr ? P.old_log_probs[row] : 0.f};
}

template <typename T>
__device__ __forceinline__ RowGrad finish_row(const PolicyParams<T>& P, int64_t row, const Given& given, Stat st, float d, float unit, bool live,
                                              bool write) {
    live = live && (st.m != -INFINITY || st.s != st.s);     // maxima pass NaN over: a row of it is told from one of -inf by its sum
    float loss = 0.f, lp = 0.f, h = 0.f, slope = 0.f;
    const float log_s = logf(st.s), inv = 1.f / st.s;
    if (live) {
        lp = d - log_s;
        h = log_s - st.u * inv * unit;
        if (P.advantages != nullptr) {
            const float adv = given.advantage;
            float gain = adv * lp;
            slope = adv;
            if (P.old_log_probs != nullptr) {
                const float ratio = expf(lp - given.old_log_prob);
                const float free_ = ratio * adv, held = fminf(fmaxf(ratio, 1.f - P.clip), 1.f + P.clip) * adv;
                gain = fminf(free_, held);
                slope = free_ <= held ? free_ : 0.f;
                // minimum and comparison pass NaN over; a ratio past the largest float times an advantage of 0 is 0 all the same
                if (ratio != ratio || adv != adv) gain = slope = ratio + adv;
            }
            loss = -P.scale * (gain + P.bonus * h);
        }
    }
    if (write) {
        if (P.loss != nullptr) P.loss[row] = loss;
        P.log_probs[row] = lp;
        P.entropy[row] = h;
    }
    RowGrad g;
    g.live = live;
    g.m = st.m;
    g.inv_s = P.inv_t * inv;
    g.c0 = P.scale * (slope + P.bonus * (h - log_s));
    g.c1 = P.scale * P.bonus * unit;
    g.hit = P.scale * slope * P.inv_t;
    return g;
}

// 65 to 2048 (fp32) or 4096 (bfloat16) actions: G lanes a row, NV vectors of it in the registers of each.
template <typename T, int G, int NV>
__global__ void __launch_bounds__(256) policy_group_kernel(const __grid_constant__ PolicyParams<T> P) {
    constexpr int N = Vec<T>::N;
    const int lane = threadIdx.x % G;
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    const bool there = row < P.R;                              // every lane takes part in the sums
    const T* x = P.logits + (there ? row : 0) * P.ld;
    const int a = there ? P.actions[row] : -1;
    const bool live = there && (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < P.A;
    const Given given = given_of(P, row, live);
    const Span sp = span_of(x, P.A);
    const int rest = sp.head + sp.vecs * N, singles = sp.head + P.A - rest;
    const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
    auto single = [&](int i) { return i < sp.head ? i : rest + i - sp.head; };
    constexpr int kOnes = (2 * N - 2 + G - 1) / G;             // elements before and behind the vectors, a lane
    uint4 v[NV];
    float one[kOnes];
    const float xa = live ? Vec<T>::load(x + a) : 0.f;
#pragma unroll
    for (int q = 0; q < NV; ++q)
        v[q] = live && q * G + lane < sp.vecs ? body[q * G + lane] : make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
#pragma unroll
    for (int q = 0; q < kOnes; ++q) one[q] = live && q * G + lane < singles ? Vec<T>::load(x + single(q * G + lane)) : -INFINITY;
    uint32_t most = Vec<T>::kNothing;
#pragma unroll
    for (int q = 0; q < NV; ++q)
        most = Vec<T>::most_number(most, Vec<T>::most_number(Vec<T>::most_number(v[q].x, v[q].y), Vec<T>::most_number(v[q].z, v[q].w)));
    Stat st = {Vec<T>::most_number_of(most), 0.f, 0.f};
#pragma unroll
    for (int q = 0; q < kOnes; ++q) st.m = fmaxf(st.m, one[q]);
#pragma unroll
    for (int o = G / 2; o; o >>= 1) st.m = fmaxf(st.m, __shfl_xor_sync(~0u, st.m, o));
    const float base = st.m == -INFINITY ? 0.f : st.m;
    const float2 less = {-base, -base}, scale = {P.exp2_t, P.exp2_t};
    float2 s = {0.f, 0.f}, u = {0.f, 0.f};
    auto take = [&](float2 f) {
        const float2 t = mul2(add2(f, less), scale), w = make_float2(exp2_of(t.x), exp2_of(t.y));
        s = add2(s, w);
        u = fma2(w, make_float2(fmaxf(t.x, kLowest), fmaxf(t.y, kLowest)), u);
    };
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        float f[N];
        Vec<T>::unpack(v[q], f);
#pragma unroll
        for (int j = 0; j < N; j += 2) take(make_float2(f[j], f[j + 1]));
    }
#pragma unroll
    for (int q = 0; q < kOnes; ++q) take(make_float2(one[q], -INFINITY));
    st.s = s.x + s.y;
    st.u = u.x + u.y;
#pragma unroll
    for (int o = G / 2; o; o >>= 1) {
        st.s += __shfl_xor_sync(~0u, st.s, o);
        st.u += __shfl_xor_sync(~0u, st.u, o);
    }
    constexpr float kLn2 = 0.6931471805599453f;
    if (!there) return;
    const RowGrad g = finish_row(P, row, given, st, (xa - st.m) * P.inv_t, kLn2, live, lane == 0);
    if (P.dlogits == nullptr) return;
    T* y = P.dlogits + row * P.ldd;
    const float c0 = g.live ? g.c0 * g.inv_s : 0.f, c1 = g.live ? g.c1 * g.inv_s : 0.f;
    const float2 two0 = {c0, c0}, two1 = {c1, c1};
#pragma unroll
    for (int q = 0; q < NV; ++q)                               // unpacked again, not kept unpacked since the sums: half the registers
        asm volatile("" : "+r"(v[q].x), "+r"(v[q].y), "+r"(v[q].z), "+r"(v[q].w));
    auto grad2 = [&](float2 f) {
        const float2 t = mul2(add2(f, less), scale);
        return mul2(make_float2(exp2_of(t.x), exp2_of(t.y)), fma2(two1, make_float2(fmaxf(t.x, kLowest), fmaxf(t.y, kLowest)), two0));
    };
    const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
    uint4* out = reinterpret_cast<uint4*>(y + sp.head);
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        if (q * G + lane >= sp.vecs) break;
        const int at = sp.head + (q * G + lane) * N;
        float f[N];
        if (g.live) {
            Vec<T>::unpack(v[q], f);
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 r = grad2(make_float2(f[j], f[j + 1]));
                f[j] = r.x;
                f[j + 1] = r.y;
            }
            if (a >= at && a < at + N) {
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] -= at + j == a ? g.hit : 0.f;
            }
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) f[j] = 0.f;
        }
        if (same) {
            out[q * G + lane] = Vec<T>::pack(f);
        } else {
#pragma unroll
            for (int j = 0; j < N; ++j) Vec<T>::store(y + at + j, f[j]);
        }
    }
#pragma unroll
    for (int q = 0; q < kOnes; ++q)
        if (q * G + lane < singles) {
            const int j = single(q * G + lane);
            Vec<T>::store(y + j, g.live ? grad2(make_float2(one[q], one[q])).x - (j == a ? g.hit : 0.f) : 0.f);
        }
}

// Rows of up to 16 KB: one warp a row, two passes over it, the second from L1 or L2 (67 million logits, shares of the copy bandwidth:
// 4096 fp32 0.63 and 8192 bfloat16 0.55, against 0.58 and 0.47 with a block a row; 8192 fp32 0.52 against 0.86).
constexpr int kWarpBytes = 16384;

template <typename T>
__global__ void __launch_bounds__(256) policy_warp_kernel(const __grid_constant__ PolicyParams<T> P) {
    constexpr int N = Vec<T>::N, kAhead = 2, NT = 32;
    const int tid = threadIdx.x & 31;
    for (int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); row < P.R; row += (int64_t)gridDim.x * 8) {
        const T* x = P.logits + row * P.ld;
        const int a = P.actions[row];
        const bool live = (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < P.A;
        const Given given = given_of(P, row, live);
        const Span sp = span_of(x, P.A);
        const int rest = sp.head + sp.vecs * N;
        const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
        Stat st = {-INFINITY, 0.f, 0.f};
        float xa = 0.f;
        if (live) {
            xa = Vec<T>::load(x + a);
            auto take = [&](const float* f, int n) {
                float top = -INFINITY;
#pragma unroll
                for (int k = 0; k < n; ++k) top = fmaxf(top, f[k]);
                if (top > st.m) st = rebase(st, top, P.exp2_t);
                // a group of -inf and NaN ahead of every other logit has no base yet: 0 keeps -inf at weight 0
                const float base = st.m == -INFINITY ? 0.f : st.m;
                float s = 0.f, u = 0.f;
#pragma unroll
                for (int k = 0; k < n; ++k) {
                    const float y = f[k] - base, w = exp2_of(y * P.exp2_t);
                    s += w;
                    u = fmaf(w, fmaxf(y, kLowest), u);
                }
                st.s += s;
                st.u += u;
            };
            int i = tid;
            for (; i + (kAhead - 1) * NT < sp.vecs; i += kAhead * NT) {
                uint4 v[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) v[k] = body[i + k * NT];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    float f[N];
                    Vec<T>::unpack(v[k], f);
                    take(f, N);
                }
            }
            for (; i < sp.vecs; i += NT) {
                float f[N];
                Vec<T>::unpack(body[i], f);
                take(f, N);
            }
            for (int j = tid; j < sp.head + P.A - rest; j += NT) {
                const float f = Vec<T>::load(x + (j < sp.head ? j : rest + j - sp.head));
                take(&f, 1);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            const Stat other = {__shfl_xor_sync(~0u, st.m, o), __shfl_xor_sync(~0u, st.s, o), __shfl_xor_sync(~0u, st.u, o)};
            st = join(st, other, P.exp2_t);
        }
        const RowGrad g = finish_row(P, row, given, st, (xa - st.m) * P.inv_t, P.inv_t, live, tid == 0);
        if (P.dlogits == nullptr) continue;
        T* y = P.dlogits + row * P.ldd;
        if (((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0) {
            uint4* out = reinterpret_cast<uint4*>(y + sp.head);
            auto give = [&](int i, const uint4& v) {
                float f[N];
                Vec<T>::unpack(v, f);
#pragma unroll
                for (int k = 0; k < N; ++k) f[k] = grad_of(f[k], g, P.exp2_t);
                const int at = a - sp.head - i * N;
                if (at >= 0 && at < N) {
#pragma unroll
                    for (int k = 0; k < N; ++k) f[k] -= k == at ? g.hit : 0.f;
                }
                out[i] = Vec<T>::pack(f);
            };
            int i = tid;
            if (!g.live) {
                for (; i < sp.vecs; i += NT) out[i] = make_uint4(0, 0, 0, 0);
            } else {
                for (; i + (kAhead - 1) * NT < sp.vecs; i += kAhead * NT) {
                    uint4 v[kAhead];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) v[k] = body[i + k * NT];
#pragma unroll
                    for (int k = 0; k < kAhead; ++k) give(i + k * NT, v[k]);
                }
                for (; i < sp.vecs; i += NT) give(i, body[i]);
            }
            for (int k = tid; k < sp.head + P.A - rest; k += NT) {
                const int j = k < sp.head ? k : rest + k - sp.head;
                Vec<T>::store(y + j, g.live ? grad_of(Vec<T>::load(x + j), g, P.exp2_t) - (j == a ? g.hit : 0.f) : 0.f);
            }
        } else {
            for (int j = tid; j < P.A; j += NT)
                Vec<T>::store(y + j, g.live ? grad_of(Vec<T>::load(x + j), g, P.exp2_t) - (j == a ? g.hit : 0.f) : 0.f);
        }
    }
}

// More actions: one cluster of `ranks` blocks a row, row after row.  Each block copies its part of a row to shared memory once (STAGED:
// parts of up to 64 KB, so that three blocks share a multiprocessor), sums, and writes the gradient from there.  Every warp has
// a contiguous share in four chunks, which it fetches itself: as a chunk's gradient is written, the next row's chunk is on
// its way into its place, without a barrier.  The blocks of a cluster send one another their sums (st.async onto a barrier that
// counts bytes): a cluster barrier would wait for the gradient's stores.  One read and one write of global memory:
// without the staging a row's second read came from HBM, not L2 (592 rows of 256 KB in flight are more than it holds; 0.68 of the copy
// bandwidth at 4096 x 131072).  Rows too long for eight parts are read twice.
//
// Sums here are in units of log2: t_j = l_j log2(e) / T - M with one fused multiply-add, M the thread's running maximum so
// scaled (any M serves: it cancels), two logits an instruction.  Logits are held above -1e30, so that t is finite where exp2(t) is
// 0.  M is rounded and the fused product is not: from |M| = 2^27 on, t at the maximum itself is more than a few units off 0, and sums
// may overflow.  Of a thread's logits that lie so far below the row's others (a mask of -1e9, say) nothing is left when the sums
// are joined; a row whose largest logit itself lies so far from 0 goes through exact().
constexpr int kBlock = 256, kWarps = kBlock / 32, kAhead = 4, kChunk = kAhead * 32, kChunks = 4, kShare = kChunks * kChunk;      // vectors of a warp
constexpr int kPart = kWarps * kShare * 16, kMostRanks = 8;

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

constexpr int kPolls = 1 << 20;                 // of a wait, before it gives up

// Bounded; a wait that runs out leaves NaN in the row's outputs.
__device__ __forceinline__ bool chunk_wait(uint32_t bar, int parity, int most) {
    for (int polls = 0; polls < most; ++polls) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
    }
    return false;
}

// What was given up is waited for once more, longer than another block of the cluster takes to give up: its place and its barrier are used
// again, and no block ends while something is on its way to it.  `stuck`: not even that helped; no more copies and no more sums, and the
// block leaves its other rows as they are.
__device__ __forceinline__ void wait_again(uint32_t bar, int parity, volatile int* stuck) {
    if (*stuck || !chunk_wait(bar, parity, 8 * kPolls)) *stuck = 1;
}

// One row as a warp of the cluster sees it.
template <typename T> struct RowPart {
    int64_t row;
    const T* x;
    int a, v0, n;                        // its vectors: n from v0 on
    Span sp;
    bool live;

    // `log_warps`: log2 of the cluster's warps
    __device__ __forceinline__ RowPart(const PolicyParams<T>& P, int64_t row_, int warp, int log_warps) : row(row_) {
        live = false;
        x = nullptr;
        a = v0 = n = 0;
        sp = Span{0, 0};
        if (row >= P.R) return;
        x = P.logits + row * P.ld;
        a = P.actions[row];
        live = (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < P.A;
        sp = span_of(x, P.A);
        const int per = (sp.vecs + (1 << log_warps) - 1) >> log_warps;
        v0 = min(warp * per, sp.vecs);
        n = min(per, sp.vecs - v0);
    }
    __device__ __forceinline__ const uint4* body() const { return reinterpret_cast<const uint4*>(x + sp.head) + v0; }
};

template <typename T, bool STAGED>
__global__ void __launch_bounds__(kBlock, 3) policy_block_kernel(const __grid_constant__ PolicyParams<T> P) {
    constexpr int N = Vec<T>::N;
    constexpr float kLn2 = 0.6931471805599453f;
    extern __shared__ uint4 held_all[];
    __shared__ Stat part[kWarps], joined;
    __shared__ __align__(16) float4 sent[2][kMostRanks];
    __shared__ RowGrad grad;
    __shared__ int stuck, leave;                             // leave: stuck as the whole block saw it
    __shared__ __align__(8) uint64_t full[kWarps][kChunks], got[2];
    namespace cg = cooperative_groups;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), clusters = gridDim.x / ranks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, my_warp = rank * kWarps + warp, log_warps = 31 - __clz(ranks * kWarps);
    const float k = P.exp2_t;
    uint4* const held = held_all + warp * kShare;
    if (tid < kWarps * kChunks) asm volatile("mbarrier.init.shared.b64 [%0], 1;" ::"r"(smem_at(&full[0][0] + tid)));
    if (tid == 0) stuck = leave = 0;
    if (tid < 2) asm volatile("mbarrier.init.shared.b64 [%0], 1;" ::"r"(smem_at(&got[tid])));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    cluster.sync();

    auto fetch = [&](const RowPart<T>& r, int c) {           // by one lane; every chunk of a live row, empty ones too
        const int left = r.n - c * kChunk, count = left < 0 ? 0 : min(left, kChunk);
        const uint32_t bar = smem_at(&full[warp][c]);
        asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(count * 16) : "memory");
        if (count > 0)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_at(held + c * kChunk)), "l"(r.body() + c * kChunk), "r"(count * 16), "r"(bar) : "memory");
    };
    // `width` lanes' sums joined: the maximum first, then one rescaling a lane
    auto shuffled = [&](Stat st, int width) {
        float m = st.m;
        for (int o = width / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
        if (m != -INFINITY) st = rebase(st, m, 1.f);
        for (int o = width / 2; o; o >>= 1) {
            st.s += __shfl_xor_sync(~0u, st.s, o);
            st.u += __shfl_xor_sync(~0u, st.u, o);
        }
        return st;
    };
    // Over the cluster, for the first warp, the same on every block of it.  Two sets of places for what the blocks send, taken in
    // turn: a block sends the sums after the next only when it has everybody's next, and nobody sends those before it has read.
    int turns = 0;
    auto gather = [&](Stat st) {
        st = shuffled(st, 32);
        if (lane == 0) part[warp] = st;
        __syncthreads();
        if (warp == 0) {
            st = shuffled(part[lane % kWarps], kWarps);
            if (ranks > 1) {
                const int turn = turns & 1;
                const uint32_t bar = smem_at(&got[turn]), place = smem_at(&sent[turn][rank]);
                const bool apart = *(volatile int*)&stuck != 0;
                if (lane == 0 && !apart) asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(ranks * 16) : "memory");
                if (lane < ranks && !apart) {
                    uint32_t there, its_bar;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(place), "r"(lane));
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(its_bar) : "r"(bar), "r"(lane));
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v4.b32 [%0], {%1, %2, %3, %4}, [%5];"
                                 ::"r"(there), "r"(__float_as_uint(st.m)), "r"(__float_as_uint(st.s)), "r"(__float_as_uint(st.u)), "r"(0), "r"(its_bar) : "memory");
                }
                const bool fine = !apart && chunk_wait(bar, (turns >> 1) & 1, P.polls);
                if (!fine) wait_again(bar, (turns >> 1) & 1, &stuck);
                const float4 v = sent[turn][lane % ranks];
                st = shuffled(Stat{v.x, fine ? v.y : __int_as_float(0x7fffffff), v.z}, ranks);
                if (!apart) ++turns;
            }
        }
        return st;
    };
    auto gather_all = [&](Stat st) {
        st = gather(st);
        if (tid == 0) joined = st;
        __syncthreads();
        st = joined;
        __syncthreads();
        return st;
    };

    RowPart<T> now(P, blockIdx.x / ranks, my_warp, log_warps);
    int loads = 0;                                           // rows fetched: the chunks' barriers go by its last bit
    if (STAGED && lane == 0 && now.live)
        for (int c = 0; c < kChunks; ++c) fetch(now, c);
    while (now.row < P.R) {
        RowPart<T> next(P, now.row + clusters, my_warp, log_warps);
        const T* x = now.x;
        T* y = P.dlogits != nullptr ? P.dlogits + now.row * P.ldd : nullptr;
        const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
        const int a = now.a, head = now.sp.head, rest = head + now.sp.vecs * N, v0 = now.v0, n = now.n;
        const uint4* body = now.body();
        uint4* out = reinterpret_cast<uint4*>(y + head) + v0;
        // the single elements before and behind the vectors: the first block's first threads
        const int singles = rank == 0 ? head + P.A - rest : 0, single = tid < head ? tid : rest + tid - head;
        const Given given = given_of(P, now.row, now.live);
        if (!now.live) {
            if (rank == 0 && tid == 0) finish_row(P, now.row, given, Stat{-INFINITY, 0.f, 0.f}, 0.f, 0.f, false, true);
            if (y != nullptr) {
                if (same) for (int i = lane; i < n; i += 32) out[i] = make_uint4(0, 0, 0, 0);
                else for (int i = lane; i < n * N; i += 32) Vec<T>::store(y + head + v0 * N + i, 0.f);
                if (tid < singles) Vec<T>::store(y + single, 0.f);
            }
            if (STAGED && lane == 0 && next.live)
                for (int c = 0; c < kChunks; ++c) fetch(next, c);
            now = next;
            continue;
        }
        const float xa = Vec<T>::load(x + a);
        const float alone = tid < singles ? Vec<T>::load(x + single) : -INFINITY;
        // the plain way, for rows whose largest logit lies far from 0: (l - max) first
        auto exact = [&]() {
            float m = -INFINITY;
            for (int i = lane; i < n; i += 32) {
                float f[N];
                Vec<T>::unpack(body[i], f);
                for (int j = 0; j < N; ++j) m = max_nan(m, f[j]);
            }
            m = max_nan(m, alone);
            m = gather_all(Stat{m, 0.f, 0.f}).m;
            Stat st = {0.f, 0.f, 0.f};
            const float base = m == -INFINITY ? 0.f : m;     // -inf then weighs 0, and NaN stays NaN
            auto take = [&](float f) {
                const float t = (f - base) * k, w = exp2_of(t);
                st.s += w;
                st.u = fmaf(w, fmaxf(t, kLowest), st.u);
            };
            for (int i = lane; i < n; i += 32) {
                float f[N];
                Vec<T>::unpack(body[i], f);
                for (int j = 0; j < N; ++j) take(f[j]);
            }
            if (tid < singles) take(alone);
            st = gather_all(st);
            st.m = m;
            return st;
        };

        Stat st = {-INFINITY, 0.f, 0.f};
        if (tid < singles && alone != -INFINITY) {
            const float f = max_nan(alone, kLowest);
            st.m = f * k;
            st.s = f == f ? 1.f : f;
        }
        auto sum_chunk = [&](int c, auto whole) {            // whole: no vector of the chunk lies behind the row's end
            const uint4* from = (STAGED ? held : body) + c * kChunk + lane;
            const int left = n - c * kChunk - lane;
            uint4 v[kAhead];
#pragma unroll
            for (int q = 0; q < kAhead; ++q)
                v[q] = whole() || q * 32 < left ? from[q * 32] : make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
            uint32_t most = Vec<T>::kNothing;
#pragma unroll
            for (int q = 0; q < kAhead; ++q) most = Vec<T>::most(most, Vec<T>::most(Vec<T>::most(v[q].x, v[q].y), Vec<T>::most(v[q].z, v[q].w)));
            const float top = Vec<T>::most_of(most);
            if (top == -INFINITY) return;
            const float M = max_nan(top, kLowest) * k;
            if (M > st.m) st = rebase(st, M, 1.f);
            const float2 scale = {k, k}, less = {-st.m, -st.m};
            float2 s = {0.f, 0.f}, u = {0.f, 0.f};
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                float f[N];
                Vec<T>::unpack(Vec<T>::floored(v[q]), f);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 t = fma2(make_float2(f[j], f[j + 1]), scale, less), w = make_float2(exp2_of(t.x), exp2_of(t.y));
                    s = add2(s, w);
                    u = fma2(w, t, u);
                }
            }
            st.s += s.x + s.y;
            st.u += u.x + u.y;
        };
        for (int c = 0; c * kChunk < n; ++c) {
            const uint32_t bar = smem_at(&full[warp][c & (kChunks - 1)]);
            if (STAGED && !chunk_wait(bar, loads & 1, P.polls)) {
                st.s = __int_as_float(0x7fffffff);
                wait_again(bar, loads & 1, &stuck);
            }
            if ((c + 1) * kChunk <= n) sum_chunk(c, [] { return true; }); else sum_chunk(c, [] { return false; });
        }
        if (STAGED)                                          // empty chunks have a phase too
            for (int c = (n + kChunk - 1) / kChunk; c < kChunks; ++c)
                if (!chunk_wait(smem_at(&full[warp][c]), loads & 1, P.polls)) wait_again(smem_at(&full[warp][c]), loads & 1, &stuck);
        ++loads;
        st = gather(st);
        if (warp == 0) {
            const float d = xa < kLowest ? xa * P.inv_t : fmaf(xa, k, -st.m) * kLn2;
            // a temperature that takes -1e30 out of range, or a maximum too far from 0: again, the plain way
            const bool again = k > 1e7f || !(fabsf(st.m) < 0x1p27f);
            RowGrad g = finish_row(P, now.row, given, st, d, kLn2, true, !again && rank == 0 && tid == 0);
            g.live = !again;
            if (tid == 0) {
                grad = g;
                leave = *(volatile int*)&stuck;
            }
        }
        __syncthreads();
        RowGrad g = grad;
        const bool plain = !g.live;
        if (plain) {
            st = exact();
            g = finish_row(P, now.row, given, st, (xa - st.m) * P.inv_t, kLn2, true, rank == 0 && tid == 0);
        }
        if (leave) {                                         // for all of the block alike
            next.live = false;
            next.row = P.R;
        }
        const float c0 = g.c0 * g.inv_s, c1 = g.c1 * g.inv_s;
        const float2 scale = {k, k}, less = {-g.m, -g.m}, two0 = {c0, c0}, two1 = {c1, c1};
        auto slow = [&](float f, int j) {
            const float t = plain ? (f - g.m) * k : fmaf(max_nan(f, kLowest), k, -g.m);
            return g.live ? exp2_of(t) * fmaf(c1, fmaxf(t, kLowest), c0) - (j == a ? g.hit : 0.f) : 0.f;
        };
        auto give_chunk = [&](int c, auto whole) {           // whole: as above, and the action is in none of its vectors
            const uint4* from = (STAGED ? held : body) + c * kChunk + lane;
            uint4* to = out + c * kChunk + lane;
            const int left = n - c * kChunk - lane;
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (!whole() && q * 32 >= left) break;
                const int at = head + (v0 + c * kChunk + q * 32 + lane) * N;
                float f[N];
                if (!whole() && plain) {
                    Vec<T>::unpack(body[c * kChunk + q * 32 + lane], f);
#pragma unroll
                    for (int j = 0; j < N; ++j) f[j] = slow(f[j], at + j);
                } else {
                    Vec<T>::unpack(Vec<T>::floored(from[q * 32]), f);
#pragma unroll
                    for (int j = 0; j < N; j += 2) {
                        const float2 t = fma2(make_float2(f[j], f[j + 1]), scale, less);
                        const float2 r = mul2(make_float2(exp2_of(t.x), exp2_of(t.y)), fma2(two1, t, two0));
                        f[j] = r.x;
                        f[j + 1] = r.y;
                    }
                    if (!whole()) {
#pragma unroll
                        for (int j = 0; j < N; ++j) f[j] -= at + j == a ? g.hit : 0.f;
                    }
                }
                if (whole() || same) {
                    to[q * 32] = Vec<T>::pack(f);
                } else {
#pragma unroll
                    for (int j = 0; j < N; ++j) Vec<T>::store(y + at + j, f[j]);
                }
            }
        };
        const int hit_at = a < head ? -1 : (a - head) / N - v0;      // the action's vector of this warp's
        for (int c = 0; c < kChunks || c * kChunk < n; ++c) {
            if (y != nullptr) {
                const bool hit = hit_at >= c * kChunk && hit_at < (c + 1) * kChunk;
                if ((c + 1) * kChunk <= n && !hit && same && !plain) give_chunk(c, [] { return true; }); else give_chunk(c, [] { return false; });
            }
            if (STAGED) {
                __syncwarp();                                // the chunk's place is free
                if (lane == 0 && next.live) fetch(next, c);
            }
        }
        if (y != nullptr && tid < singles) Vec<T>::store(y + single, slow(alone, single));
        now = next;
    }
    if (leave && ranks > 1 && warp == 0) {                   // what the others send before they find this block gone
        const uint32_t bar = smem_at(&got[turns & 1]);
        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"((ranks - 1) * 16) : "memory");
        chunk_wait(bar, (turns >> 1) & 1, 8 * kPolls);
    }
}

// Up to 64 actions: one thread a row.  The block brings its rows to shared memory as fp32 (16-byte loads where rows follow one
// another), a thread walks its own row there, and the gradients leave the same way.  Rows lie an odd number of words apart, so that
// the threads of a warp meet different banks, and every thread takes the same number of steps (walking from a place of its own
// instead cost four times the instructions).
constexpr int kSmallRows = 128, kSmallA = 64;

template <typename T>
__global__ void __launch_bounds__(kSmallRows) policy_small_kernel(const __grid_constant__ PolicyParams<T> P, uint32_t a_mul) {
    constexpr int N = Vec<T>::N;
    extern __shared__ __align__(16) float tile[];
    const int A = P.A, stride = A | 1, gap = stride - A, tid = threadIdx.x;
    const int64_t row0 = (int64_t)blockIdx.x * kSmallRows, row = row0 + tid;
    const int rows = P.R - row0 < kSmallRows ? (int)(P.R - row0) : kSmallRows, n = rows * A;
    const T* from = P.logits + row0 * P.ld;
    T* to = P.dlogits != nullptr ? P.dlogits + row0 * P.ldd : nullptr;
    auto of = [&](int i) { return a_mul != 0 ? (int)__umulhi((uint32_t)i, a_mul) : i; };      // the row of flat element i
    // flat vectors to and from the rows' places
    auto put = [&](int i, const float* f) {
        if (gap == 0) {
#pragma unroll
            for (int k = 0; k < N; k += 4) *reinterpret_cast<float4*>(tile + i + k) = make_float4(f[k], f[k + 1], f[k + 2], f[k + 3]);
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 2) {                 // A is even, and so is i: two neighbours share a row
                const int at = i + k + (int)__umulhi((uint32_t)(i + k), a_mul);
                tile[at] = f[k];
                tile[at + 1] = f[k + 1];
            }
        }
    };
    auto get = [&](int i, float* f) {
        if (gap == 0) {
#pragma unroll
            for (int k = 0; k < N; k += 4) {
                const float4 v = *reinterpret_cast<const float4*>(tile + i + k);
                f[k] = v.x; f[k + 1] = v.y; f[k + 2] = v.z; f[k + 3] = v.w;
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; k += 2) {
                const int at = i + k + (int)__umulhi((uint32_t)(i + k), a_mul);
                f[k] = tile[at];
                f[k + 1] = tile[at + 1];
            }
        }
    };
    const int a = tid < rows ? P.actions[row] : -1;
    const bool live = tid < rows && (P.mask == nullptr || P.mask[row] != 0) && a >= 0 && a < A;
    const Given given = given_of(P, row, live);
    if (P.ld == A && (reinterpret_cast<uintptr_t>(from) & 15) == 0) {
#pragma unroll 4
        for (int i = tid * N; i < n - N + 1; i += kSmallRows * N) {
            float f[N];
            Vec<T>::unpack(*reinterpret_cast<const uint4*>(from + i), f);
            put(i, f);
        }
        for (int i = n / N * N + tid; i < n; i += kSmallRows) tile[i + gap * of(i)] = Vec<T>::load(from + i);
    } else {
#pragma unroll 4
        for (int i = tid; i < n; i += kSmallRows) {
            const int r = of(i);
            tile[i + gap * r] = Vec<T>::load(from + r * P.ld + (i - r * A));
        }
    }
    __syncthreads();
    if (tid < rows) {
        float* x = tile + tid * stride;
        Stat st = {-INFINITY, 0.f, 0.f};
        float xa = 0.f;
        if (live) {
            xa = x[a];
#pragma unroll 4
            for (int j = 0; j < A; ++j) st.m = fmaxf(st.m, x[j]);
            const float base = st.m == -INFINITY ? 0.f : st.m;
#pragma unroll 4
            for (int j = 0; j < A; ++j) {
                const float y = x[j] - base, w = exp2_of(y * P.exp2_t);
                st.s += w;
                st.u = fmaf(w, fmaxf(y, kLowest), st.u);
            }
        }
        const RowGrad g = finish_row(P, row, given, st, (xa - st.m) * P.inv_t, P.inv_t, live, true);
        if (to != nullptr) {
            const float c0 = g.c0 * g.inv_s, c1 = g.c1 * g.inv_s;
            if (g.live) {
#pragma unroll 4
                for (int j = 0; j < A; ++j) {
                    const float y = x[j] - g.m;
                    x[j] = exp2_of(y * P.exp2_t) * fmaf(c1, fmaxf(y, kLowest), c0);
                }
                x[a] -= g.hit;
            } else {
                for (int j = 0; j < A; ++j) x[j] = 0.f;
            }
        }
    }
    if (to == nullptr) return;
    __syncthreads();
    if (P.ldd == A && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
#pragma unroll 4
        for (int i = tid * N; i < n - N + 1; i += kSmallRows * N) {
            float f[N];
            get(i, f);
            *reinterpret_cast<uint4*>(to + i) = Vec<T>::pack(f);
        }
        for (int i = n / N * N + tid; i < n; i += kSmallRows) Vec<T>::store(to + i, tile[i + gap * of(i)]);
    } else {
#pragma unroll 4
        for (int i = tid; i < n; i += kSmallRows) {
            const int r = of(i);
            Vec<T>::store(to + r * P.ldd + (i - r * A), tile[i + gap * r]);
        }
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// One cluster a row, as many as the GPU holds at once: asked for once a device and cluster size (a cluster too many would start when the others have ended and double the time).
template <typename T, bool STAGED>
int launch_block(const PolicyParams<T>& P, int ranks, cudaStream_t s) {
    const auto kernel = policy_block_kernel<T, STAGED>;
    static int at_once[64][kMostRanks + 1];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RLCS_ERR_CUDA;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ranks);
    cfg.blockDim = dim3(kBlock);
    cfg.dynamicSmemBytes = STAGED ? kPart : 0;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (at_once[dev][ranks] == 0) {
        if (STAGED && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPart) != cudaSuccess) return RLCS_ERR_CUDA;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) return RLCS_ERR_CUDA;
        at_once[dev][ranks] = n;
    }
    cfg.gridDim = dim3((unsigned)((P.R < at_once[dev][ranks] ? P.R : at_once[dev][ranks]) * ranks));
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

template <typename T>
int policy_run(const T* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
               const float* old_log_probs, float* loss, float* log_probs, float* entropy, T* dlogits, int64_t ldd,
               int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* stream) {
    if (R < 0 || A < 0 || A > (int64_t(1) << 22) || R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (R == 0) return RLCS_OK;
    if (A == 0 || ld < A || (dlogits != nullptr && ldd < A)) return RLCS_ERR_SIZE;
    if (ld > (int64_t(1) << 40) / R || ldd > (int64_t(1) << 40) / R) return RLCS_ERR_SIZE;
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.4426950408889634f / temperature)) return RLCS_ERR_ARG;
    if (!(clip >= 0.f) || !std::isfinite(entropy_coef) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (logits == nullptr || actions == nullptr || log_probs == nullptr || entropy == nullptr) return RLCS_ERR_NULL;
    if ((loss != nullptr || dlogits != nullptr || old_log_probs != nullptr) && advantages == nullptr) return RLCS_ERR_NULL;
    const void* words[] = {actions, advantages, old_log_probs, loss, log_probs, entropy};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(dlogits, sizeof(T))) return RLCS_ERR_ALIGN;
    PolicyParams<T> P = {logits, ld, actions, mask, advantages, old_log_probs, loss, log_probs, entropy, dlogits, ldd, R, (int)A,
                         1.f / temperature, 1.4426950408889634f / temperature, clip, entropy_coef, scale,
                         rlcs_hooks::g_wait_polls >= 0 ? rlcs_hooks::g_wait_polls : kPolls};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (A <= kSmallA) {
        const int64_t blocks = (R + kSmallRows - 1) / kSmallRows;
        if (blocks > (int64_t(1) << 31) - 1) return RLCS_ERR_SIZE;
        const uint32_t mul = A > 1 ? (uint32_t)(((uint64_t(1) << 32) + A - 1) / A) : 0;
        policy_small_kernel<T><<<(unsigned)blocks, kSmallRows, kSmallRows * (A | 1) * sizeof(float), s>>>(P, mul);
    } else if (const int64_t vecs = A / Vec<T>::N; vecs <= 512) {
        const int lanes = vecs <= 64 ? 8 : 32;
        const int64_t blocks = (R * lanes + 255) / 256;
        if (blocks > (int64_t(1) << 31) - 1) return RLCS_ERR_SIZE;
        const unsigned n = (unsigned)blocks;
        if (vecs <= 32) policy_group_kernel<T, 8, 4><<<n, 256, 0, s>>>(P);
        else if (vecs <= 64) policy_group_kernel<T, 8, 8><<<n, 256, 0, s>>>(P);
        else if (vecs <= 128) policy_group_kernel<T, 32, 4><<<n, 256, 0, s>>>(P);
        else if (vecs <= 256) policy_group_kernel<T, 32, 8><<<n, 256, 0, s>>>(P);
        else policy_group_kernel<T, 32, 16><<<n, 256, 0, s>>>(P);
    } else if (A * (int64_t)sizeof(T) <= kWarpBytes) {
        const int64_t blocks = (R + 7) / 8;
        policy_warp_kernel<T><<<(unsigned)(blocks < (1 << 20) ? blocks : (1 << 20)), 256, 0, s>>>(P);
    } else {
        // blocks a row: parts of at most 64 KB; more while the GPU has room for two a multiprocessor and a part keeps 8 KB
        const int64_t bytes = A * (int64_t)sizeof(T);
        int ranks = 1;
        while (ranks < kMostRanks && (bytes > (int64_t)ranks * kPart || (R * ranks < 2 * rlcs_device::limits().sms && bytes / (2 * ranks) >= 8192)))
            ranks *= 2;
        const bool staged = bytes <= (int64_t)ranks * kPart;
        const int st = staged ? launch_block<T, true>(P, ranks, s) : launch_block<T, false>(P, ranks, s);
        if (st != RLCS_OK) return st;
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_policy_grad(const float* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
                     const float* old_log_probs, float* loss, float* log_probs, float* entropy, float* dlogits, int64_t ldd,
                     int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* cuda_stream) {
    return policy_run<float>(logits, ld, actions, mask, advantages, old_log_probs, loss, log_probs, entropy, dlogits, ldd, R, A,
                             temperature, clip, entropy_coef, scale, cuda_stream);
}

int rlcs_policy_grad_bf16(const uint16_t* logits, int64_t ld, const int32_t* actions, const uint8_t* mask, const float* advantages,
                          const float* old_log_probs, float* loss, float* log_probs, float* entropy, uint16_t* dlogits, int64_t ldd,
                          int64_t R, int64_t A, float temperature, float clip, float entropy_coef, float scale, void* cuda_stream) {
    return policy_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, actions, mask, advantages, old_log_probs, loss, log_probs,
                            entropy, reinterpret_cast<bf16*>(dlogits), ldd, R, A, temperature, clip, entropy_coef, scale, cuda_stream);
}

}  // extern "C"

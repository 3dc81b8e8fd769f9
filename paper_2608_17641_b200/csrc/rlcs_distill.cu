// Loss towards the strongest logits of a teacher, and its gradient, from a student's logits [R, A].
//
//   lq = log softmax(l / T) over all A,   p = softmax(teacher / T) over the row's given entries
//   loss = scale * sum_i p_i (log p_i - lq_{id_i}),   d loss / d l_j = scale / T * (exp(lq_j) - sum_{i: id_i = j} p_i)
//
// One read of the logits and one write of the gradient are the floor.  With m the row's maximum, S = sum exp((l - m) / T) and q_j =
// exp((l_j - m) / T) / S: the gradient is q_j scale / T everywhere but at the teacher's entries, which are written once more, after the
// rest, with what they lack: a row's K entries are few.  The maximum is taken off before the division, so that logits far from 0 lose nothing.
//
// Measured: 4096 x 131072 bfloat16, K = 64, 440 us (0.75 of the copy bandwidth; 413 without the teacher's entries): the exponential unit 59 % busy,
// a row's chain (sums over the cluster, entries) under it; 1021 x 50021 fp32, K = 20, 15 % masked, 92 us (0.63: 9.8 rows a cluster
// count as ten and more).  Not kept: entries one after the other by a whole warp (484 us), eight blocks a row (648).
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

template <typename T> struct DistillParams {
    const T* logits;
    const int32_t* ids;
    const float* teacher;
    const uint8_t* mask;
    float* loss;
    T* dlogits;
    int64_t ld, ldd, R;
    int32_t A, K;
    float inv_t, exp2_t, scale;            // 1 / T and log2(e) / T
    int polls;                             // kPolls, or a test's
};

constexpr int kMostTop = 1024;

// maximum, with the sum of exponentials relative to it
struct Sum {
    float m, s;
};

// The sum relative to a maximum that is not below its own; nothing is left of nothing, a NaN stays.
__device__ __forceinline__ float faded(Sum a, float m, float k) { return a.m == m ? a.s : a.s * exp2_of((a.m - m) * k); }

// Over `width` lanes; maxima pass NaN over, sums keep it.
__device__ __forceinline__ Sum join_lanes(Sum a, int width, float k) {
    float m = a.m;
    for (int o = width / 2; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
    float s = faded(a, m, k);
    for (int o = width / 2; o; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
    return Sum{m, s};
}

// What a row's gradient and loss need: softmax sums of the student's row and of the teacher's entries.
struct Both {
    Sum student, teacher;
    __device__ __forceinline__ bool live() const {       // something on either side; NaN counts as something
        return (student.m != -INFINITY || student.s != student.s) && (teacher.m != -INFINITY || teacher.s != teacher.s);
    }
};

// A teacher entry's probability.
__device__ __forceinline__ float chance(float t, const Both& r, float k) { return exp2_of((t - r.teacher.m) * k) / r.teacher.s; }

// p (log p - log q): an entry's part of the loss.
template <typename T> __device__ __forceinline__ float term(const DistillParams<T>& P, float t, float x, const Both& r, float log_gap) {
    const float p = chance(t, r, P.exp2_t);
    return p == 0.f ? 0.f : p * ((t - r.teacher.m) * P.inv_t - (x - r.student.m) * P.inv_t + log_gap);      // log_gap: log S - log Z
}

__device__ __forceinline__ void add_one(Sum* a, float f, float k) {
    if (!(f <= a->m)) {                                      // larger, or NaN
        a->s = a->m == -INFINITY ? a->s : a->s * exp2_of((a->m - f) * k);
        a->m = f;
    }
    if (a->m != -INFINITY) a->s += exp2_of((f - a->m) * k);
}

// ---------------------------------------------------------------------------------------------- short rows
// What G lanes have, joined: by shuffles in a warp, over the block through shared memory (`room` serves one join).
template <int G> struct Lanes {
    static __device__ __forceinline__ void sync() {
        if constexpr (G > 32) __syncthreads(); else __syncwarp();
    }
    template <typename F> static __device__ __forceinline__ float join(float v, float nothing, float* room, F op) {
#pragma unroll
        for (int o = (G < 32 ? G : 32) / 2; o; o >>= 1) v = op(v, __shfl_xor_sync(~0u, v, o));
        if constexpr (G > 32) {
            if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = v;
            __syncthreads();
            v = nothing;
#pragma unroll
            for (int w = 0; w < G / 32; ++w) v = op(v, room[w]);
        }
        return v;
    }
    static __device__ __forceinline__ float most(float v, float* room) { return join(v, -INFINITY, room, [](float a, float b) { return fmaxf(a, b); }); }
    static __device__ __forceinline__ float sum(float v, float* room) { return join(v, 0.f, room, [](float a, float b) { return a + b; }); }
};

// Up to 2048 (fp32) or 4096 (bfloat16) entries, up to four times that with G = 256: G lanes a row, NV vectors of it in the registers
// of each, and up to E of the teacher's entries (E = 0: any number, read again when needed; what they are to get waits in shared
// memory until the rest is written).  A bit a student's entry tells whether one is named twice.
template <typename T, int G, int NV, int E>
__global__ void __launch_bounds__(256) distill_group_kernel(const __grid_constant__ DistillParams<T> P) {
    constexpr int N = Vec<T>::N;
    extern __shared__ uint32_t room[];                       // a row: K values (E = 0), then a bit for each of the A entries
    __shared__ float joined[6][8];
    const int lane = threadIdx.x % G, words = (P.A + 31) / 32;
    const int64_t row = (int64_t)blockIdx.x * (256 / G) + threadIdx.x / G;
    const bool there = row < P.R && (P.mask == nullptr || P.mask[row] != 0);       // every lane takes part in the sums
    const int kept = E > 0 ? 0 : P.K;
    float* const value = reinterpret_cast<float*>(room + threadIdx.x / G * (kept + words));
    uint32_t* const named = room + threadIdx.x / G * (kept + words) + kept;
    const T* x = P.logits + (row < P.R ? row : 0) * P.ld;
    const Span sp = span_of(x, P.A);
    const int rest = sp.head + sp.vecs * N, singles = sp.head + P.A - rest;
    const uint4* body = reinterpret_cast<const uint4*>(x + sp.head);
    auto single = [&](int i) { return i < sp.head ? i : rest + i - sp.head; };
    constexpr int kOnes = (2 * N - 2 + G - 1) / G;           // elements before and behind the vectors, a lane
    uint4 v[NV];
    float one[kOnes];
#pragma unroll
    for (int q = 0; q < NV; ++q)
        v[q] = there && q * G + lane < sp.vecs ? body[q * G + lane] : make_uint4(Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing, Vec<T>::kNothing);
#pragma unroll
    for (int q = 0; q < kOnes; ++q) one[q] = there && q * G + lane < singles ? Vec<T>::load(x + single(q * G + lane)) : -INFINITY;
    const int32_t* ids = P.ids + row * P.K;
    const float* teacher = P.teacher + row * P.K;
    int my_id[E > 0 ? E : 1];
    float my_t[E > 0 ? E : 1], my_x[E > 0 ? E : 1];
#pragma unroll
    for (int q = 0; q < E; ++q) {
        const bool any = there && q * G + lane < P.K;
        my_id[q] = any ? ids[q * G + lane] : -1;
        my_t[q] = any ? teacher[q * G + lane] : 0.f;
    }
    for (int i = lane; i < words; i += G) named[i] = 0;
    Lanes<G>::sync();
    Both r = {{-INFINITY, 0.f}, {-INFINITY, 0.f}};
    bool twice = false;
#pragma unroll
    for (int q = 0; q < E; ++q) {
        if (my_id[q] >= P.A) my_id[q] = -1;
        if (my_id[q] < 0) continue;
        my_x[q] = Vec<T>::load(x + my_id[q]);
        r.teacher.m = max_nan(r.teacher.m, my_t[q]);
        twice = twice || (atomicOr(named + my_id[q] / 32, 1u << my_id[q] % 32) >> my_id[q] % 32 & 1);
    }
#pragma unroll
    for (int q = 0; q < E; ++q)
        if (my_id[q] >= 0 && r.teacher.m != -INFINITY) r.teacher.s += exp2_of((my_t[q] - r.teacher.m) * P.exp2_t);
    if (E == 0 && there)
        for (int i = lane; i < P.K; i += G) {
            const int id = ids[i];
            if (id < 0 || id >= P.A) continue;
            add_one(&r.teacher, teacher[i], P.exp2_t);
            twice = twice || (atomicOr(named + id / 32, 1u << id % 32) >> id % 32 & 1);
        }
    twice = Lanes<G>::most(twice ? 1.f : 0.f, joined[0]) > 0.f;
    uint32_t most = Vec<T>::kNothing;
#pragma unroll
    for (int q = 0; q < NV; ++q)
        most = Vec<T>::most_number(most, Vec<T>::most_number(Vec<T>::most_number(v[q].x, v[q].y), Vec<T>::most_number(v[q].z, v[q].w)));
    float m = Vec<T>::most_number_of(most);
#pragma unroll
    for (int q = 0; q < kOnes; ++q) m = fmaxf(m, one[q]);
    m = Lanes<G>::most(m, joined[1]);
    const float base = m == -INFINITY ? 0.f : m;             // -inf then weighs 0, and NaN stays NaN
    const float2 less = {-base, -base}, scale = {P.exp2_t, P.exp2_t};
    float2 s = {0.f, 0.f};
    auto weight2 = [&](float2 f) {
        const float2 t = mul2(add2(f, less), scale);
        return make_float2(exp2_of(t.x), exp2_of(t.y));
    };
#pragma unroll
    for (int q = 0; q < NV; ++q) {
        float f[N];
        Vec<T>::unpack(v[q], f);
#pragma unroll
        for (int j = 0; j < N; j += 2) s = add2(s, weight2(make_float2(f[j], f[j + 1])));
    }
#pragma unroll
    for (int q = 0; q < kOnes; ++q) s.x += weight2(make_float2(one[q], -INFINITY)).x;
    r.student = Sum{m, Lanes<G>::sum(s.x + s.y, joined[2])};
    {
        const float tm = Lanes<G>::most(r.teacher.m, joined[3]);
        r.teacher = Sum{tm, Lanes<G>::sum(faded(r.teacher, tm, P.exp2_t), joined[4])};
    }
    const bool live = there && r.live();
    const float unit = live ? P.scale * P.inv_t : 0.f;
    const float c = r.teacher.s == r.teacher.s ? unit / r.student.s : r.teacher.s;      // a teacher of NaN: the whole row
    float loss = 0.f;
    if (live) {
        const float log_gap = logf(r.student.s) - logf(r.teacher.s);
#pragma unroll
        for (int q = 0; q < E; ++q) {
            if (my_id[q] < 0) continue;
            float p = chance(my_t[q], r, P.exp2_t);
            loss += term(P, my_t[q], my_x[q], r, log_gap);
            if (twice) {
                p = 0.f;
                for (int k = 0; k < P.K; ++k)
                    if (ids[k] == my_id[q]) p += chance(teacher[k], r, P.exp2_t);
            }
            my_t[q] = exp2_of((my_x[q] - base) * P.exp2_t) * c - unit * p;      // what the entry is to get
        }
        for (int i = lane; E == 0 && i < P.K; i += G) {
            const int id = ids[i];
            if (id < 0 || id >= P.A) continue;
            const float xi = Vec<T>::load(x + id);
            float p = chance(teacher[i], r, P.exp2_t);
            loss += term(P, teacher[i], xi, r, log_gap);
            if (twice) {
                p = 0.f;
                for (int k = 0; k < P.K; ++k)
                    if (ids[k] == id) p += chance(teacher[k], r, P.exp2_t);
            }
            value[i] = exp2_of((xi - base) * P.exp2_t) * c - unit * p;
        }
    }
    loss = Lanes<G>::sum(loss, joined[5]);
    if (row < P.R && lane == 0 && P.loss != nullptr) P.loss[row] = live ? P.scale * loss : 0.f;
    Lanes<G>::sync();                                        // logits that are overwritten have been read
    if (row < P.R && P.dlogits != nullptr) {
        T* y = P.dlogits + row * P.ldd;
        const float2 two = {c, c};
#pragma unroll
        for (int q = 0; q < NV; ++q)                         // unpacked again, not kept unpacked since the sums: half the registers
            asm volatile("" : "+r"(v[q].x), "+r"(v[q].y), "+r"(v[q].z), "+r"(v[q].w));
        const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
        uint4* out = reinterpret_cast<uint4*>(y + sp.head);
#pragma unroll
        for (int q = 0; q < NV; ++q) {
            if (q * G + lane >= sp.vecs) break;
            float f[N];
            if (live) {
                Vec<T>::unpack(v[q], f);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 g = mul2(weight2(make_float2(f[j], f[j + 1])), two);
                    f[j] = g.x;
                    f[j + 1] = g.y;
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) f[j] = 0.f;
            }
            if (same) {
                out[q * G + lane] = Vec<T>::pack(f);
            } else {
                const int at = sp.head + (q * G + lane) * N;
#pragma unroll
                for (int j = 0; j < N; ++j) Vec<T>::store(y + at + j, f[j]);
            }
        }
#pragma unroll
        for (int q = 0; q < kOnes; ++q)
            if (q * G + lane < singles) Vec<T>::store(y + single(q * G + lane), live ? weight2(make_float2(one[q], one[q])).x * c : 0.f);
    }
    Lanes<G>::sync();
    if (live && P.dlogits != nullptr) {
#pragma unroll
        for (int q = 0; q < E; ++q)
            if (my_id[q] >= 0) Vec<T>::store(P.dlogits + row * P.ldd + my_id[q], my_t[q]);      // all that name an entry have the same value for it
        for (int i = lane; E == 0 && i < P.K; i += G) {
            const int id = ids[i];
            if (id >= 0 && id < P.A) Vec<T>::store(P.dlogits + row * P.ldd + id, value[i]);
        }
    }
}

// ---------------------------------------------------------------------------------------------- long rows
// One cluster of `ranks` blocks a row, row after row.  Each block copies its part of a row to shared memory once (STAGED: parts
// of up to 64 KB, so that three blocks share a multiprocessor), sums, and writes the gradient from there.  Every warp has a contiguous
// share in four chunks, which it fetches itself: as a chunk's gradient is written, the next row's chunk is on its way into its place,
// without a barrier.  The blocks of a cluster send one another their sums (st.async onto a barrier that counts bytes): a cluster
// barrier would wait for the gradient's stores.  Every block has all of the row's teacher entries, two rows of them in turn; a
// warp writes those that fall into its share, after the share.  Rows too long for eight parts are read twice.
constexpr int kBlock = 256, kWarps = kBlock / 32, kAhead = 4, kChunk = kAhead * 32, kChunks = 4, kShare = kChunks * kChunk;      // vectors of a warp
constexpr int kPart = kWarps * kShare * 16, kMostRanks = 8, kMine = kMostTop / kBlock;      // kMine: teacher entries a thread fetches
constexpr int kPolls = 1 << 20;                 // of a wait, before it gives up

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

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
    int v0, n;                           // its vectors: n from v0 on
    Span sp;
    bool wanted;

    // `log_warps`: log2 of the cluster's warps
    __device__ __forceinline__ RowPart(const DistillParams<T>& P, int64_t row_, int warp, int log_warps) : row(row_) {
        wanted = false;
        x = nullptr;
        v0 = n = 0;
        sp = Span{0, 0};
        if (row >= P.R) return;
        x = P.logits + row * P.ld;
        wanted = P.mask == nullptr || P.mask[row] != 0;
        sp = span_of(x, P.A);
        const int per = (sp.vecs + (1 << log_warps) - 1) >> log_warps;
        v0 = min(warp * per, sp.vecs);
        n = min(per, sp.vecs - v0);
    }
    __device__ __forceinline__ const uint4* body() const { return reinterpret_cast<const uint4*>(x + sp.head) + v0; }
};

template <typename T, bool STAGED>
__global__ void __launch_bounds__(kBlock, 3) distill_block_kernel(const __grid_constant__ DistillParams<T> P) {
    constexpr int N = Vec<T>::N;
    extern __shared__ uint4 held_all[];
    __shared__ Both part[kWarps], joined;
    __shared__ __align__(8) float2 sent[2][kMostRanks];
    __shared__ uint16_t listed[kWarps][32];                  // teacher entries that fall to a warp
    __shared__ int stuck, leave;                             // leave: stuck as the whole block saw it
    __shared__ __align__(8) uint64_t full[kWarps][kChunks], got[2];
    namespace cg = cooperative_groups;
    const cg::cluster_group cluster = cg::this_cluster();
    const int ranks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), clusters = gridDim.x / ranks;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, my_warp = rank * kWarps + warp, log_warps = 31 - __clz(ranks * kWarps);
    const float k = P.exp2_t;
    uint4* const held = held_all + warp * kShare;
    // the teacher's entries of this row and the next: numbers (-1: absent), logits, the student's logits there
    int32_t* const entry_id = reinterpret_cast<int32_t*>(held_all + (STAGED ? kPart / 16 : 0));
    float *const entry_t = reinterpret_cast<float*>(entry_id + 2 * P.K), *const entry_x = entry_t + 2 * P.K;
    if (tid < kWarps * kChunks) asm volatile("mbarrier.init.shared.b64 [%0], 1;" ::"r"(smem_at(&full[0][0] + tid)));
    if (tid == 0) stuck = leave = 0;
    if (tid < 2) asm volatile("mbarrier.init.shared.b64 [%0], 1;" ::"r"(smem_at(&got[tid])));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    cluster.sync();

    auto fetch = [&](const RowPart<T>& r, int c) {           // by one lane; every chunk of a wanted row, empty ones too
        const int left = r.n - c * kChunk, count = left < 0 ? 0 : min(left, kChunk);
        const uint32_t bar = smem_at(&full[warp][c]);
        asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(count * 16) : "memory");
        if (count > 0)
            asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                         ::"r"(smem_at(held + c * kChunk)), "l"(r.body() + c * kChunk), "r"(count * 16), "r"(bar) : "memory");
    };
    int next_id[kMine];
    float next_t[kMine];
    auto fetch_entries = [&](const RowPart<T>& r) {
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            const int i = q * kBlock + tid;
            next_id[q] = -1;
            if (q * kBlock >= P.K) break;
            if (r.wanted && i < P.K) {
                next_id[q] = P.ids[r.row * P.K + i];
                next_t[q] = P.teacher[r.row * P.K + i];
            }
        }
    };
    // Both sums over the block, the student's over the cluster, for the first warp, the same on every block of it.  Two sets of places
    // for what the blocks send, taken in turn: a block sends the sums after the next only when it has everybody's next, and nobody
    // sends those before it has read.
    int turns = 0;
    auto gather = [&](Both r) {
        r.student = join_lanes(r.student, 32, k);
        r.teacher = join_lanes(r.teacher, 32, k);
        if (lane == 0) part[warp] = r;
        __syncthreads();
        if (warp == 0) {
            r = part[lane % kWarps];
            r.student = join_lanes(r.student, kWarps, k);
            r.teacher = join_lanes(r.teacher, kWarps, k);
            if (ranks > 1) {
                const int turn = turns & 1;
                const uint32_t bar = smem_at(&got[turn]), place = smem_at(&sent[turn][rank]);
                const bool apart = *(volatile int*)&stuck != 0;
                if (lane == 0 && !apart) asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(ranks * 8) : "memory");
                if (lane < ranks && !apart) {
                    uint32_t there, its_bar;
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(place), "r"(lane));
                    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(its_bar) : "r"(bar), "r"(lane));
                    asm volatile("st.async.weak.shared::cluster.mbarrier::complete_tx::bytes.v2.b32 [%0], {%1, %2}, [%3];"
                                 ::"r"(there), "r"(__float_as_uint(r.student.m)), "r"(__float_as_uint(r.student.s)), "r"(its_bar) : "memory");
                }
                const bool fine = !apart && chunk_wait(bar, (turns >> 1) & 1, P.polls);
                if (!fine) wait_again(bar, (turns >> 1) & 1, &stuck);
                const float2 v = sent[turn][lane % ranks];
                r.student = join_lanes(Sum{v.x, fine ? v.y : __int_as_float(0x7fffffff)}, ranks, k);
                if (!apart) ++turns;
            }
        }
        return r;
    };

    RowPart<T> now(P, blockIdx.x / ranks, my_warp, log_warps);
    int loads = 0;                                           // rows fetched: the chunks' barriers and the entries' places go by its last bit
    if (STAGED && lane == 0 && now.wanted)
        for (int c = 0; c < kChunks; ++c) fetch(now, c);
    fetch_entries(now);
    while (now.row < P.R) {
        RowPart<T> next(P, now.row + clusters, my_warp, log_warps);
        const T* x = now.x;
        T* y = P.dlogits != nullptr ? P.dlogits + now.row * P.ldd : nullptr;
        const bool same = ((reinterpret_cast<uintptr_t>(x) ^ reinterpret_cast<uintptr_t>(y)) & 15) == 0;
        const int head = now.sp.head, rest = head + now.sp.vecs * N, v0 = now.v0, n = now.n;
        const uint4* body = now.body();
        uint4* out = reinterpret_cast<uint4*>(y + head) + v0;
        // the single elements before and behind the vectors: the first block's first threads
        const int singles = rank == 0 ? head + P.A - rest : 0, single = tid < head ? tid : rest + tid - head;
        auto zeros = [&]() {
            if (rank == 0 && tid == 0 && P.loss != nullptr) P.loss[now.row] = 0.f;
            if (y == nullptr) return;
            if (same) for (int i = lane; i < n; i += 32) out[i] = make_uint4(0, 0, 0, 0);
            else for (int i = lane; i < n * N; i += 32) Vec<T>::store(y + head + v0 * N + i, 0.f);
            if (tid < singles) Vec<T>::store(y + single, 0.f);
        };
        if (!now.wanted) {
            zeros();
            if (STAGED && lane == 0 && next.wanted)
                for (int c = 0; c < kChunks; ++c) fetch(next, c);
            now = next;
            fetch_entries(now);
            continue;
        }
        // the row's entries: their logits are on the way while the sums are made
        int32_t* const id = entry_id + (loads & 1) * P.K;
        float *const t = entry_t + (loads & 1) * P.K, *const xs = entry_x + (loads & 1) * P.K;
        Both r = {{-INFINITY, 0.f}, {-INFINITY, 0.f}};
        float x_at[kMine];
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            if (q * kBlock >= P.K) break;
            const int i = q * kBlock + tid;
            const bool there = next_id[q] >= 0 && next_id[q] < P.A;
            x_at[q] = there ? Vec<T>::load(x + next_id[q]) : 0.f;
            if (there) add_one(&r.teacher, next_t[q], k);
            if (i < P.K) {
                id[i] = there ? next_id[q] : -1;
                t[i] = next_t[q];
            }
        }
        fetch_entries(next);
        if (tid < singles) add_one(&r.student, Vec<T>::load(x + single), k);
        const float alone = tid < singles ? Vec<T>::load(x + single) : 0.f;
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
            if (!(top <= r.student.m)) {                     // larger, or NaN, which the sum then keeps
                r.student.s = r.student.m == -INFINITY ? r.student.s : r.student.s * exp2_of((r.student.m - top) * k);
                r.student.m = top;
            }
            if (r.student.m == -INFINITY) return;
            const float2 scale = {k, k}, less = {-r.student.m, -r.student.m};
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
            r.student.s += (s[0].x + s[1].x) + (s[0].y + s[1].y);
        };
        for (int c = 0; c * kChunk < n; ++c) {
            const uint32_t bar = smem_at(&full[warp][c & (kChunks - 1)]);
            if (STAGED && !chunk_wait(bar, loads & 1, P.polls)) {
                r.student.s = __int_as_float(0x7fffffff);
                wait_again(bar, loads & 1, &stuck);
            }
            if ((c + 1) * kChunk <= n) sum_chunk(c, [] { return true; }); else sum_chunk(c, [] { return false; });
        }
        if (STAGED)                                          // empty chunks have a phase too
            for (int c = (n + kChunk - 1) / kChunk; c < kChunks; ++c)
                if (!chunk_wait(smem_at(&full[warp][c]), loads & 1, P.polls)) wait_again(smem_at(&full[warp][c]), loads & 1, &stuck);
        ++loads;
#pragma unroll
        for (int q = 0; q < kMine; ++q) {
            if (q * kBlock >= P.K) break;
            if (q * kBlock + tid < P.K) xs[q * kBlock + tid] = x_at[q];
        }
        r = gather(r);
        if (tid == 0) {
            joined = r;
            leave = *(volatile int*)&stuck;
        }
        __syncthreads();
        r = joined;
        if (leave) {                                         // for all of the block alike
            next.wanted = false;
            next.row = P.R;
        }
        const bool live = r.live();
        const float unit = P.scale * P.inv_t, c0 = r.teacher.s == r.teacher.s ? unit / r.student.s : r.teacher.s;      // a teacher of NaN: the whole row
        const float2 scale = {k, k}, less = {-r.student.m, -r.student.m}, two = {c0, c0};
        auto slow = [&](float f) { return exp2_of((f - r.student.m) * k) * c0; };
        if (rank == 0 && warp == kWarps - 1 && P.loss != nullptr) {
            const float log_gap = logf(r.student.s) - logf(r.teacher.s);
            float loss = 0.f;
            for (int i = lane; i < P.K; i += 32)
                if (live && id[i] >= 0) loss += term(P, t[i], xs[i], r, log_gap);
            loss = warp_sum(loss);
            if (lane == 0) P.loss[now.row] = live ? P.scale * loss : 0.f;
        }
        auto give_chunk = [&](int c, auto whole) {
            const uint4* from = (STAGED ? held : body) + c * kChunk + lane;
            uint4* to = out + c * kChunk + lane;
            const int left = n - c * kChunk - lane;
#pragma unroll
            for (int q = 0; q < kAhead; ++q) {
                if (!whole() && q * 32 >= left) break;
                float f[N];
                Vec<T>::unpack(from[q * 32], f);
#pragma unroll
                for (int j = 0; j < N; j += 2) {
                    const float2 d = mul2(add2(make_float2(f[j], f[j + 1]), less), scale);
                    const float2 g = mul2(make_float2(exp2_of(d.x), exp2_of(d.y)), two);
                    f[j] = g.x;
                    f[j + 1] = g.y;
                }
                if (whole() || same) {
                    to[q * 32] = Vec<T>::pack(f);
                } else {
                    const int at = head + (v0 + c * kChunk + q * 32 + lane) * N;
#pragma unroll
                    for (int j = 0; j < N; ++j) Vec<T>::store(y + at + j, f[j]);
                }
            }
        };
        if (!live) zeros();
        for (int c = 0; c < kChunks || c * kChunk < n; ++c) {
            if (y != nullptr && live) {
                if ((c + 1) * kChunk <= n && same) give_chunk(c, [] { return true; }); else give_chunk(c, [] { return false; });
            }
            if (STAGED) {
                __syncwarp();                                // the chunk's place is free
                if (lane == 0 && next.wanted) fetch(next, c);
            }
        }
        if (y != nullptr && live) {
            if (tid < singles) Vec<T>::store(y + single, slow(alone));
            __syncwarp();
            // entries that fall to this warp: its vectors', and the single elements' to the first block's first warp
            const int lo = head + v0 * N, hi = lo + n * N;
            const bool ends = rank == 0 && warp == 0;
            const float z = 1.f / r.teacher.s;
            auto mine = [&](int e) { return e >= 0 && ((e >= lo && e < hi) || (ends && (e < head || e >= rest))); };
            int count = 0;
            for (int i0 = 0; i0 < P.K; i0 += 32) {
                const bool hit = mine(i0 + lane < P.K ? id[i0 + lane] : -1);
                const unsigned hits = __ballot_sync(~0u, hit);
                const int at = count + __popc(hits & ((1u << lane) - 1));
                if (hit && at < 32) listed[warp][at] = (uint16_t)(i0 + lane);
                count += __popc(hits);
            }
            __syncwarp();
            const int i = lane < count && lane < 32 ? listed[warp][lane] : -1;
            const int which = i >= 0 ? id[i] : -1 - lane;
            const bool alone_in_place = __popc(__match_any_sync(~0u, which)) == 1;
            if (count <= 32 && __all_sync(~0u, alone_in_place)) {
                if (i >= 0) Vec<T>::store(y + which, slow(xs[i]) - unit * (exp2_of((t[i] - r.teacher.m) * k) * z));
            } else {                                         // many, or some named twice: one after the other, with all that name it
                for (int i0 = 0; i0 < P.K; i0 += 32) {
                    const int e = i0 + lane < P.K ? id[i0 + lane] : -1;
                    unsigned hits = __ballot_sync(~0u, mine(e));
                    while (hits != 0) {
                        const int src = __ffs(hits) - 1, one = __shfl_sync(~0u, e, src);
                        hits &= hits - 1;
                        float p = 0.f;
                        bool before = false;                 // served already
                        for (int k0 = 0; k0 < P.K; k0 += 32)
                            if (k0 + lane < P.K && id[k0 + lane] == one) {
                                p += exp2_of((t[k0 + lane] - r.teacher.m) * k) * z;
                                before = before || k0 + lane < i0 + src;
                            }
                        p = warp_sum(p);
                        if (__any_sync(~0u, before)) continue;
                        if (lane == 0) Vec<T>::store(y + one, slow(xs[i0 + src]) - unit * p);
                    }
                }
            }
            __syncwarp();                                    // the list has been read
        }
        now = next;
    }
    if (leave && ranks > 1 && warp == 0) {                   // what the others send before they find this block gone
        const uint32_t bar = smem_at(&got[turns & 1]);
        if (lane == 0) asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"((ranks - 1) * 8) : "memory");
        chunk_wait(bar, (turns >> 1) & 1, 8 * kPolls);
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

template <typename T, int G, int NV> int launch_group(const DistillParams<T>& P, cudaStream_t s) {
    const int64_t blocks = (P.R * G + 255) / 256;
    if (blocks > (int64_t(1) << 31) - 1) return RLCS_ERR_SIZE;
    const int words = (P.A + 31) / 32;
    if (P.K <= 2 * G) distill_group_kernel<T, G, NV, 2><<<(unsigned)blocks, 256, 256 / G * words * 4, s>>>(P);
    else if (P.K <= 8 * G) distill_group_kernel<T, G, NV, 8><<<(unsigned)blocks, 256, 256 / G * words * 4, s>>>(P);
    else if constexpr (8 * G < kMostTop) distill_group_kernel<T, G, NV, 0><<<(unsigned)blocks, 256, 256 / G * (P.K + words) * 4, s>>>(P);      // at most 8 (1024 + 128) words
    return RLCS_OK;
}

// One cluster a row, as many as the GPU holds at once: asked for once a device, cluster size and size class of the teacher's
// entries (a cluster too many would start when the others have ended and double the time).
template <typename T, bool STAGED> int launch_block(const DistillParams<T>& P, int ranks, cudaStream_t s) {
    const auto kernel = distill_block_kernel<T, STAGED>;
    static int at_once[64][kMostRanks + 1][3];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RLCS_ERR_CUDA;
    const int kind = P.K <= 128 ? 0 : P.K <= 384 ? 1 : 2, most = kind == 0 ? 128 : kind == 1 ? 384 : kMostTop;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ranks);
    cfg.blockDim = dim3(kBlock);
    cfg.dynamicSmemBytes = (STAGED ? kPart : 0) + most * 24;
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ranks;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (at_once[dev][ranks][kind] == 0) {
        if (STAGED && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPart + kMostTop * 24) != cudaSuccess) return RLCS_ERR_CUDA;
        int n = 0;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) return RLCS_ERR_CUDA;
        at_once[dev][ranks][kind] = n;
    }
    const int64_t n = at_once[dev][ranks][kind];
    cfg.gridDim = dim3((unsigned)((P.R < n ? P.R : n) * ranks));
    return cudaLaunchKernelEx(&cfg, kernel, P) == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

template <typename T>
int distill_run(const T* logits, int64_t ld, const int32_t* ids, const float* teacher, const uint8_t* mask, float* loss, T* dlogits, int64_t ldd,
                int64_t R, int64_t A, int64_t K, float temperature, float scale, void* stream) {
    if (R < 0 || A < 0 || K < 0 || A > (int64_t(1) << 22) || K > kMostTop || R > (int64_t(1) << 40)) return RLCS_ERR_SIZE;
    if (R == 0) return RLCS_OK;
    if (A == 0 || ld < A || (dlogits != nullptr && ldd < A)) return RLCS_ERR_SIZE;
    if (ld > (int64_t(1) << 40) / R || ldd > (int64_t(1) << 40) / R) return RLCS_ERR_SIZE;
    if (!(temperature > 0.f) || !std::isfinite(temperature) || !std::isfinite(1.4426950408889634f / temperature) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (logits == nullptr || (K > 0 && (ids == nullptr || teacher == nullptr)) || (loss == nullptr && dlogits == nullptr)) return RLCS_ERR_NULL;
    const void* words[] = {ids, teacher, loss};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(logits, sizeof(T)) || !aligned_to(dlogits, sizeof(T))) return RLCS_ERR_ALIGN;
    const DistillParams<T> P = {logits, ids, teacher, mask, loss, dlogits, ld, ldd, R, (int32_t)A, (int32_t)K, 1.f / temperature,
                                1.4426950408889634f / temperature, scale, rlcs_hooks::g_wait_polls >= 0 ? rlcs_hooks::g_wait_polls : kPolls};
    const cudaStream_t s = static_cast<cudaStream_t>(stream);
    int st = RLCS_OK;
    if (const int64_t vecs = A / Vec<T>::N; vecs <= 512) {
        // As few lanes a row as hold it, and as few vectors a lane (us, bfloat16; fp32 is alike): 100000 rows of 19 8.1 with two lanes, 10 with
        // four; of 67 12 with four, 20 with eight; 50000 of 259 15 with eight and four vectors, 20 with eight vectors, 37 with a warp; of 515
        // 34 with eight lanes, 41 with a warp; 20000 of 1027 21 with four vectors, 27 with eight; 10000 of 2051 20 with eight, 27 with sixteen.  The
        // other way where entries are many (50000 of 515 with 64: 53 with eight lanes, 45 with a warp) or rows few (2000 of 403: 5.6, 3.9).  A warp
        // wherever a row has more than 64 entries: 50000 of 163 with 128 63 us, 90 with eight lanes (of 67 with 90 it is 419 and 381)
        if (vecs <= 2 && K <= 64) st = launch_group<T, 2, 2>(P, s);
        else if (vecs <= 8 && K <= 64) st = launch_group<T, 4, 2>(P, s);
        else if (vecs <= 32 && K <= 64) st = launch_group<T, 8, 4>(P, s);
        else if (vecs <= 64 && K <= 64) st = launch_group<T, 8, 8>(P, s);
        else if (vecs <= 128) st = launch_group<T, 32, 4>(P, s);
        else if (vecs <= 256) st = launch_group<T, 32, 8>(P, s);
        else st = launch_group<T, 32, 16>(P, s);
    } else if (vecs <= 2048 && R >= 2 * rlcs_device::limits().sms) {
        // a block a row: 29245 rows of 11 KB 169 us, 320 from shared memory; 3000 of 8003 in bfloat16 26 (34 with eight vectors a thread, 44 from
        // shared memory), 2000 of 16003 30 (38).  A warp a row up to 512 vectors: 5000 of 4099 21, 35 with a block.  Fewer rows are cut over clusters
        st = vecs <= 1024 ? launch_group<T, 256, 4>(P, s) : launch_group<T, 256, 8>(P, s);
    } else {
        // blocks a row: parts of at most 64 KB; more while the GPU has room for two a multiprocessor and a part keeps 8 KB
        const int64_t bytes = A * (int64_t)sizeof(T);
        int ranks = 1;
        while (ranks < kMostRanks && (bytes > (int64_t)ranks * kPart || (R * ranks < 2 * rlcs_device::limits().sms && bytes / (2 * ranks) >= 8192)))
            ranks *= 2;
        st = bytes <= (int64_t)ranks * kPart ? launch_block<T, true>(P, ranks, s) : launch_block<T, false>(P, ranks, s);
    }
    if (st != RLCS_OK) return st;
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

int rlcs_distill_grad(const float* logits, int64_t ld, const int32_t* teacher_ids, const float* teacher_logits, const uint8_t* mask, float* loss,
                      float* dlogits, int64_t ldd, int64_t R, int64_t A, int64_t K, float temperature, float scale, void* cuda_stream) {
    return distill_run<float>(logits, ld, teacher_ids, teacher_logits, mask, loss, dlogits, ldd, R, A, K, temperature, scale, cuda_stream);
}

int rlcs_distill_grad_bf16(const uint16_t* logits, int64_t ld, const int32_t* teacher_ids, const float* teacher_logits, const uint8_t* mask,
                           float* loss, uint16_t* dlogits, int64_t ldd, int64_t R, int64_t A, int64_t K, float temperature, float scale,
                           void* cuda_stream) {
    return distill_run<bf16>(reinterpret_cast<const bf16*>(logits), ld, teacher_ids, teacher_logits, mask, loss, reinterpret_cast<bf16*>(dlogits),
                             ldd, R, A, K, temperature, scale, cuda_stream);
}

}  // extern "C"

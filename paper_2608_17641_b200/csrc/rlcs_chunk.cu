// Attention of chunks of new tokens over a paged cache that holds them already.
//
//   token i of trajectory b's chunk of n_b:  p_i = lens_b - n_b + i,  c_j = scale q_i . k_j  for j <= p_i
//   o_i = sum_j exp(c_j) v_j / sum_j exp(c_j),   lse_i = log sum_j exp(c_j)
//
// The tokens of a chunk and the heads that share a key head are the rows of one tile: row x is token x / r, head x % r.
#include "rlcs_attention.cuh"

namespace {

using namespace rlcs_attn;

struct ChunkParams {
    AttnParams a;                  // B: tokens of the step; block_table, lens: of the trajectories
    const int32_t* offsets;        // [seqs + 1]
    int seqs, max_new;
    int tiles;                     // of 16 rows, a trajectory; 0: blocks of 128 rows
    int slots;                     // of blocks of 128 rows over all trajectories
    uint32_t r_mul;                // ceil(2^32 / r); 0 for r = 1
    int boxes;                     // whether a block's queries come, and its outputs leave, as boxes of whole tokens
};

struct Chunk {
    int first, count, start;       // first token of the step, tokens, place of the first in its trajectory (may be negative)
    int all;                       // tokens before the cut to max_new
};

__device__ __forceinline__ Chunk chunk_of(const ChunkParams& C, int b) {
    Chunk c;
    c.first = clamp_to(C.offsets[b], 0, C.a.B);
    c.count = clamp_to(C.offsets[b + 1], c.first, C.a.B) - c.first;
    c.start = clamp_to(C.a.lens[b], 0, 0x7fffff00) - c.count;      // no sum with rows of a tile wraps
    c.all = c.count;
    c.count = min(c.count, C.max_new);
    return c;
}

// Keys that the rows below `rows` of a chunk see, at most.
__device__ __forceinline__ int keys_of(const ChunkParams& C, const Chunk& c, int rows) {
    return clamp_to(c.start + (rows + C.a.r - 1) / C.a.r, 0, C.a.max_len);
}

__device__ __forceinline__ int divide_up_device(int a, int b) { return (a + b - 1) / b; }

template <int D, bool TMA>
__global__ void __launch_bounds__(kThreads)
chunk_kernel(const __grid_constant__ ChunkParams C, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    extern __shared__ char raw[];
    __shared__ int ids[kMaxIds + kTile];
    __shared__ __align__(8) uint64_t bars[4 * OwnShape<D>::kStages];
    __shared__ int gave_up;
    const AttnParams& P = C.a;
    int64_t block = blockIdx.x;
    const int tile = (int)(block % C.tiles);
    block /= C.tiles;
    const int kv_head = (int)(block % P.Hk);
    block /= P.Hk;
    const int b = (int)(block % C.seqs), seg = (int)(block / C.seqs);
    const Chunk c = chunk_of(C, b);
    const int rows = c.count * P.r, first_row = tile * 16;
    if (first_row >= rows) return;
    const int begin = seg * P.own_seg, end = min(begin + P.own_seg, keys_of(C, c, min(first_row + 16, rows)));
    if (begin >= end) {
        if (P.own_segs <= 1)                                      // rows without keys, which nobody joins
            for (int i = threadIdx.x; i < min(16, rows - first_row) * (P.d / 8); i += kThreads) {
                const int row = first_row + i / (P.d / 8);
                const int64_t at = (int64_t)(c.first + row / P.r) * P.H + kv_head * P.r + row % P.r;
                *reinterpret_cast<uint4*>(P.out + at * P.d + i % (P.d / 8) * 8) = make_uint4(0, 0, 0, 0);
                if (i % (P.d / 8) == 0 && P.lse != nullptr) P.lse[at] = -INFINITY;
            }
        return;
    }
    segment<D, TMA, true>(P, &k_map, &v_map, raw, ids, bars, &gave_up, P.block_table + (int64_t)b * P.own_width, P.own_width, begin, end, kv_head,
                          first_row, rows, c.first, seg, c.start + 1 - begin);
}

// ---------------------------------------------------------------------------------------------- chunks of more than 16 rows
// A tile of 128 rows a block on tcgen05, 64 keys a step.  Scores go into one of two 64-column buffers of tensor memory, the weights
// back over them as two bfloat16 parts (32 columns each), O += P V is accumulated in tensor memory.  Four warps have one row a thread (maximum,
// exponentials, sums).  Two warps issue the products, one the scores and one the values: the scores of the next step are there when the
// weights of this one leave.  Two warps copy keys and values through the page table into a ring of slots, as TMA boxes where pages
// divide 64 keys into parts of at least eight rows or are whole tiles, piece by piece otherwise.  Two blocks share a
// multiprocessor, so that one's start (lookups, queries) and end run under the other's products.
//
// The weights' two parts hold 16 bits, as those of the 16-row tiles do: a token comes out the same, but for the order of fp32 sums, whatever
// else is in its step.  The second part is half as many value products again, 8 to 21 % of the time (7 prompts 341 us with one part, long context
// 458, drafts 158); one rounding, 2^-8 of each weight, would be an error as large as the output's own.
//
// Where the heads on a key head divide 128, a block's queries come, and its outputs leave, as boxes of whole tokens: sixteen loads a thread
// took 2.6 us under the other block's exponentials.
//
// Bound by shared memory: a step's scores read 48 KB (queries and keys), its values 32, its copies write 32, for two blocks 224 KB or 1790
// cycles of 128 bytes, against 1536 cycles of products and 1024 of exponentials; a step takes about 2000.  Measured (heads of 128): 7 prompts
// of up to 4096 tokens, 32 heads on 8, 385 us for 321 GFLOP (0.50 of the bf16 rate); 1000 tokens behind 32768, 28 on 4, 557 us for
// 477 GFLOP (0.52); 64 chunks of up to 8 tokens behind 4096 171 us (0.73 of the copy bandwidth).  Not kept, measured with one part: two row tiles a block that share
// their keys, one block a multiprocessor (377, 488 us, and 216 for the chunks of drafts: nothing runs under a block's start and end); 128 keys a step into a single
// buffer (467, 516: scores, weights and values in turn, some 250 cycles at every barrier); a quarter of the exponentials by polynomial
// (no change); blocks of 126 rows where 7 heads share a key head, to have their boxes (500: one tile more is a round of blocks more).
constexpr int kKeys = 64, kRows = 128, kWideThreads = 256, kCopiers = 64, kMostSegment = 65536;

// Boxes of queries and outputs [T, H, d].
__device__ __forceinline__ void box_load3(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

__device__ __forceinline__ void box_store3(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// Products and commits are issued by one thread of a warp: elected once, it waits and issues by itself, which takes a third of the
// time at each barrier that a whole warp with an election an instruction takes.
__device__ __forceinline__ bool one_lane() {
    uint32_t r;
    asm volatile("{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\nselp.u32 %0, 1, 0, e;\n}" : "=r"(r));
    return r != 0;
}

__device__ __forceinline__ void issue_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

__device__ __forceinline__ void issue_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, int add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"(add) : "memory");
}

__device__ __forceinline__ void issue_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, int add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"(add) : "memory");
}

template <int D> struct WideShape {
    static constexpr int kSlot = kKeys * D * 2, kSlots = D == 128 ? 4 : 8, kQ = kRows * D * 2;
    static constexpr int kBytes = kQ + kSlots * kSlot + 1024;          // + alignment
};

struct WideTile {
    int b, first_row;              // b: -1 where the slot has no rows
    Chunk c;
    int held;                      // tokens of the trajectory: what of its memory may be read
};

// Which rows a slot has, for one warp: blocks with many keys first, so that the last to start are short.  Up to 128 trajectories
// go by the tile's place in its chunk (level by level from the highest), more by trajectory.
__device__ __forceinline__ WideTile wide_tile(const ChunkParams& C, int slot, int lane) {
    WideTile t;
    t.b = -1;
    auto tiles_of = [&](const Chunk& c) { return (int)(((int64_t)c.count * C.a.r + kRows - 1) / kRows); };
    if (C.seqs <= 128) {
        Chunk c[4];
        int n[4], most = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            c[q] = Chunk{0, 0, 0, 0};
            if (q * 32 + lane < C.seqs) c[q] = chunk_of(C, q * 32 + lane);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            n[q] = tiles_of(c[q]);
            most = max(most, n[q]);
        }
        most = __reduce_max_sync(~0u, most);
        auto from = [&](int level) {                              // tiles at or above a level
            int sum = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) sum += max(n[q] - level, 0);
            return __reduce_add_sync(~0u, sum);
        };
        if (slot >= from(0)) return t;
        int lo = 0, hi = most - 1;                                // the highest level with more than `slot` tiles at or above it
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (from(mid) > slot) lo = mid; else hi = mid - 1;
        }
        int rank = slot - from(lo + 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned some = __ballot_sync(~0u, n[q] > lo);
            if (t.b < 0 && rank < __popc(some)) {
                const int at = (int)__fns(some, 0, rank + 1);
                t.b = q * 32 + at;
                t.c = Chunk{__shfl_sync(~0u, c[q].first, at), __shfl_sync(~0u, c[q].count, at), __shfl_sync(~0u, c[q].start, at),
                            __shfl_sync(~0u, c[q].all, at)};
            }
            rank -= __popc(some);
        }
        t.first_row = lo * kRows;
    } else {
        // trajectory b's tiles start at slot floor(offset_b r / kRows) + b: at least as many slots as tiles for any sizes
        int lo = 0, hi = C.seqs - 1;
        auto first_slot = [&](int b) { return (int)((int64_t)clamp_to(C.offsets[b], 0, C.a.B) * C.a.r / kRows) + b; };
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (first_slot(mid) <= slot) lo = mid; else hi = mid - 1;
        }
        t.c = chunk_of(C, lo);
        const int at = slot - first_slot(lo), n = tiles_of(t.c);
        if (at < 0 || at >= n) return t;
        t.b = lo;
        t.first_row = (n - 1 - at) * kRows;
    }
    t.held = max(t.c.start + t.c.all, 0);
    return t;
}

template <int D, bool TMA>
__global__ void __launch_bounds__(kWideThreads, 2)
wide_kernel(const __grid_constant__ ChunkParams C, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
            const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap out_map) {
    typedef WideShape<D> Shape;
    constexpr int kSlots = Shape::kSlots, kPieces = D / 8;
    constexpr uint32_t kScores = 1u << 4 | 1u << 7 | 1u << 10 | (kKeys >> 3) << 17 | (128 >> 4) << 24;
    constexpr uint32_t kValues = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 16 | (D >> 3) << 17 | (128 >> 4) << 24;      // V: keys by rows
    extern __shared__ char raw[];
    __shared__ int ids[kMaxIds + kKeys + 8];
    __shared__ __align__(8) uint64_t bars[2 * kSlots + 8];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up, missing_any;
    __shared__ WideTile which;
    const AttnParams& P = C.a;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t q_at = (smem_at(raw) + 1023) & ~1023u, ring = q_at + Shape::kQ;
    const uint32_t full = smem_at(bars), empty = full + 8 * kSlots, drained = empty + 8 * kSlots;
    const uint32_t s_full = drained + 8, p_full = s_full + 16, o_done = p_full + 16, q_full = o_done + 16;      // two each, taken in turn
    const int kv_head = (int)(blockIdx.x / C.slots) % P.Hk, seg = (int)(blockIdx.x / C.slots) / P.Hk;
    if (warp == 0) {
        const WideTile w = wide_tile(C, (int)(blockIdx.x % C.slots), lane);
        if (lane == 0) which = w;
    } else if (warp == 5) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_at)), "n"(256) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else if (tid == 32) {
        gave_up = missing_any = 0;
        for (int i = 0; i < kSlots; ++i) { bar_init(full + 8 * i, TMA ? 1 : kCopiers); bar_init(empty + 8 * i, 1); }
        for (int i = 0; i < 2; ++i) { bar_init(s_full + 8 * i, 1); bar_init(p_full + 8 * i, 128); bar_init(o_done + 8 * i, 1); }
        bar_init(q_full, C.boxes ? 1 : 128);
        bar_init(drained, 2);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = tmem_at;
    const int b = which.b, first_row = which.first_row, held = which.held;
    const Chunk c = which.c;
    const int mine_rows = min(kRows, c.count * P.r - first_row);      // the block's
    const int begin = seg * P.own_seg, end = b < 0 ? begin : min(begin + P.own_seg, keys_of(C, c, first_row + mine_rows));
    const bool whole_row = P.own_segs <= 1;                       // outputs leave at once, not as parts to be joined
    const int tiles = divide_up_device(end - begin, kKeys);
    const int offset = begin % P.page;
    // the block's rows, counted from its first: tokens and heads
    const int token0 = first_row / P.r, head0 = first_row % P.r;
    auto token_of = [&](int k) { return C.r_mul != 0 ? (int)__umulhi((uint32_t)(head0 + k), C.r_mul) : k; };      // from token0 on; (r + 256) r < 2^32
    if (begin >= end) {
        if (b >= 0 && whole_row && seg == 0)
            for (int i = tid; i < mine_rows * (P.d / 8); i += kWideThreads) {
                const int row = first_row + i / (P.d / 8);
                const int64_t at = (int64_t)(c.first + row / P.r) * P.H + kv_head * P.r + row % P.r;
                *reinterpret_cast<uint4*>(P.out + at * P.d + i % (P.d / 8) * 8) = make_uint4(0, 0, 0, 0);
                if (i % (P.d / 8) == 0 && P.lse != nullptr) P.lse[at] = -INFINITY;
            }
    } else
    if (warp < 4) {
        const int row = warp * 32 + lane;                         // of the block's
        const uint32_t mine = tmem + ((uint32_t)(warp * 32) << 16), o_at = mine + 128;
        const bool any_row = warp * 32 < mine_rows;
        const int lim = row < mine_rows ? clamp_to(min(c.start + token0 + token_of(row) + 1, P.max_len) - begin, 0, end - begin) : end - begin;
        const int least = __reduce_min_sync(~0u, lim);
        const int64_t rows_at = (int64_t)(c.first + token0) * P.H + kv_head * P.r;      // of the outputs [T, H]
        auto row_at = [&](int k) { return rows_at + (int64_t)token_of(k) * P.H + (head0 + k - token_of(k) * P.r); };
        if (!C.boxes) {
            // the warp's queries, zeros where there are none: kPieces lanes a row
            constexpr int kLoads = kPieces, kTogether = 32 / kPieces;
            uint4 v[kLoads];
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int k = warp * 32 + j * kTogether + lane / kPieces, piece = lane % kPieces, token = token_of(k);
                v[j] = make_uint4(0, 0, 0, 0);
                if (k < mine_rows && piece * 8 < P.d)
                    v[j] = *reinterpret_cast<const uint4*>(P.q + (int64_t)(c.first + token0 + token) * P.q_stride + (int64_t)(kv_head * P.r + head0 + k - token * P.r) * P.d + piece * 8);
            }
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                const int k = warp * 32 + j * kTogether + lane / kPieces, piece = lane % kPieces;
                const uint32_t dst = q_at + (piece >> 3) * (128 * 128) + k * 128 + (((piece & 7) ^ (k & 7)) << 4);
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(v[j].x), "r"(v[j].y), "r"(v[j].z), "r"(v[j].w) : "memory");
            }
            fence_async();
            bar_arrive(q_full);
        }
        bool missing = false;
        float m = -INFINITY, l = 0.f;
        bool fine = true;
        for (int i = 0; i < tiles; ++i) {
            const uint32_t s_at = mine + (i & 1) * kKeys;
            fine = __all_sync(~0u, bar_wait(s_full + 8 * (i & 1), (i >> 1) & 1, &gave_up, P.polls));
            if (!fine) break;
            fence_after();
            if (i == 0) missing = *(volatile int*)&missing_any != 0;      // written before the first key was fetched
            if (any_row) {
                uint32_t s[kKeys];
#pragma unroll
                for (int k = 0; k < kKeys; k += 32) tmem_load32(s + k, s_at + k);
                tmem_wait_load();
                if ((i + 1) * kKeys > least || missing) {
                    const int left = lim - i * kKeys;
#pragma unroll
                    for (int k = 0; k < kKeys; ++k) {
                        const bool there = k < left && (!missing || ids[page_of(P, offset + i * kKeys + k)] >= 0);
                        if (!there) s[k] = __float_as_uint(-INFINITY);
                    }
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < kKeys; k += 8)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[e] = fmaxf(fmaxf(top[e], __uint_as_float(s[k + 2 * e])), __uint_as_float(s[k + 2 * e + 1]));
                const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * P.scale_log2;
                // the base follows the maximum only when it is 2^8 behind: the weights stay below 2^8, and O is seldom rescaled
                if (__any_sync(~0u, now > m + 8.f)) {
                    const float next = fmaxf(m, now), fade = m == -INFINITY ? 0.f : exp2_of(m - next);
                    if (i > 0) {
                        fine = __all_sync(~0u, bar_wait(o_done + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, &gave_up, P.polls));
                        if (!fine) break;
                        fence_after();
#pragma unroll
                        for (int k = 0; k < D; k += 16) {
                            uint32_t o[16];
                            tmem_load16(o, o_at + k);
                            tmem_wait_load();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * fade);
                            tmem_store16(o_at + k, o);
                        }
                    }
                    l *= fade;
                    m = next;
                }
                const float base = m == -INFINITY ? 0.f : m;
                const float2 scale = {P.scale_log2, P.scale_log2}, less = {-base, -base};
                float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                for (int part = 0; part < 2; ++part) {
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float2 p = fma2(make_float2(__uint_as_float(s[part * 32 + 2 * k]), __uint_as_float(s[part * 32 + 2 * k + 1])), scale, less);
                        p = make_float2(exp2_of(p.x), exp2_of(p.y));
                        sum[k & 1] = add2(sum[k & 1], p);
                        hi[k] = pack2(p.x, p.y);
                        p = fma2(make_float2(__uint_as_float(hi[k] << 16), __uint_as_float(hi[k] & 0xffff0000u)), make_float2(-1.f, -1.f), p);
                        lo[k] = pack2(p.x, p.y);
                    }
                    tmem_store16(s_at + part * 16, hi);
                    tmem_store16(s_at + kKeys / 2 + part * 16, lo);
                }
                l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
                tmem_wait_store();
            }
            fence_before();
            bar_arrive(p_full + 8 * (i & 1));
        }
        if (any_row) {
            for (int i = max(tiles - 2, 0); i < tiles && fine; ++i)
                fine = __all_sync(~0u, bar_wait(o_done + 8 * (i & 1), (i >> 1) & 1, &gave_up, P.polls));
            fine = fine && *(volatile int*)&gave_up == 0;         // a thread that copies may have given up alone
            fence_after();
            if (!fine) l = __int_as_float(0x7fffffff);
        }
        if (C.boxes && whole_row && mine_rows == kRows) {
            // whole tokens leave as boxes, through the place of the queries, which are done with; in their layout
            const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
            for (int k = 0; k < D; k += 32) {
                uint32_t o[32];
                tmem_load32(o, o_at + k);
                tmem_wait_load();
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t w[4];
                    const int piece = (k + e) / 8;
#pragma unroll
                    for (int h = 0; h < 4; ++h) w[h] = l == 0.f ? 0u : pack2(__uint_as_float(o[e + 2 * h]) * inv, __uint_as_float(o[e + 2 * h + 1]) * inv);
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(q_at + (piece >> 3) * (128 * 128) + row * 128 + (((piece & 7) ^ (row & 7)) << 4)),
                                 "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]) : "memory");
                }
            }
            fence_async();
            asm volatile("bar.sync 3, 128;" ::: "memory");
            if (tid == 0) {
#pragma unroll
                for (int half = 0; half < D / 64; ++half)
                    box_store3(&out_map, q_at + half * (128 * 128), half * 64, kv_head * P.r, c.first + token0);
                asm volatile("cp.async.bulk.commit_group;\ncp.async.bulk.wait_group.read 0;" ::: "memory");
            }
            if (row < mine_rows && P.lse != nullptr) P.lse[row_at(row)] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        } else if (any_row) {
            // rows leave through the place of the warp's queries, 256 bytes of a row at a time, written by the row's thread, stored by sixteen
            // lanes a row
            const float inv = l != 0.f ? 1.f / l : 0.f;
            const uint32_t mine_at = q_at + warp * (Shape::kQ / 4);
            constexpr int kRound = D == 128 ? 16 : 8;                 // 16-byte pieces of a row a round: D values of 16 bits, D / 2 of 32
            char* const parts = reinterpret_cast<char*>(P.part_o + (int64_t)seg * P.B * P.H * D);
            const int rounds = whole_row ? 1 : 2;
            for (int round = 0; round < rounds; ++round) {
                __syncwarp();
#pragma unroll
                for (int k = 0; k < D; k += 32) {
                    if (!whole_row && k / (D / 2) != round) continue;
                    uint32_t o[32];
                    tmem_load32(o, o_at + k);
                    tmem_wait_load();
                    auto put = [&](int piece, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
                        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(mine_at + lane * (kRound * 16) + ((piece ^ (lane & (kRound - 1))) << 4)), "r"(x),
                                     "r"(y), "r"(z), "r"(w) : "memory");
                    };
                    if (whole_row) {
#pragma unroll
                        for (int e = 0; e < 32; e += 8) {
                            uint32_t w[4];
#pragma unroll
                            for (int h = 0; h < 4; ++h) w[h] = l == 0.f ? 0u : pack2(__uint_as_float(o[e + 2 * h]) * inv, __uint_as_float(o[e + 2 * h + 1]) * inv);
                            put((k + e) / 8, w[0], w[1], w[2], w[3]);
                        }
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; e += 4) put((k % (D / 2) + e) / 4, o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                }
                __syncwarp();
#pragma unroll
                for (int j = 0; j < kRound; ++j) {
                    const int k = j * (32 / kRound) + lane / kRound, piece = lane % kRound;
                    uint4 v;
                    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                                 : "r"(mine_at + k * (kRound * 16) + ((piece ^ (k & (kRound - 1))) << 4)) : "memory");
                    if (warp * 32 + k >= mine_rows) continue;
                    const int64_t at = row_at(warp * 32 + k);
                    if (!whole_row) *reinterpret_cast<uint4*>(parts + at * (D * 4) + round * (D * 2) + piece * 16) = v;
                    else if (piece * 8 < P.d) *reinterpret_cast<uint4*>(P.out + at * P.d + piece * 8) = v;
                }
            }
            if (row < mine_rows) {
                const int64_t at = row_at(row);
                if (!whole_row) P.part_ml[(int64_t)seg * P.B * P.H + at] = fine ? make_float2(m, l) : make_float2(0.f, l);
                else if (P.lse != nullptr) P.lse[at] = l != 0.f ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
            }
        }
        fence_before();
    } else {
        if (C.boxes && tid == 128) {                              // queries; rows behind the chunk's are somebody else's and come to nothing
            bar_expect(q_full, (D / 64) * kRows * 128);
#pragma unroll
            for (int half = 0; half < D / 64; ++half)
                box_load3(q_at + half * (128 * 128), &q_map, q_full, half * 64, kv_head * P.r, c.first + token0);
        }
        // page numbers of the keys, by the four warps that are left; -1: no such page
        {
            const int32_t* table = P.block_table + (int64_t)b * P.own_width;
            const int first = begin / P.page, count = (min(begin + tiles * kKeys, held) - 1) / P.page - first + 1;
            bool some = false;
#pragma unroll 4
            for (int i = tid - 128; i < count; i += 128) {
                int id = first + i < P.own_width ? table[first + i] : -1;
                if (id < 0 || id >= P.pages) { id = -1; some = true; }
                ids[i] = id;
            }
            if (some) missing_any = 1;
            asm volatile("bar.sync 2, %0;" ::"n"(128) : "memory");
        }
        if (warp == 4 || warp == 7) {
            const int me = (warp == 4 ? 0 : 32) + lane, piece = me % kPieces, row0 = me / kPieces;
            constexpr int kStep = kCopiers / kPieces, kEach = kKeys / kStep;
            const uint32_t lane_at = ring + (piece >> 3) * (kKeys * 128);
            auto pieces = [&](int item) {                         // one tile of keys or values, zeros where there is no key
                const __nv_bfloat16* from = (item & 1 ? P.v : P.k) + kv_head * P.head_stride + piece * 8;
                const uint32_t dst = lane_at + (item % kSlots) * Shape::kSlot;
#pragma unroll 4
                for (int k = 0; k < kEach; ++k) {
                    const int row = row0 + k * kStep, local = (item >> 1) * kKeys + row;
                    int64_t place = 0;
                    bool there = begin + local < held && piece * 8 < P.d;
                    if (there) {
                        const int in = offset + local, pg = page_of(P, in), id = ids[pg];
                        there = id >= 0;
                        if (there) place = id * P.page_stride + (in - pg * P.page) * P.token_stride;
                    }
                    copy16(dst + row * 128 + (((piece & 7) ^ (row & 7)) << 4), from + place, there);
                }
            };
            auto room = [&](int item) { return item < kSlots || bar_wait(empty + 8 * (item % kSlots), (item / kSlots - 1) & 1, &gave_up, P.polls); };
            bool fine = true;
            if constexpr (TMA) {
                // all but the tile in which the trajectory ends: what lies behind its last value may be anything
                const int whole = min(tiles, (held - begin) / kKeys), box = P.page < kKeys ? P.page : kKeys;
                int issued = 0;
                if (me == 0)
                    for (int i = 0; i < 2 * whole && fine; ++i) {
                        fine = room(i);
                        if (!fine) break;
                        const uint32_t bar = full + 8 * (i % kSlots), dst = ring + (i % kSlots) * Shape::kSlot;
                        issued = i + 1;
                        bar_expect(bar, Shape::kSlot);
                        for (int row = 0; row < kKeys; row += box) {
                            const int in = offset + (i >> 1) * kKeys + row, pg = page_of(P, in);
#pragma unroll
                            for (int half = 0; half < D / 64; ++half)     // a page number of -1 lies outside the map: zeros
                                box_load(dst + half * (kKeys * 128) + row * 128, i & 1 ? &v_map : &k_map, bar, half * 64, in - pg * P.page, kv_head, ids[pg]);
                        }
                    }
                if (whole < tiles) {
                    asm volatile("bar.sync 1, %0;" ::"n"(kCopiers) : "memory");
                    for (int i = 2 * whole; i < 2 * whole + 2 && fine; ++i) {
                        fine = room(i);
                        if (fine) pieces(i);
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_async();
                    asm volatile("bar.sync 1, %0;" ::"n"(kCopiers) : "memory");
                    if (me == 0 && fine) {
                        bar_arrive(full + 8 * (2 * whole % kSlots));
                        bar_arrive(full + 8 * ((2 * whole + 1) % kSlots));
                    }
                }
                // no boxes in flight when the block ends, whoever gave up (where the partial tile's slots were free, theirs had arrived)
                int late = 0;
                for (int i = max(0, issued - kSlots + (fine && whole < tiles ? 2 : 0)); i < issued; ++i)
                    bar_wait(full + 8 * (i % kSlots), (i / kSlots) & 1, &late, kPolls);
            } else {
                for (int i = 0; i < 2 * tiles && fine; ++i) {
                    fine = room(i);
                    if (!fine) break;
                    pieces(i);
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    fence_async();
                    bar_arrive(full + 8 * (i % kSlots));
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (C.boxes && me == 0) {
                int late = 0;
                bar_wait(q_full, 0, &late, kPolls);
            }
        } else {
            const uint32_t base = __shfl_sync(~0u, tmem, 0);
            if (one_lane()) {
                auto wait = [&](uint32_t bar, int parity) { return bar_wait(bar, parity & 1, &gave_up, P.polls); };
                bool fine = true;
                if (warp == 5) {
                    const uint64_t q_desc = describe(q_at, 16), k_desc = describe(ring, 16);
                    fine = wait(q_full, 0);
                    for (int i = 0; i < tiles && fine; ++i) {
                        const int item = 2 * i, slot = item % kSlots;
                        fine = wait(full + 8 * slot, item / kSlots);
                        if (!fine) break;
                        // the buffer's weights must have been multiplied before new scores go there
                        fine = i < 2 || wait(o_done + 8 * (i & 1), (i - 2) >> 1);
                        if (!fine) break;
                        fence_after();
                        const uint64_t k_at = k_desc + slot * (Shape::kSlot >> 4);
#pragma unroll
                        for (int s = 0; s < D / 16; ++s)
                            issue_ss(base + (i & 1) * kKeys, q_desc + (((s >> 2) * (128 * 128) + (s & 3) * 32) >> 4),
                                     k_at + (((s >> 2) * (kKeys * 128) + (s & 3) * 32) >> 4), kScores, s > 0);
                        issue_commit(s_full + 8 * (i & 1));
                        issue_commit(empty + 8 * slot);
                    }
                } else {
                    const uint64_t v_desc = describe(ring, kKeys * 128);
                    for (int i = 0; i < tiles && fine; ++i) {
                        const int item = 2 * i + 1, slot = item % kSlots;
                        fine = wait(full + 8 * slot, item / kSlots);
                        if (!fine) break;
                        fine = wait(p_full + 8 * (i & 1), i >> 1);
                        if (!fine) break;
                        fence_after();
                        const uint64_t v_at = v_desc + slot * (Shape::kSlot >> 4);
#pragma unroll
                        for (int s = 0; s < kKeys / 16; ++s)
#pragma unroll
                            for (int part = 0; part < 2; ++part)
                                issue_ts(base + 128, base + (i & 1) * kKeys + part * (kKeys / 2) + s * 8, v_at + ((s * 2048) >> 4), kValues, i > 0 || s > 0 || part > 0);
                        issue_commit(o_done + 8 * (i & 1));
                        issue_commit(empty + 8 * slot);
                    }
                }
                issue_commit(drained);                            // nothing in flight when the memory is given back
                int late = 0;
                bar_wait(drained, 0, &late, kPolls);
            }
        }
    }
    __syncwarp();
    __syncthreads();
    if (warp == 5) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(256) : "memory");
    }
}

// Joins a row's segments: one warp a (token, head).
template <int D>
__global__ void __launch_bounds__(kThreads) chunk_join_kernel(const __grid_constant__ ChunkParams C) {
    constexpr int kPer = D / 32;
    const AttnParams& P = C.a;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), all = (int64_t)P.B * P.H;
    const int lane = threadIdx.x & 31;
    if (at >= all) return;
    const int token = (int)(at / P.H);
    int lo = 0, hi = C.seqs - 1;                              // the last trajectory that starts at or before the token
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (C.offsets[mid] <= token) lo = mid; else hi = mid - 1;
    }
    const Chunk c = chunk_of(C, lo);
    if (token < c.first || token >= c.first + c.count) return;
    const int segs = (clamp_to(c.start + token - c.first + 1, 0, P.max_len) + P.own_seg - 1) / P.own_seg;
    float top = -INFINITY, sum = 0.f, o[kPer] = {};
    for (int i = 0; i < segs; ++i) {
        const int64_t row = (int64_t)i * all + at;
        const float2 ml = P.part_ml[row];
        if (!(ml.y > 0.f) && ml.y == ml.y) continue;          // nothing there
        const float now = fmaxf(top, ml.x), f0 = exp2_of(top - now), f1 = exp2_of(ml.x - now);
        top = now;
        sum = sum * f0 + ml.y * f1;
#pragma unroll
        for (int k = 0; k < kPer; ++k) o[k] = o[k] * f0 + P.part_o[row * D + lane * kPer + k] * f1;
    }
    const float inv = sum != 0.f ? 1.f / sum : 0.f;
#pragma unroll
    for (int k = 0; k < kPer; k += 2)
        if (lane * kPer + k < P.d)
            *reinterpret_cast<uint32_t*>(P.out + at * P.d + lane * kPer + k) = pack2(o[k] * inv, o[k + 1] * inv);
    if (lane == 0 && P.lse != nullptr) P.lse[at] = sum != 0.f ? (top + log2f(sum)) * 0.6931471805599453f : -INFINITY;
}

// Wide blocks run `slots` at once: whole rows while there are two rounds of blocks or more, else the number of segments that makes
// the rounds shortest, a segment costing about eight steps beyond its own (start, first loads, the partial result and its joining).
int plan_wide(int64_t longest, int64_t units, int page, int64_t slots) {
    const int64_t by_ids = (int64_t)(kMaxIds - 2) * page / kKeys * kKeys, most = (by_ids < kMostSegment ? by_ids : kMostSegment) / kKeys;
    const int64_t tiles = divide_up(longest > 0 ? longest : 1, kKeys);
    int64_t best = most, cost = INT64_MAX;
    for (int64_t segs = divide_up(tiles, most); segs <= tiles && segs <= 256; ++segs) {
        const int64_t per = divide_up(tiles, segs), c = divide_up(units * segs, slots) * (per + 8);
        if (c < cost) { cost = c; best = per; }
        if (units >= 2 * slots) break;
    }
    return (int)(best * kKeys);
}

// Sizes only: shared by the call and its workspace query.
int check_shape(ChunkParams& C, int64_t T, int64_t seqs, int64_t H, int64_t Hk, int64_t d, int64_t page, int64_t max_new, int64_t max_len) {
    AttnParams& P = C.a;
    const int64_t kMostLen = (int64_t(1) << 31) - 1 - 65536;
    if (T < 0 || seqs < 0 || H < 0 || Hk < 0 || max_new < 0 || max_len < 0 || page < 1) return RLCS_ERR_SIZE;
    if (T > (1 << 24) || seqs > (1 << 20) || H > 4096 || max_len > kMostLen || page > 32768) return RLCS_ERR_SIZE;
    if (d < 8 || d > 128 || d % 8 != 0) return RLCS_ERR_SIZE;
    if (H > 0 && (Hk == 0 || H % Hk != 0)) return RLCS_ERR_SIZE;
    P.B = (int)T;
    P.H = (int)H;
    P.Hk = (int)Hk;
    P.r = Hk > 0 ? (int)(H / Hk) : 0;
    P.d = (int)d;
    P.page = (int)page;
    P.max_len = (int)max_len;
    P.page_mul = page > 1 ? (uint32_t)(((uint64_t(1) << 32) + page - 1) / page) : 0;
    C.seqs = (int)seqs;
    C.r_mul = P.r > 1 ? (uint32_t)(((uint64_t(1) << 32) + P.r - 1) / P.r) : 0;
    C.max_new = (int)(max_new < T ? max_new : T);
    if (T == 0 || H == 0 || seqs == 0 || C.max_new == 0) return RLCS_OK;
    if ((int64_t)C.max_new * P.r > (1 << 30)) return RLCS_ERR_SIZE;
    // 16-row tiles for single tiles, and where all of them run at once on short contexts: 6 to 8 us against 10 to 20 of a block of 128 rows
    const int64_t narrow = divide_up((int64_t)C.max_new * P.r, 16);
    if (narrow == 1 || (P.max_len <= 768 && narrow * Hk * seqs <= 3 * rlcs_device::limits().sms)) {
        C.tiles = (int)narrow;
        // up to 768 keys one segment takes no longer than several and their joining (480 keys: 6 us against 9, and 5 us less host time)
        const int one = divide_up(P.max_len > 0 ? P.max_len : 1, kTile) * kTile;
        P.own_seg = one <= 768 && (one - 1) / P.page + 2 <= kMaxIds ? one : plan_segment(P.max_len, narrow * Hk * seqs, P.page, 1024);
    } else {
        const int64_t rows = T * P.r, some = seqs < T ? seqs : T, units = rows / kRows + (some + 1) / 2;
        C.slots = (int)(rows / kRows + seqs);
        P.own_seg = plan_wide(P.max_len, Hk * (units > some ? units : some), P.page, rlcs_device::limits().sms * 2);
    }
    P.own_segs = divide_up(P.max_len, P.own_seg);
    if ((double)(C.tiles > 0 ? C.tiles * seqs : C.slots) * Hk * (P.own_segs > 0 ? P.own_segs : 1) > 2147483647.0 || T * H > (int64_t(1) << 32)) return RLCS_ERR_SIZE;
    return RLCS_OK;
}

size_t workspace_of(const ChunkParams& C) {
    if (C.a.own_segs <= 1) return 0;
    const size_t rows = (size_t)C.a.own_segs * C.a.B * C.a.H;
    return rows * ((C.a.d <= 64 ? 64 : 128) + 2) * sizeof(float) + 16;
}

template <int D, bool TMA>
int launch_chunk(const ChunkParams& C, int64_t blocks, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s) {
    static bool granted[64];
    if (!grant(chunk_kernel<D, TMA>, OwnShape<D>::kBytes, granted)) return RLCS_ERR_CUDA;
    chunk_kernel<D, TMA><<<(unsigned)blocks, kThreads, OwnShape<D>::kBytes, s>>>(C, k_map, v_map);
    return RLCS_OK;
}

// Queries or outputs [T, H, d] as a map of boxes [whole tokens of a block, heads on a key head, 64 dimensions].
bool token_map(CUtensorMap* map, const ChunkParams& C, const void* base, int64_t stride) {
    const EncodeTiled encode = encode_tiled();
    if (encode == nullptr) return false;
    const cuuint64_t extent[3] = {(cuuint64_t)C.a.d, (cuuint64_t)C.a.H, (cuuint64_t)C.a.B};
    const cuuint64_t strides[2] = {(cuuint64_t)C.a.d * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)C.a.r, (cuuint32_t)(kRows / C.a.r)}, step[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), extent, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TMA>
int launch_wide(ChunkParams C, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s) {
    CUtensorMap q_map = {}, out_map = {};
    C.boxes = kRows % C.a.r == 0 && token_map(&q_map, C, C.a.q, C.a.q_stride) && token_map(&out_map, C, C.a.out, (int64_t)C.a.H * C.a.d);
    static bool granted[64];
    if (!grant(wide_kernel<D, TMA>, WideShape<D>::kBytes, granted)) return RLCS_ERR_CUDA;
    const int segs = C.a.own_segs > 0 ? C.a.own_segs : 1;         // rows without keys are written too
    wide_kernel<D, TMA><<<(unsigned)(C.slots * C.a.Hk * segs), kWideThreads, WideShape<D>::kBytes, s>>>(C, k_map, v_map, q_map, out_map);
    return RLCS_OK;
}

template <int D> int launch(const ChunkParams& C, cudaStream_t s) {
    CUtensorMap k_map = {}, v_map = {};
    const AttnParams& P = C.a;
    if (C.tiles == 0) {
        const bool boxes = box_map(&k_map, P, P.k, kKeys) && box_map(&v_map, P, P.v, kKeys);
        const int st = boxes ? launch_wide<D, true>(C, k_map, v_map, s) : launch_wide<D, false>(C, k_map, v_map, s);
        if (st != RLCS_OK || P.own_segs <= 1) return st != RLCS_OK ? st : cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
        chunk_join_kernel<D><<<(unsigned)divide_up((int64_t)P.B * P.H, kThreads / 32), kThreads, 0, s>>>(C);
        return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
    }
    const int64_t blocks = (int64_t)C.tiles * P.Hk * C.seqs * (P.own_segs > 0 ? P.own_segs : 1);      // rows without keys are written too
    // a few blocks on short contexts wait for the call, not for the copies: the maps of the boxes would be 1.6 us of host time for nothing
    const bool few = P.max_len <= 512 && blocks < rlcs_device::limits().sms;
    const bool boxes = !few && box_map(&k_map, P, P.k, kPart) && box_map(&v_map, P, P.v, kPart);
    const int st = boxes ? launch_chunk<D, true>(C, blocks, k_map, v_map, s) : launch_chunk<D, false>(C, blocks, k_map, v_map, s);
    if (st != RLCS_OK || P.own_segs <= 1) return st != RLCS_OK ? st : cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
    chunk_join_kernel<D><<<(unsigned)divide_up((int64_t)P.B * P.H, kThreads / 32), kThreads, 0, s>>>(C);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t rlcs_chunk_attention_workspace_bytes(int64_t T, int64_t B, int64_t H, int64_t Hk, int64_t d, int64_t page_size, int64_t max_new,
                                            int64_t max_len) {
    ChunkParams C = {};
    if (check_shape(C, T, B, H, Hk, d, page_size, max_new, max_len) != RLCS_OK || T == 0 || H == 0 || B == 0 || max_new == 0) return 0;
    return workspace_of(C);
}

int rlcs_chunk_attention_bf16(const uint16_t* q, int64_t q_stride, const uint16_t* k_cache, const uint16_t* v_cache, int64_t pages,
                              int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* block_table, int64_t width,
                              const int32_t* offsets, const int32_t* lens, uint16_t* out, float* lse, int64_t T, int64_t B, int64_t H,
                              int64_t Hk, int64_t d, int64_t page_size, int64_t max_new, int64_t max_len, float scale, void* workspace,
                              size_t workspace_bytes, void* cuda_stream) {
    ChunkParams C = {};
    AttnParams& P = C.a;
    const int st = check_shape(C, T, B, H, Hk, d, page_size, max_new, max_len);
    if (st != RLCS_OK) return st;
    if (pages < 0 || pages > (int64_t(1) << 31) - 1 || width < 0 || width > (1 << 30)) return RLCS_ERR_SIZE;
    if (T == 0 || H == 0 || B == 0 || max_new == 0) return RLCS_OK;
    if (q_stride < H * d || page_stride < 0 || token_stride < 0 || head_stride < 0) return RLCS_ERR_SIZE;
    if (!(scale > 0.f) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (q == nullptr || out == nullptr || lens == nullptr || offsets == nullptr) return RLCS_ERR_NULL;
    if (P.max_len > 0 && (k_cache == nullptr || v_cache == nullptr || (width > 0 && block_table == nullptr))) return RLCS_ERR_NULL;
    const void* words[] = {block_table, offsets, lens, lse};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(q, 16) || !aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || !aligned_to(out, 16)) return RLCS_ERR_ALIGN;
    if (q_stride % 8 || page_stride % 8 || token_stride % 8 || head_stride % 8) return RLCS_ERR_ALIGN;
    const size_t need = workspace_of(C);
    if (need > 0 && (workspace == nullptr || workspace_bytes < need)) return RLCS_ERR_WORKSPACE;
    if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    P.q = reinterpret_cast<const __nv_bfloat16*>(q);
    P.k = reinterpret_cast<const __nv_bfloat16*>(k_cache);
    P.v = reinterpret_cast<const __nv_bfloat16*>(v_cache);
    P.block_table = block_table;
    P.lens = lens;
    P.out = reinterpret_cast<__nv_bfloat16*>(out);
    P.lse = lse;
    P.q_stride = q_stride;
    P.page_stride = page_stride;
    P.token_stride = token_stride;
    P.head_stride = head_stride;
    P.pages = pages;
    P.own_width = (int)width;
    P.scale_log2 = scale * 1.4426950408889634f;
    P.polls = rlcs_hooks::g_wait_polls >= 0 ? rlcs_hooks::g_wait_polls : kPolls;
    C.offsets = offsets;
    const size_t rows = (size_t)P.own_segs * P.B * P.H;
    P.part_o = static_cast<float*>(workspace);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + rows * (P.d <= 64 ? 64 : 128));
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return P.d <= 64 ? launch<64>(C, s) : launch<128>(C, s);
}

}  // extern "C"

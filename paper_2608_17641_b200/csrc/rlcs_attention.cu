// Attention of one query a trajectory over a paged cache whose trajectories share their group's prompt.
//
//   keys of row b:  the prefix of its group (prefix_table, prefix_lens), then its own tokens (block_table, lens)
//   c_j = scale q . k_j,   o = sum_j exp(c_j) v_j / sum_j exp(c_j),   lse = log sum_j exp(c_j)
//
// A group's prefix is multiplied with all of the group's queries at once: the queries of all its rows and of the heads
// that share a key head are the rows of one tile.  A row's own tokens meet the heads that share a key head only.  Both
// run over key segments that leave (running maximum, sum, product) behind; a second kernel joins a row's segments.
//
// Bounds and measurements (B200, 32 heads on 8 key heads of 128): own tokens by HBM, 5.3 TB/s (0.82 of the copy bandwidth) at 128
// trajectories of up to 2048; a prefix of 32768 tokens against 256 trajectories by products, 200 us for 137 GFLOP (0.43 of the
// bf16 rate; the second part of the weights is a third of what the matrix unit does), 16 prefixes of 2048 against 8 each 34 us.
#include <cuda.h>
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"
#include "rlcs_pair.cuh"

namespace rlcs_hooks {
extern int g_wait_polls;      // rlcs_debug_set_wait_polls; defined in rlcs_api.cu
}

namespace {

using namespace rlcs_pair;

constexpr int kPolls = 1 << 20;                 // of a wait, before it gives up

struct AttnParams {
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    const int32_t* prefix_table;
    const int32_t* prefix_lens;
    const int32_t* group_offsets;
    const int32_t* block_table;
    const int32_t* lens;
    __nv_bfloat16* out;
    float* lse;
    float* part_o;                 // [segments, B, H, Dp]
    float2* part_ml;               // [segments, B, H]
    int64_t q_stride, page_stride, token_stride, head_stride, pages;
    int B, H, Hk, r, d, groups, prefix_width, own_width, page;
    uint32_t page_mul;             // ceil(2^32 / page); 0 for pages of one token
    int max_prefix, max_len;
    int prefix_seg, own_seg;       // keys a segment
    int prefix_segs, own_segs;     // segments a row
    int prefix_rows;               // rows of a prefix block: 256 or 128 (tensor memory), or 16
    int prefix_tiles, own_tiles;   // slots of prefix tiles over all groups; tiles of 16 rows a trajectory
    int prefix_blocks;             // thread blocks of the prefix part
    int polls;                     // kPolls, or a test's
    float scale_log2;
};

constexpr int kTile = 64;                       // keys a step
constexpr int kThreads = 128;
constexpr int kMaxIds = 2048;                   // page numbers a segment may need; its last tile may look up a tile's more

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0));
}

__device__ __forceinline__ void ldsm4(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}

__device__ __forceinline__ void ldsm4t(uint32_t* r, uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}

__device__ __forceinline__ void mma(float* c, const uint32_t* a, const uint32_t* b) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared.b64 [%0], %1;" ::"r"(bar), "r"(count)); }

__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared.b64 _, [%0];" ::"r"(bar) : "memory"); }

// Bounded: a wait that runs out of polls, or sees that another did, gives up, and the block's rows come out NaN.
__device__ __forceinline__ bool bar_wait(uint32_t bar, int parity, volatile int* gave_up, int most) {
    for (int polls = 0; polls < most; ++polls) {
        uint32_t done;
        asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}"
                     : "=r"(done) : "r"(bar), "r"(parity) : "memory");
        if (done) return true;
        if ((polls & 63) == 63 && *gave_up) return false;
    }
    *gave_up = 1;
    return false;
}

__device__ __forceinline__ void bar_expect(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}

__device__ __forceinline__ void box_load(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}

__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Page (from the segment's first) of place `in` of that page's and the following tokens; in and page below 2^16.
__device__ __forceinline__ int page_of(const AttnParams& P, int in) { return P.page_mul != 0 ? (int)__umulhi((uint32_t)in, P.page_mul) : in; }

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

// Page numbers of the keys [begin, end); a page that is not there (-1) masks its keys.  Returns whether there is one.
__device__ __forceinline__ int read_ids(const AttnParams& P, int* ids, const int32_t* table, int width, int begin, int end, int tid, int threads) {
    const int first = begin / P.page, n = (end - 1) / P.page - first + 1;
    int missing = 0;
    for (int i = tid; i < n; i += threads) {
        int id = first + i < width ? table[first + i] : -1;
        if (id < 0 || id >= P.pages) { id = -1; missing = 1; }
        ids[i] = id;
    }
    return __syncthreads_or(missing);
}

// One segment of keys against 16 rows.  The block's four warps share the rows and take 16 of every 64 keys each, without
// waiting for one another: a warp keeps a ring of 16-key stages of its own (keys and values in 128-byte rows whose 16-byte
// pieces are exchanged by row, as the copies' boxes write them and the 8x8 matrix loads want them) and joins the others
// after the last.
constexpr int kPart = 16;                       // keys a warp and step

template <int D> struct OwnShape {
    static constexpr int kHalf = kPart * 128, kStage = 2 * (D / 64) * kHalf, kStages = D == 128 ? 2 : 4;      // K, then V
    static constexpr int kBytes = 4 * kStages * kStage + 1024;                                                 // + alignment
    static_assert(4 * kStages * kStage >= 4 * 16 * D * 4 + 4 * 16 * 8, "the warps' shares are joined in the stages' room");
};

template <int D, bool TMA>
__device__ __forceinline__ void segment(const AttnParams& P, const CUtensorMap* k_map, const CUtensorMap* v_map, char* raw, int* ids,
                                        uint64_t* bars, int* gave_up, const int32_t* table, int table_width, int begin, int end, int kv_head,
                                        int first_row, int rows, int b0, int slot) {
    typedef OwnShape<D> Shape;
    constexpr int kSteps = D / 16, kStages = Shape::kStages, kHalf = Shape::kHalf, kValues = (D / 64) * kHalf;
    constexpr int kCols = 2;                                  // 8-key columns a warp computes
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    char* const smem = raw + ((1024 - (smem_at(raw) & 1023)) & 1023);
    const uint32_t ring = smem_at(smem) + warp * kStages * Shape::kStage, bar = smem_at(bars) + warp * kStages * 8;

    const int offset = begin % P.page;
    if (TMA && tid < 4 * kStages) {
        bar_init(smem_at(bars) + 8 * tid, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (tid == 0) *gave_up = 0;
    const int missing = read_ids(P, ids, table, table_width, begin, end, tid, kThreads);

    const int len = end - begin - warp * kPart, steps = len > 0 ? (len + kTile - 1) / kTile : 0;      // every 64th key on from the warp's first
    auto at = [&](int row, int c) { return (uint32_t)((c >> 3) * kHalf + row * 128 + (((c & 7) ^ (row & 7)) << 4)); };
    auto load = [&](int t) {
        const uint32_t dst = ring + (t % kStages) * Shape::kStage;
        const int local = warp * kPart + t * kTile;
        if constexpr (TMA) {
            if (t < steps && lane == 0) {
                const uint32_t b = bar + 8 * (t % kStages);
                const int box = P.page < kPart ? P.page : kPart;
                bar_expect(b, Shape::kStage);
                for (int row = 0; row < kPart; row += box) {
                    const int in = offset + local + row, pg = page_of(P, in);
                    const int id = local + row < end - begin ? ids[pg] : -1;      // -1 lies outside the map: zeros
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) {
                        box_load(dst + half * kHalf + row * 128, k_map, b, half * 64, in - pg * P.page, kv_head, id);
                        box_load(dst + kValues + half * kHalf + row * 128, v_map, b, half * 64, in - pg * P.page, kv_head, id);
                    }
                }
            }
        } else {
            if (t < steps) {
#pragma unroll
                for (int i = lane; i < kPart * (D / 8); i += 32) {
                    const int row = i / (D / 8), c = i % (D / 8), in = offset + local + row, pg = page_of(P, in), id = ids[pg];
                    const bool there = local + row < end - begin && c * 8 < P.d && id >= 0;
                    const int64_t from = there ? id * P.page_stride + (in - pg * P.page) * P.token_stride + kv_head * P.head_stride + c * 8 : 0;
                    copy16(dst + at(row, c), P.k + from, there);
                    copy16(dst + kValues + at(row, c), P.v + from, there);
                }
            }
            asm volatile("cp.async.commit_group;");
        }
    };
#pragma unroll
    for (int t = 0; t < kStages; ++t) load(t);

    // queries as the left operand: rows lane / 4 and lane / 4 + 8 of the warp's 16
    uint32_t qf[kSteps][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = first_row + (lane >> 2) + h * 8;
        const bool in = row < rows;
        const int b = b0 + row / P.r, head = kv_head * P.r + row % P.r;
        const __nv_bfloat16* src = P.q + (in ? (int64_t)b * P.q_stride + (int64_t)head * P.d : 0);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = s * 16 + e * 8 + (lane & 3) * 2;
                qf[s][e * 2 + h] = in && col < P.d ? *reinterpret_cast<const uint32_t*>(src + col) : 0u;
            }
    }
    float o[D / 8][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    bool fine = true;
    int t = 0;
    for (; t < steps; ++t) {
        const uint32_t kt = ring + (t % kStages) * Shape::kStage, vt = kt + kValues;
        const int left = len - t * kTile;                     // keys that are there
        if constexpr (TMA) {
            fine = __all_sync(~0u, bar_wait(bar + 8 * (t % kStages), (t / kStages) & 1, gave_up, P.polls));
            if (!fine) break;
            if (left < kPart) {                               // values behind the last key: zeros, whatever the page holds
                for (int i = lane; i < (kPart - left) * (D / 8); i += 32)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(vt + at(left + i / (D / 8), i % (D / 8))), "r"(0) : "memory");
                __syncwarp();
            }
        } else {
            asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
            __syncwarp();
        }
        float s[kCols][4] = {}, s2[kCols][4] = {};            // even and odd dimension steps: shorter chains of products
#pragma unroll
        for (int st = 0; st < kSteps; ++st) {
            uint32_t b[4];                                    // 16 keys, dimensions st*16 .. +15
            ldsm4(b, kt + at((lane & 7) + ((lane >> 4) << 3), st * 2 + ((lane >> 3) & 1)));
            mma(st & 1 ? s2[0] : s[0], qf[st], b);
            mma(st & 1 ? s2[1] : s[1], qf[st], b + 2);
        }
#pragma unroll
        for (int j = 0; j < kCols; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[j][e] += s2[j][e];
        if (left < kPart || missing) {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int key = j * 8 + (lane & 3) * 2 + e;
                    const bool there = key < left && (!missing || ids[page_of(P, offset + warp * kPart + t * kTile + key)] >= 0);
                    if (!there) s[j][e] = s[j][2 + e] = -INFINITY;
                }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < kCols; ++j) top = fmaxf(top, fmaxf(s[j][h * 2], s[j][h * 2 + 1]));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 1));
            top = fmaxf(top, __shfl_xor_sync(~0u, top, 2));
            // the base follows the maximum only when it is 2^8 behind: the weights stay below 2^8, and sums are seldom rescaled
            const float now = top * P.scale_log2;
            if (__any_sync(~0u, now > m[h] + 8.f)) {
                const float next = fmaxf(m[h], now), fade = m[h] == -INFINITY ? 0.f : exp2_of(m[h] - next);
                m[h] = next;
                l[h] *= fade;
#pragma unroll
                for (int n = 0; n < D / 8; ++n) { o[n][h * 2] *= fade; o[n][h * 2 + 1] *= fade; }
            }
            const float base = m[h] == -INFINITY ? 0.f : m[h];
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = exp2_of(fmaf(s[j][h * 2 + e], P.scale_log2, -base));
                    s[j][h * 2 + e] = p;
                    sum += p;
                }
            l[h] += sum;
        }
        // the weights as two bfloat16 parts: what one rounding would lose is as large as the output's own
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = s[e >> 1][(e & 1) * 2], y = s[e >> 1][(e & 1) * 2 + 1];
            hi[e] = pack2(x, y);
            lo[e] = pack2(x - __uint_as_float(hi[e] << 16), y - __uint_as_float(hi[e] & 0xffff0000u));
        }
#pragma unroll
        for (int n = 0; n < D / 8; n += 2) {
            uint32_t b[4];                                    // 16 keys, dimensions n*8 .. +15
            ldsm4t(b, vt + at(lane & 15, n + (lane >> 4)));
            mma(o[n], hi, b);
            mma(o[n], lo, b);
            mma(o[n + 1], hi, b + 2);
            mma(o[n + 1], lo, b + 2);
        }
        __syncwarp();
        load(t + kStages);
    }
    if (!fine) {
        l[0] = l[1] = __int_as_float(0x7fffffff);
        int late = 0;                                         // the boxes in flight land before their place is used otherwise
        for (int u = t; u < min(t + kStages, steps); ++u) bar_wait(bar + 8 * (u % kStages), (u / kStages) & 1, &late, kPolls);
    }
    __syncthreads();                                          // every warp is done with its stages
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(~0u, l[h], 1);
        l[h] += __shfl_xor_sync(~0u, l[h], 2);
    }
    const int64_t seg_rows = (int64_t)slot * P.B * P.H;
    {
        // the four warps' shares, joined through shared memory (the tiles are done with)
        float* so = reinterpret_cast<float*>(smem);           // [4][16][D]
        float2* sml = reinterpret_cast<float2*>(smem + 4 * 16 * D * 4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int row = (lane >> 2) + h * 8;
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
                *reinterpret_cast<float2*>(so + (warp * 16 + row) * D + n * 8 + (lane & 3) * 2) = make_float2(o[n][h * 2], o[n][h * 2 + 1]);
            if ((lane & 3) == 0) sml[warp * 16 + row] = make_float2(m[h], l[h]);
        }
        __syncthreads();
        for (int i = tid; i < 16 * (D / 4); i += kThreads) {
            const int row = i / (D / 4), c = (i % (D / 4)) * 4;
            if (first_row + row >= rows) continue;
            float top = -INFINITY;
            for (int w = 0; w < 4; ++w) top = fmaxf(top, sml[w * 16 + row].x);
            const float base = top == -INFINITY ? 0.f : top;
            float4 sum = {0.f, 0.f, 0.f, 0.f};
            float all = 0.f;
            for (int w = 0; w < 4; ++w) {
                const float f = exp2_of(sml[w * 16 + row].x - base);
                const float4 x = *reinterpret_cast<const float4*>(so + (w * 16 + row) * D + c);
                sum.x += x.x * f; sum.y += x.y * f; sum.z += x.z * f; sum.w += x.w * f;
                all += sml[w * 16 + row].y * f;
            }
            const int rr = first_row + row;
            const int64_t at = seg_rows + (int64_t)(b0 + rr / P.r) * P.H + kv_head * P.r + rr % P.r;
            *reinterpret_cast<float4*>(P.part_o + at * D + c) = sum;
            if (c == 0) P.part_ml[at] = make_float2(top, all);
        }
    }
}

// Which rows and keys a block of the prefix part has.
struct PrefixTile {
    int group, kv_head, seg, first_row, rows, b0, begin, end;      // rows from first_row of the group's `rows`
};

__device__ __forceinline__ bool prefix_tile(const AttnParams& P, int block, PrefixTile* t) {
    const int slot = block % P.prefix_tiles;
    block /= P.prefix_tiles;
    t->kv_head = block % P.Hk;
    t->seg = block / P.Hk;
    // group g's tiles start at slot floor(offset_g r / tile rows) + g: at least as many slots as tiles for any sizes
    int lo = 0, hi = P.groups - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((int64_t)clamp_to(P.group_offsets[mid], 0, P.B) * P.r / P.prefix_rows + mid <= slot) lo = mid; else hi = mid - 1;
    }
    t->group = lo;
    t->b0 = clamp_to(P.group_offsets[lo], 0, P.B);
    t->rows = (clamp_to(P.group_offsets[lo + 1], t->b0, P.B) - t->b0) * P.r;
    t->first_row = (slot - (int)((int64_t)t->b0 * P.r / P.prefix_rows + lo)) * P.prefix_rows;
    const int len = clamp_to(P.prefix_lens[lo], 0, P.max_prefix);
    t->begin = t->seg * P.prefix_seg;
    t->end = min(len, t->begin + P.prefix_seg);
    return t->first_row >= 0 && t->first_row < t->rows && t->begin < t->end;
}

// Tiles of 16 rows, the least an mma.sync has: 4 rows of 16 filled still leave the tensor unit a quarter busy under the loads.
// A trajectory's own keys, and prefixes of groups with few rows (blocks below `prefix_blocks`).
template <int D, bool TMA>
__global__ void __launch_bounds__(kThreads)
attention_kernel(const __grid_constant__ AttnParams P, int prefix_blocks, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    extern __shared__ char raw[];
    __shared__ int ids[kMaxIds + kTile];
    __shared__ __align__(8) uint64_t bars[4 * OwnShape<D>::kStages];
    __shared__ int gave_up;
    int block = blockIdx.x;
    if (block < prefix_blocks) {
        PrefixTile t;
        if (!prefix_tile(P, block, &t)) return;
        segment<D, TMA>(P, &k_map, &v_map, raw, ids, bars, &gave_up, P.prefix_table + (int64_t)t.group * P.prefix_width, P.prefix_width, t.begin, t.end, t.kv_head, t.first_row,
                   t.rows, t.b0, t.seg);
    } else {
        block -= prefix_blocks;
        const int tile = block % P.own_tiles;
        block /= P.own_tiles;
        const int kv_head = block % P.Hk;
        block /= P.Hk;
        const int b = block % P.B, seg = block / P.B;
        const int len = clamp_to(P.lens[b], 0, P.max_len), begin = seg * P.own_seg, end = min(len, begin + P.own_seg);
        if (begin >= end) return;
        segment<D, TMA>(P, &k_map, &v_map, raw, ids, bars, &gave_up, P.block_table + (int64_t)b * P.own_width, P.own_width, begin, end, kv_head, tile * 16, P.r, b,
                   P.prefix_segs + seg);
    }
}

// ---------------------------------------------------------------------------------------------- prefixes of many rows
// RT tiles of 128 rows a block (RT = 2 where groups have more than 128) on tcgen05, each tile: scores S = Q K^T of 64 keys at a
// time into one of two 64-column buffers of tensor memory, the weights back over them as two bfloat16 parts (32 columns
// each), O += P V accumulated in tensor memory.  Four warps a row tile: one row a thread (maximum, exponentials, sums).  Two warps copy keys and values through the page table into a ring of
// slots in the layout that the matrix instructions read (128-byte rows, pieces exchanged by row).  Two warps a row tile issue
// its products, one the scores and one the values: an issuing warp waits about 100 cycles at each barrier, in which the others
// keep the matrix unit busy.  With one row tile a block, two blocks share a multiprocessor to the same end.
// Pages that divide a tile of 64 keys into parts of at least eight rows, or are whole tiles, are copied by TMA boxes (TMA =
// true; a segment's last, partial tile apart, whose missing keys must be zeros); other page sizes piece by piece.
constexpr int kLoaders = 64;

template <int D, int RT> struct PrefixShape {
    static constexpr int kThreads = RT * 192 + kLoaders, kSlot = kTile * D * 2, kSlots = D == 128 && RT == 1 ? 4 : 8;
    static constexpr int kQ = 128 * D * 2, kColumns = 256 * RT;    // of tensor memory: two score buffers and O, a row tile
    static constexpr int kBytes = RT * kQ + kSlots * kSlot + 1024; // + alignment
};

// Matrix instructions and their commits are reached by the whole warp and issued by its elected lane, the same one every
// time, so that their operands stay in uniform registers.
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("{\n.reg .pred e;\nelect.sync _|e, 0xffffffff;\n"
                 "@e tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar) : "memory");
}

// 128-byte rows with exchanged pieces; `lead`: bytes between blocks of 64 along the contiguous dimension (not used where
// that is the summed one), 1024 bytes between groups of eight rows.
__device__ __forceinline__ uint64_t describe(uint32_t at, uint32_t lead) {
    return (uint64_t)((at & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, int add) {
    asm volatile("{\n.reg .pred e, p;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %4, 0;\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(kind), "r"(add) : "memory");
}

__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, int add) {
    asm volatile("{\n.reg .pred e, p;\nelect.sync _|e, 0xffffffff;\nsetp.ne.b32 p, %4, 0;\n@e tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(kind), "r"(add) : "memory");
}

__device__ __forceinline__ void tmem_load32(uint32_t* r, uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"
                 "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
                   "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
                   "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]) : "r"(at) : "memory");
}

__device__ __forceinline__ void tmem_load16(uint32_t* r, uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                   "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(at) : "memory");
}

__device__ __forceinline__ void tmem_store16(uint32_t at, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
                 "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

__device__ __forceinline__ void tmem_wait_load() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_store() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

template <int D, bool TMA, int RT>
__global__ void __launch_bounds__(PrefixShape<D, RT>::kThreads, 3 - RT)
prefix_kernel(const __grid_constant__ AttnParams P, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
    typedef PrefixShape<D, RT> Shape;
    constexpr int kSlots = Shape::kSlots, kPieces = D / 8, kIssuer = RT * 4 + kLoaders / 32;
    constexpr uint32_t kScores = 1u << 4 | 1u << 7 | 1u << 10 | (kTile >> 3) << 17 | (128 >> 4) << 24;
    constexpr uint32_t kValues = 1u << 4 | 1u << 7 | 1u << 10 | 1u << 16 | (D >> 3) << 17 | (128 >> 4) << 24;      // V: keys by rows
    extern __shared__ char raw[];
    __shared__ int ids[kMaxIds + kTile];
    __shared__ __align__(8) uint64_t bars[2 * kSlots + 6 * RT + 1];
    __shared__ uint32_t tmem_at;
    __shared__ int gave_up;
    PrefixTile t;
    if (!prefix_tile(P, blockIdx.x, &t)) return;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t q_at = (smem_at(raw) + 1023) & ~1023u, ring = q_at + RT * Shape::kQ;
    const uint32_t full = smem_at(bars), empty = full + 8 * kSlots, drained = empty + 8 * kSlots;
    const uint32_t s_full = drained + 8, p_full = s_full + 16 * RT, o_done = p_full + 16 * RT;      // two a row tile, taken in turn
    const int row_tiles = RT == 2 && t.rows - t.first_row <= 128 ? 1 : RT;
    if (warp == kIssuer) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&tmem_at)), "n"(Shape::kColumns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        gave_up = 0;
        for (int i = 0; i < kSlots; ++i) { bar_init(full + 8 * i, TMA ? 1 : kLoaders); bar_init(empty + 8 * i, row_tiles); }
        for (int i = 0; i < 2 * RT; ++i) { bar_init(s_full + 8 * i, 1); bar_init(p_full + 8 * i, 128); bar_init(o_done + 8 * i, 1); }
        bar_init(drained, 2 * RT);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    // queries, zeros where there are none
    for (int i = tid; i < RT * 128 * kPieces; i += Shape::kThreads) {
        const int row = i / kPieces, c = i % kPieces, at = t.first_row + row;
        uint4 v = {0, 0, 0, 0};
        if (at < t.rows && c * 8 < P.d)
            v = *reinterpret_cast<const uint4*>(P.q + (int64_t)(t.b0 + at / P.r) * P.q_stride + (int64_t)(t.kv_head * P.r + at % P.r) * P.d + c * 8);
        const uint32_t dst = q_at + (row >> 7) * Shape::kQ + (c >> 3) * (128 * 128) + (row & 127) * 128 + (((c & 7) ^ (row & 7)) << 4);
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
    }
    fence_async();
    fence_before();
    const int missing = read_ids(P, ids, P.prefix_table + (int64_t)t.group * P.prefix_width, P.prefix_width, t.begin, t.end, tid, Shape::kThreads);
    fence_after();
    const uint32_t tmem = tmem_at;
    const int offset = t.begin % P.page, tiles = (t.end - t.begin + kTile - 1) / kTile;

    if (warp < 4 * RT) {
        const int rt = warp >> 2;
        const uint32_t mine = ((uint32_t)((warp & 3) * 32) << 16) + rt * 256, o_at = tmem + mine + 128;
        const uint32_t my_s = s_full + 16 * rt, my_p = p_full + 16 * rt, my_o = o_done + 16 * rt;
        const bool any_row = t.first_row + warp * 32 < t.rows;
        float m = -INFINITY, l = 0.f;
        bool fine = true;
        for (int i = 0; i < tiles && rt < row_tiles; ++i) {
            const uint32_t at = tmem + mine + (i & 1) * kTile;
            fine = __all_sync(~0u, bar_wait(my_s + 8 * (i & 1), (i >> 1) & 1, &gave_up, P.polls));
            if (!fine) break;
            fence_after();
            if (any_row) {
                uint32_t s[kTile];
                tmem_load32(s, at);
                tmem_load32(s + 32, at + 32);
                tmem_wait_load();
                const int left = t.end - t.begin - i * kTile;
                if (left < kTile || missing) {
#pragma unroll
                    for (int k = 0; k < kTile; ++k) {
                        const bool there = k < left && (!missing || ids[page_of(P, offset + i * kTile + k)] >= 0);
                        if (!there) s[k] = __float_as_uint(-INFINITY);
                    }
                }
                float top[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int k = 0; k < kTile; k += 8)
#pragma unroll
                    for (int c = 0; c < 4; ++c) top[c] = fmaxf(fmaxf(top[c], __uint_as_float(s[k + 2 * c])), __uint_as_float(s[k + 2 * c + 1]));
                const float now = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3])) * P.scale_log2;
                // the base follows the maximum only when it is 2^8 behind: the weights stay below 2^8, and O is seldom rescaled
                if (__any_sync(~0u, now > m + 8.f)) {
                    const float next = fmaxf(m, now), fade = m == -INFINITY ? 0.f : exp2_of(m - next);
                    if (i > 0) {
                        fine = __all_sync(~0u, bar_wait(my_o + 8 * ((i - 1) & 1), ((i - 1) >> 1) & 1, &gave_up, P.polls));
                        if (!fine) break;
                        fence_after();
#pragma unroll
                        for (int c = 0; c < D; c += 16) {
                            uint32_t o[16];
                            tmem_load16(o, o_at + c);
                            tmem_wait_load();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * fade);
                            tmem_store16(o_at + c, o);
                        }
                    }
                    l *= fade;
                    m = next;
                }
                const float base = m == -INFINITY ? 0.f : m;
                const float2 scale = {P.scale_log2, P.scale_log2}, less = {-base, -base}, minus = {-1.f, -1.f};
                float2 sum[2] = {{0.f, 0.f}, {0.f, 0.f}};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t hi[16], lo[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float2 p = fma2(make_float2(__uint_as_float(s[half * 32 + 2 * k]), __uint_as_float(s[half * 32 + 2 * k + 1])), scale, less);
                        p = make_float2(exp2_of(p.x), exp2_of(p.y));
                        sum[k & 1] = add2(sum[k & 1], p);
                        hi[k] = pack2(p.x, p.y);
                        p = fma2(make_float2(__uint_as_float(hi[k] << 16), __uint_as_float(hi[k] & 0xffff0000u)), minus, p);
                        lo[k] = pack2(p.x, p.y);
                    }
                    tmem_store16(at + half * 16, hi);
                    tmem_store16(at + 32 + half * 16, lo);
                }
                l += (sum[0].x + sum[1].x) + (sum[0].y + sum[1].y);
                tmem_wait_store();
            }
            fence_before();
            bar_arrive(my_p + 8 * (i & 1));
        }
        if (any_row) {
            for (int i = max(tiles - 2, 0); i < tiles && fine; ++i)
                fine = __all_sync(~0u, bar_wait(my_o + 8 * (i & 1), (i >> 1) & 1, &gave_up, P.polls));
            fine = fine && *(volatile int*)&gave_up == 0;         // a thread that copies may have given up alone
            fence_after();
            const int at = t.first_row + warp * 32 + lane;
            const int64_t dst = (int64_t)t.seg * P.B * P.H + (int64_t)(t.b0 + at / P.r) * P.H + t.kv_head * P.r + at % P.r;
#pragma unroll
            for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tmem_load32(o, o_at + c);
                tmem_wait_load();
                if (at < t.rows)
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        *reinterpret_cast<uint4*>(P.part_o + dst * D + c + k) = make_uint4(o[k], o[k + 1], o[k + 2], o[k + 3]);
            }
            if (at < t.rows) P.part_ml[dst] = fine ? make_float2(m, l) : make_float2(0.f, __int_as_float(0x7fffffff));
        }
        fence_before();
    } else if (warp < kIssuer) {
        const int me = tid - RT * 128, c = me % kPieces, row0 = me / kPieces;
        constexpr int kStep = kLoaders / kPieces, kRows = (kTile + kStep - 1) / kStep;
        constexpr int kAhead = kSlots - 2;                        // slots being filled
        const __nv_bfloat16* from[2] = {P.k + t.kv_head * P.head_stride + c * 8, P.v + t.kv_head * P.head_stride + c * 8};
        const uint32_t lane_at = ring + (c >> 3) * (kTile * 128);
        int64_t place[kRows];                                     // of the thread's rows in the caches, -1: no such key
        auto places = [&](int tile) {
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                const int local = tile * kTile + row0 + k * kStep, in = offset + local, pg = page_of(P, in), id = ids[pg];
                const int64_t at = id * P.page_stride + (in - pg * P.page) * P.token_stride;
                place[k] = t.begin + local < t.end && c * 8 < P.d && id >= 0 ? at : -1;
            }
        };
        auto pieces = [&](int item) {
            const __nv_bfloat16* base = from[item & 1];
            const uint32_t dst = lane_at + (item % kSlots) * Shape::kSlot;
#pragma unroll
            for (int k = 0; k < kRows; ++k) {
                const int row = row0 + k * kStep;
                if (row < kTile) copy16(dst + row * 128 + (((c & 7) ^ (row & 7)) << 4), base + (place[k] < 0 ? 0 : place[k]), place[k] >= 0);
            }
        };
        auto room = [&](int item) { return item < kSlots || bar_wait(empty + 8 * (item % kSlots), (item / kSlots - 1) & 1, &gave_up, P.polls); };
        bool fine = true;
        if constexpr (TMA) {
            const int whole = (t.end - t.begin) / kTile, box = P.page < kTile ? P.page : kTile;
            int issued = 0;
            if (me == 0)
                for (int i = 0; i < 2 * whole && fine; ++i) {
                    fine = room(i);
                    if (!fine) break;
                    const uint32_t bar = full + 8 * (i % kSlots), dst = ring + (i % kSlots) * Shape::kSlot;
                    issued = i + 1;
                    bar_expect(bar, Shape::kSlot);
                    for (int row = 0; row < kTile; row += box) {
                        const int in = offset + (i >> 1) * kTile + row, pg = page_of(P, in);
#pragma unroll
                        for (int half = 0; half < D / 64; ++half)     // a page number of -1 lies outside the map: zeros
                            box_load(dst + half * (kTile * 128) + row * 128, i & 1 ? &v_map : &k_map, bar, half * 64, in - pg * P.page, t.kv_head, ids[pg]);
                    }
                }
            if (whole < tiles) {
                asm volatile("bar.sync 1, %0;" ::"n"(kLoaders) : "memory");
                places(whole);
                for (int i = 2 * whole; i < 2 * whole + 2 && fine; ++i) {
                    fine = room(i);
                    if (fine) pieces(i);
                }
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_async();
                asm volatile("bar.sync 1, %0;" ::"n"(kLoaders) : "memory");
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
            for (int i = 0; i < 2 * tiles + kAhead && fine; ++i) {
                if (i < 2 * tiles) {
                    if ((i & 1) == 0) places(i >> 1);
                    fine = room(i);
                    if (!fine) break;
                    pieces(i);
                }
                asm volatile("cp.async.commit_group;");
                if (i >= kAhead) {                                // the copies of kAhead items ago are complete
                    asm volatile("cp.async.wait_group %0;" ::"n"(kAhead) : "memory");
                    fence_async();
                    bar_arrive(full + 8 * ((i - kAhead) % kSlots));
                }
            }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        const int rt = (warp - kIssuer) >> 1;
        const uint32_t base = __shfl_sync(~0u, tmem, 0) + rt * 256;
        const uint32_t my_s = s_full + 16 * rt, my_p = p_full + 16 * rt, my_o = o_done + 16 * rt;
        auto wait = [&](uint32_t bar, int parity) { return (bool)__all_sync(~0u, bar_wait(bar, parity & 1, &gave_up, P.polls)); };
        const int n = rt < row_tiles ? tiles : 0;
        bool fine = true;
        if (((warp - kIssuer) & 1) == 0) {
            const uint64_t q_desc = describe(q_at + rt * Shape::kQ, 16), k_desc = describe(ring, 16);
            for (int i = 0; i < n; ++i) {
                const int item = 2 * i, slot = item % kSlots;
                // the buffer's weights must have been multiplied before new scores go there
                fine = (i < 2 || wait(my_o + 8 * (i & 1), (i - 2) >> 1)) && wait(full + 8 * slot, item / kSlots);
                if (!fine) break;
                fence_after();
                const uint64_t k_at = k_desc + slot * (Shape::kSlot >> 4);
#pragma unroll
                for (int s = 0; s < D / 16; ++s)
                    mma_ss(base + (i & 1) * kTile, q_desc + (((s >> 2) * (128 * 128) + (s & 3) * 32) >> 4),
                           k_at + (((s >> 2) * (kTile * 128) + (s & 3) * 32) >> 4), kScores, s > 0);
                commit(my_s + 8 * (i & 1));
                commit(empty + 8 * slot);
            }
        } else {
            const uint64_t v_desc = describe(ring, kTile * 128);
            for (int i = 0; i < n; ++i) {
                const int item = 2 * i + 1, slot = item % kSlots;
                fine = wait(full + 8 * slot, item / kSlots) && wait(my_p + 8 * (i & 1), i >> 1);
                if (!fine) break;
                fence_after();
                const uint64_t v_at = v_desc + slot * (Shape::kSlot >> 4);
                const uint32_t p_at = base + (i & 1) * kTile;
#pragma unroll
                for (int part = 0; part < 2; ++part)
#pragma unroll
                    for (int s = 0; s < kTile / 16; ++s)
                        mma_ts(base + 128, p_at + part * 32 + s * 8, v_at + ((s * 2048) >> 4), kValues, i > 0 || part > 0 || s > 0);
                commit(my_o + 8 * (i & 1));
                commit(empty + 8 * slot);
            }
        }
        commit(drained);                                          // nothing in flight when the memory is given back
        int late = 0;
        bar_wait(drained, 0, &late, kPolls);
    }
    __syncwarp();
    __syncthreads();
    if (warp == kIssuer) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(Shape::kColumns) : "memory");
    }
}

// Joins a row's segments: one warp a (row, head).
template <int D>
__global__ void __launch_bounds__(kThreads) join_kernel(const __grid_constant__ AttnParams P) {
    constexpr int kPer = D / 32;
    const int64_t at = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), all = (int64_t)P.B * P.H;
    const int lane = threadIdx.x & 31;
    if (at >= all) return;
    const int b = (int)(at / P.H);
    int lo = 0, hi = P.groups;                                // the last group that starts at or before b
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (mid < P.groups && P.group_offsets[mid] <= b) lo = mid; else hi = mid - 1;
    }
    const bool grouped = P.groups > 0 && b >= P.group_offsets[lo] && b < P.group_offsets[lo + 1];
    const int pre = grouped ? (clamp_to(P.prefix_lens[lo], 0, P.max_prefix) + P.prefix_seg - 1) / P.prefix_seg : 0;
    const int own = (clamp_to(P.lens[b], 0, P.max_len) + P.own_seg - 1) / P.own_seg;
    float top = -INFINITY, sum = 0.f, o[kPer] = {};
    for (int i = 0; i < pre + own; ++i) {
        const int64_t row = (int64_t)(i < pre ? i : P.prefix_segs + i - pre) * all + at;
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

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

int divide_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// How the keys are cut into segments: enough thread blocks for the GPU, segments of at least four tiles.
int plan_segment(int64_t longest, int64_t units, int page, int64_t most) {
    if (longest <= 0) return kTile;
    const int64_t want = rlcs_device::limits().sms * 2 * 2;
    int64_t segs = units >= want ? 1 : (want + units - 1) / (units > 0 ? units : 1);
    const int64_t least = divide_up(longest, 4 * kTile);
    if (segs > least) segs = least;
    int64_t len = divide_up(divide_up(longest, segs), kTile) * (int64_t)kTile;
    if (len > most) len = most;
    const int64_t by_ids = (int64_t)(kMaxIds - 2) * page / kTile * kTile;
    return (int)(len < by_ids ? len : by_ids);
}

// The prefix kernel runs `slots` blocks at once: the number of segments that makes its rounds of blocks shortest, a
// segment costing three tiles beyond its own (start, first loads, the partial result).
int plan_prefix(int64_t longest, int64_t units, int page, int64_t slots) {
    const int64_t tiles = divide_up(longest, kTile);
    const int64_t by_ids = (int64_t)(kMaxIds - 2) * page / kTile, most = by_ids < 256 ? by_ids : 256;
    int64_t best = 1, cost = INT64_MAX;
    for (int64_t segs = divide_up(tiles, most); segs <= tiles && segs <= 256; ++segs) {
        const int64_t c = divide_up(units * segs, slots) * (int64_t)(divide_up(tiles, segs) + 3);
        if (c < cost) { cost = c; best = divide_up(tiles, segs); }
    }
    return (int)((cost == INT64_MAX ? most : best) * kTile);
}

int plan(AttnParams& P) {
    const int64_t rows = (int64_t)P.B * P.r;
    P.own_tiles = divide_up(P.r, 16);
    P.prefix_rows = P.groups <= 0 || rows <= 16 * (int64_t)P.groups ? 16 : rows <= 128 * (int64_t)P.groups ? 128 : 256;
    P.prefix_tiles = P.groups > 0 ? (int)(rows / P.prefix_rows) + P.groups : 0;
    const int64_t units = P.groups > 0 ? (int64_t)P.Hk * P.groups * divide_up(divide_up(rows, P.groups), P.prefix_rows) : 0;
    P.prefix_seg = P.max_prefix <= 0 ? kTile : P.prefix_rows == 16 ? plan_segment(P.max_prefix, units, P.page, 1024)
                   : plan_prefix(P.max_prefix, units, P.page, rlcs_device::limits().sms * (P.prefix_rows == 128 ? 2 : 1));
    P.own_seg = plan_segment(P.max_len, rows > 0 ? (int64_t)P.B * P.Hk * P.own_tiles : 1, P.page, 1024);
    P.prefix_segs = P.groups > 0 ? divide_up(P.max_prefix, P.prefix_seg) : 0;
    P.own_segs = divide_up(P.max_len, P.own_seg);
    const int64_t pb = (int64_t)P.prefix_tiles * P.Hk * P.prefix_segs, ob = (int64_t)P.own_tiles * P.Hk * P.B * P.own_segs;
    if (pb + ob > (int64_t(1) << 31) - 1) return RLCS_ERR_SIZE;
    P.prefix_blocks = (int)pb;
    return RLCS_OK;
}

// Sizes only: shared by the call and its workspace query.
int check_shape(AttnParams& P, int64_t B, int64_t H, int64_t Hk, int64_t d, int64_t page, int64_t groups, int64_t max_prefix,
                int64_t max_len) {
    const int64_t kMostLen = (int64_t(1) << 31) - 1 - 65536;
    if (B < 0 || H < 0 || Hk < 0 || groups < 0 || max_prefix < 0 || max_len < 0 || page < 1) return RLCS_ERR_SIZE;
    if (B > (1 << 20) || H > 4096 || groups > (1 << 20) || max_prefix > kMostLen || max_len > kMostLen || page > 32768) return RLCS_ERR_SIZE;
    if (d < 8 || d > 128 || d % 8 != 0) return RLCS_ERR_SIZE;
    if (H > 0 && (Hk == 0 || H % Hk != 0)) return RLCS_ERR_SIZE;
    P.B = (int)B;
    P.H = (int)H;
    P.Hk = (int)Hk;
    P.r = Hk > 0 ? (int)(H / Hk) : 0;
    P.d = (int)d;
    P.page = (int)page;
    P.groups = (int)groups;
    P.max_prefix = groups > 0 ? (int)max_prefix : 0;
    P.max_len = (int)max_len;
    P.page_mul = page > 1 ? (uint32_t)(((uint64_t(1) << 32) + page - 1) / page) : 0;
    return B == 0 || H == 0 ? RLCS_OK : plan(P);
}

size_t workspace_of(const AttnParams& P) {
    const size_t rows = (size_t)(P.prefix_segs + P.own_segs) * P.B * P.H;
    return rows * ((P.d <= 64 ? 64 : 128) + 2) * sizeof(float) + 16;
}

// Room beyond 48 KB of shared memory, asked for once a device.
template <typename F> bool grant(F kernel, int bytes, bool* granted) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!granted[dev]) granted[dev] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    return granted[dev];
}

// The cache as a map of boxes [at most `rows` places of a page, 64 dimensions]; false where pages cannot be cut into such boxes of at
// least eight places, or the driver takes no such strides.
bool box_map(CUtensorMap* map, const AttnParams& P, const void* base, int rows) {
    if (P.page >= rows ? P.page % rows != 0 : P.page < 8 || rows % P.page != 0) return false;
    typedef CUresult (*Encode)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                               const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static const Encode encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess) fn = nullptr;
        return reinterpret_cast<Encode>(fn);
    }();
    if (encode == nullptr || P.pages < 1) return false;
    const cuuint64_t extent[4] = {(cuuint64_t)P.d, (cuuint64_t)P.page, (cuuint64_t)P.Hk, (cuuint64_t)P.pages};
    const cuuint64_t stride[3] = {(cuuint64_t)P.token_stride * 2, (cuuint64_t)P.head_stride * 2, (cuuint64_t)P.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)(P.page < rows ? P.page : rows), 1, 1}, step[4] = {1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), extent, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TMA, int RT>
int launch_prefix(const AttnParams& P, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s) {
    typedef PrefixShape<D, RT> Shape;
    static bool granted[64];
    if (!grant(prefix_kernel<D, TMA, RT>, Shape::kBytes, granted)) return RLCS_ERR_CUDA;
    prefix_kernel<D, TMA, RT><<<(unsigned)P.prefix_blocks, Shape::kThreads, Shape::kBytes, s>>>(P, k_map, v_map);
    return RLCS_OK;
}

template <int D, bool TMA>
int launch_own(const AttnParams& P, int64_t blocks, int prefix_blocks, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t s) {
    static bool granted[64];
    if (!grant(attention_kernel<D, TMA>, OwnShape<D>::kBytes, granted)) return RLCS_ERR_CUDA;
    attention_kernel<D, TMA><<<(unsigned)blocks, kThreads, OwnShape<D>::kBytes, s>>>(P, prefix_blocks, k_map, v_map);
    return RLCS_OK;
}

template <int D> int launch(const AttnParams& P, cudaStream_t s) {
    CUtensorMap k_map = {}, v_map = {};
    int st = RLCS_OK;
    const bool wide = P.prefix_rows > 16;
    if (wide && P.prefix_blocks > 0) {
        const bool boxes = box_map(&k_map, P, P.k, kTile) && box_map(&v_map, P, P.v, kTile);
        st = P.prefix_rows == 256 ? (boxes ? launch_prefix<D, true, 2>(P, k_map, v_map, s) : launch_prefix<D, false, 2>(P, k_map, v_map, s))
                                  : (boxes ? launch_prefix<D, true, 1>(P, k_map, v_map, s) : launch_prefix<D, false, 1>(P, k_map, v_map, s));
        if (st != RLCS_OK) return st;
    }
    const int narrow_blocks = wide ? 0 : P.prefix_blocks;
    const int64_t blocks = narrow_blocks + (int64_t)P.own_tiles * P.Hk * P.B * P.own_segs;
    if (blocks > 0) {
        const bool boxes = box_map(&k_map, P, P.k, kPart) && box_map(&v_map, P, P.v, kPart);
        st = boxes ? launch_own<D, true>(P, blocks, narrow_blocks, k_map, v_map, s) : launch_own<D, false>(P, blocks, narrow_blocks, k_map, v_map, s);
        if (st != RLCS_OK) return st;
    }
    join_kernel<D><<<(unsigned)divide_up((int64_t)P.B * P.H, kThreads / 32), kThreads, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // namespace

extern "C" {

size_t rlcs_prefix_attention_workspace_bytes(int64_t B, int64_t H, int64_t Hk, int64_t d, int64_t page_size, int64_t groups,
                                             int64_t max_prefix_len, int64_t max_len) {
    AttnParams P = {};
    if (check_shape(P, B, H, Hk, d, page_size, groups, max_prefix_len, max_len) != RLCS_OK || B == 0 || H == 0) return 0;
    return workspace_of(P);
}

int rlcs_prefix_attention_bf16(const uint16_t* q, int64_t q_stride, const uint16_t* k_cache, const uint16_t* v_cache, int64_t pages,
                               int64_t page_stride, int64_t token_stride, int64_t head_stride, const int32_t* prefix_table,
                               int64_t prefix_width, const int32_t* prefix_lens, const int32_t* group_offsets, const int32_t* block_table,
                               int64_t own_width, const int32_t* lens, uint16_t* out, float* lse, int64_t B, int64_t H, int64_t Hk,
                               int64_t d, int64_t page_size, int64_t groups, int64_t max_prefix_len, int64_t max_len, float scale,
                               void* workspace, size_t workspace_bytes, void* cuda_stream) {
    AttnParams P = {};
    const int st = check_shape(P, B, H, Hk, d, page_size, groups, max_prefix_len, max_len);
    if (st != RLCS_OK) return st;
    if (pages < 0 || pages > (int64_t(1) << 31) - 1 || prefix_width < 0 || own_width < 0 || prefix_width > (1 << 30) || own_width > (1 << 30))
        return RLCS_ERR_SIZE;
    if (B == 0 || H == 0) return RLCS_OK;
    if (q_stride < H * d || page_stride < 0 || token_stride < 0 || head_stride < 0) return RLCS_ERR_SIZE;
    if (!(scale > 0.f) || !std::isfinite(scale)) return RLCS_ERR_ARG;
    if (q == nullptr || out == nullptr || lens == nullptr) return RLCS_ERR_NULL;
    if ((P.max_prefix > 0 || P.max_len > 0) && (k_cache == nullptr || v_cache == nullptr)) return RLCS_ERR_NULL;
    if (groups > 0 && (group_offsets == nullptr || prefix_lens == nullptr)) return RLCS_ERR_NULL;
    if ((P.max_prefix > 0 && prefix_width > 0 && prefix_table == nullptr) || (P.max_len > 0 && own_width > 0 && block_table == nullptr))
        return RLCS_ERR_NULL;
    const void* words[] = {prefix_table, prefix_lens, group_offsets, block_table, lens, lse};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(q, 16) || !aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || !aligned_to(out, 16)) return RLCS_ERR_ALIGN;
    if (q_stride % 8 || page_stride % 8 || token_stride % 8 || head_stride % 8) return RLCS_ERR_ALIGN;
    if (workspace == nullptr || workspace_bytes < workspace_of(P)) return RLCS_ERR_WORKSPACE;
    if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    P.q = reinterpret_cast<const __nv_bfloat16*>(q);
    P.k = reinterpret_cast<const __nv_bfloat16*>(k_cache);
    P.v = reinterpret_cast<const __nv_bfloat16*>(v_cache);
    P.prefix_table = prefix_table;
    P.prefix_lens = prefix_lens;
    P.group_offsets = group_offsets;
    P.block_table = block_table;
    P.lens = lens;
    P.out = reinterpret_cast<__nv_bfloat16*>(out);
    P.lse = lse;
    P.q_stride = q_stride;
    P.page_stride = page_stride;
    P.token_stride = token_stride;
    P.head_stride = head_stride;
    P.pages = pages;
    P.prefix_width = (int)prefix_width;
    P.own_width = (int)own_width;
    P.scale_log2 = scale * 1.4426950408889634f;
    P.polls = rlcs_hooks::g_wait_polls >= 0 ? rlcs_hooks::g_wait_polls : kPolls;
    const size_t rows = (size_t)(P.prefix_segs + P.own_segs) * P.B * P.H;
    P.part_o = static_cast<float*>(workspace);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + rows * (P.d <= 64 ? 64 : 128));
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return P.d <= 64 ? launch<64>(P, s) : launch<128>(P, s);
}

}  // extern "C"

// What the attention kernels over a paged cache share: parameters, copies through the page table, one segment of keys against a
// tile of 16 rows, the wrappers of the matrix and tensor-memory instructions, and the host's planning of segments.
#pragma once

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

namespace rlcs_attn {

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

// Page (from the segment's first) of place `in` of that page's and the following tokens; exact while in * page < 2^32: pages hold up to 32768
// tokens and segments up to 65536 and a tile, so that in stays below 98368.
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

// CAUSAL: row k of the tile's 16 sees the first seen0 + (first_row + k) / r keys from `begin` on.
template <int D, bool TMA, bool CAUSAL = false>
__device__ __forceinline__ void segment(const AttnParams& P, const CUtensorMap* k_map, const CUtensorMap* v_map, char* raw, int* ids,
                                        uint64_t* bars, int* gave_up, const int32_t* table, int table_width, int begin, int end, int kv_head,
                                        int first_row, int rows, int b0, int slot, int seen0 = 0) {
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
        if constexpr (CAUSAL) {
            const int first = warp * kPart + t * kTile;       // of the 16 keys
            if (first + kPart > seen0 + first_row / P.r) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int sees = seen0 + (first_row + (lane >> 2) + h * 8) / P.r - first;
#pragma unroll
                    for (int j = 0; j < kCols; ++j)
#pragma unroll
                        for (int e = 0; e < 2; ++e)
                            if (j * 8 + (lane & 3) * 2 + e >= sees) s[j][h * 2 + e] = -INFINITY;
                }
            }
        }
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
            if constexpr (CAUSAL)
                if (P.own_segs == 1) {                            // the only segment: nothing to be joined
                    const int64_t to = (int64_t)(b0 + rr / P.r) * P.H + kv_head * P.r + rr % P.r;
                    const float inv = all != 0.f ? 1.f / all : 0.f;
                    if (c < P.d)
                        *reinterpret_cast<uint2*>(P.out + to * P.d + c) = all != 0.f ? make_uint2(pack2(sum.x * inv, sum.y * inv), pack2(sum.z * inv, sum.w * inv)) : make_uint2(0, 0);
                    if (c == 0 && P.lse != nullptr) P.lse[to] = all != 0.f ? (top + log2f(all)) * 0.6931471805599453f : -INFINITY;
                    continue;
                }
            const int64_t at = seg_rows + (int64_t)(b0 + rr / P.r) * P.H + kv_head * P.r + rr % P.r;
            *reinterpret_cast<float4*>(P.part_o + at * D + c) = sum;
            if (c == 0) P.part_ml[at] = make_float2(top, all);
        }
    }
}

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

inline bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

inline int divide_up(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

// How the keys are cut into segments: enough thread blocks for the GPU, segments of at least four tiles.
inline int plan_segment(int64_t longest, int64_t units, int page, int64_t most) {
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

// Room beyond 48 KB of shared memory, asked for once a device.
template <typename F> bool grant(F kernel, int bytes, bool* granted) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return false;
    if (!granted[dev]) granted[dev] = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) == cudaSuccess;
    return granted[dev];
}

typedef CUresult (*EncodeTiled)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps, null where it has none.
inline EncodeTiled encode_tiled() {
    static const EncodeTiled encode = [] {
        void* fn = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess) fn = nullptr;
        return reinterpret_cast<EncodeTiled>(fn);
    }();
    return encode;
}

// The cache as a map of boxes [at most `rows` places of a page, 64 dimensions]; false where pages cannot be cut into such boxes of at
// least eight places, or the driver takes no such strides.
inline bool box_map(CUtensorMap* map, const AttnParams& P, const void* base, int rows) {
    if (P.page >= rows ? P.page % rows != 0 : P.page < 8 || rows % P.page != 0) return false;
    const EncodeTiled encode = encode_tiled();
    if (encode == nullptr || P.pages < 1) return false;
    const cuuint64_t extent[4] = {(cuuint64_t)P.d, (cuuint64_t)P.page, (cuuint64_t)P.Hk, (cuuint64_t)P.pages};
    const cuuint64_t stride[3] = {(cuuint64_t)P.token_stride * 2, (cuuint64_t)P.head_stride * 2, (cuuint64_t)P.page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)(P.page < rows ? P.page : rows), 1, 1}, step[4] = {1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), extent, stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace rlcs_attn

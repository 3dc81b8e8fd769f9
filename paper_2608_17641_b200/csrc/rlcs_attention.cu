// Attention of one query a trajectory over a paged cache whose trajectories share their group's prompt.
//
//   keys of row b:  the prefix of its group (prefix_table, prefix_lens), then its own tokens (block_table, lens)
//   c_j = scale q . k_j,   o = sum_j exp(c_j) v_j / sum_j exp(c_j),   lse = log sum_j exp(c_j)
//
// A group's prefix is multiplied with all of the group's queries at once: the queries of all its rows and of the heads
// that share a key head are the rows of one tile.  A row's own tokens meet the heads that share a key head only.  Both
// run over key segments that leave (running maximum, sum, product) behind; a second kernel joins a row's segments.
#include <cuda_bf16.h>

#include <cmath>
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"

namespace {

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
    int prefix_tiles, own_tiles;   // tiles of 64 rows over all groups; tiles of 16 rows a trajectory
    int prefix_blocks;             // thread blocks of the prefix part
    float scale_log2;
};

constexpr int kTile = 64;                       // keys a step
constexpr int kThreads = 128;
constexpr int kMaxIds = 2048;                   // page numbers a segment may need

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

__device__ __forceinline__ float exp2_of(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// byte offset of 16-byte piece c of row `row` in a tile whose rows hold D values: pieces exchanged within
// groups of eight rows, so that the eight rows of an 8x8 matrix lie in different banks
template <int D> __device__ __forceinline__ uint32_t piece(int row, int c) { return row * (D * 2) + ((c ^ (row & 7)) << 4); }

// Page (from the segment's first) of place `in` of that page's and the following tokens; in and page below 2^16.
__device__ __forceinline__ int page_of(const AttnParams& P, int in) { return P.page_mul != 0 ? (int)__umulhi((uint32_t)in, P.page_mul) : in; }

// One segment of keys against 16 rows a warp.  KEYS_SPLIT: the block's four warps share the 16 rows and take 16 of each
// tile's 64 keys each; otherwise every warp has 16 rows of its own and all of the keys.
template <int D, bool KEYS_SPLIT>
__device__ __forceinline__ void segment(const AttnParams& P, char* smem, int* ids, const int32_t* table, int table_width, int begin,
                                        int end, int kv_head, int first_row, int rows, int b0, int slot) {
    constexpr int kPieces = D / 8, kTileBytes = kTile * D * 2, kSteps = D / 16;
    constexpr int kCols = KEYS_SPLIT ? 2 : 8;                 // 8-key columns a warp computes
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

    // page numbers of the segment; a page that is not there masks its keys
    const int first_page = begin / P.page, offset = begin - first_page * P.page;
    const int n_ids = (end - 1) / P.page - first_page + 1;
    int missing = 0;
    for (int i = tid; i < n_ids; i += kThreads) {
        int id = first_page + i < table_width ? table[first_page + i] : -1;
        if (id < 0 || id >= P.pages) { id = -1; missing = 1; }
        ids[i] = id;
    }
    missing = __syncthreads_or(missing);

    auto load = [&](int base, char* k_at, char* v_at) {       // keys [base, base + 64) of the segment, zeros where there are none
#pragma unroll 4
        for (int i = tid; i < kTile * kPieces; i += kThreads) {
            const int row = i / kPieces, c = i % kPieces, local = base + row;
            bool there = begin + local < end && c * 8 < P.d;
            int64_t at = 0;
            if (there) {
                const int in = offset + local, pg = page_of(P, in);
                const int id = ids[pg];
                there = id >= 0;
                if (there) at = id * P.page_stride + (in - pg * P.page) * P.token_stride + kv_head * P.head_stride + c * 8;
            }
            copy16(smem_at(k_at) + piece<D>(row, c), P.k + at, there);
            copy16(smem_at(v_at) + piece<D>(row, c), P.v + at, there);
        }
        asm volatile("cp.async.commit_group;");
    };
    char* ring = smem;
    load(0, ring, ring + kTileBytes);

    // queries as the left operand: rows lane / 4 and lane / 4 + 8 of the warp's 16
    uint32_t qf[kSteps][4];
    int64_t out_row[2];
    bool row_in[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int row = first_row + (KEYS_SPLIT ? 0 : warp * 16) + (lane >> 2) + h * 8;
        row_in[h] = row < rows;
        const int b = b0 + row / P.r, head = kv_head * P.r + row % P.r;
        out_row[h] = (int64_t)b * P.H + head;
        const __nv_bfloat16* src = P.q + (row_in[h] ? (int64_t)b * P.q_stride + (int64_t)head * P.d : 0);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int col = s * 16 + e * 8 + (lane & 3) * 2;
                qf[s][e * 2 + h] = row_in[h] && col < P.d ? *reinterpret_cast<const uint32_t*>(src + col) : 0u;
            }
    }
    float o[D / 8][4] = {};
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    const int tiles = (end - begin + kTile - 1) / kTile;
    for (int t = 0; t < tiles; ++t) {
        char* kt = ring + (t & 1) * 2 * kTileBytes;
        char* vt = kt + kTileBytes;
        if (t + 1 < tiles) {
            char* next = ring + ((t + 1) & 1) * 2 * kTileBytes;
            load((t + 1) * kTile, next, next + kTileBytes);
            asm volatile("cp.async.wait_group 1;");
        } else {
            asm volatile("cp.async.wait_group 0;");
        }
        __syncthreads();
        const int key0 = KEYS_SPLIT ? warp * 16 : 0;
        float s[kCols][4] = {};
#pragma unroll
        for (int j = 0; j < kCols; j += 2) {
#pragma unroll
            for (int st = 0; st < kSteps; ++st) {
                uint32_t b[4];                                // keys j*8 .. j*8+15, dimensions st*16 .. +15
                const int row = key0 + j * 8 + (lane & 7) + ((lane >> 4) << 3);
                ldsm4(b, smem_at(kt) + piece<D>(row, st * 2 + ((lane >> 3) & 1)));
                mma(s[j], qf[st], b);
                mma(s[j + 1], qf[st], b + 2);
            }
        }
        const int left = end - begin - t * kTile;             // keys that are there
        if (left < kTile || missing) {
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int key = key0 + j * 8 + (lane & 3) * 2 + e;
                    const bool there = key < left && (!missing || ids[page_of(P, offset + t * kTile + key)] >= 0);
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
            const float now = fmaxf(m[h], top * P.scale_log2);
            const float base = now == -INFINITY ? 0.f : now;
            const float fade = exp2_of(m[h] - base);
            m[h] = now;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < kCols; ++j)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = exp2_of(fmaf(s[j][h * 2 + e], P.scale_log2, -base));
                    s[j][h * 2 + e] = p;
                    sum += p;
                }
            l[h] = l[h] * fade + sum;
#pragma unroll
            for (int n = 0; n < D / 8; ++n) { o[n][h * 2] *= fade; o[n][h * 2 + 1] *= fade; }
        }
        // the weights as two bfloat16 parts: what one rounding would lose is as large as the output's own
#pragma unroll
        for (int j = 0; j < kCols; j += 2) {
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float a = s[j + (e >> 1)][(e & 1) * 2], b = s[j + (e >> 1)][(e & 1) * 2 + 1];
                hi[e] = pack2(a, b);
                lo[e] = pack2(a - __uint_as_float(hi[e] << 16), b - __uint_as_float(hi[e] & 0xffff0000u));
            }
#pragma unroll
            for (int n = 0; n < D / 8; n += 2) {
                uint32_t b[4];                                // keys j*8 .. +15, dimensions n*8 .. +15
                const int row = key0 + j * 8 + (lane & 15);
                ldsm4t(b, smem_at(vt) + piece<D>(row, n + (lane >> 4)));
                mma(o[n], hi, b);
                mma(o[n], lo, b);
                mma(o[n + 1], hi, b + 2);
                mma(o[n + 1], lo, b + 2);
            }
        }
        __syncthreads();
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        l[h] += __shfl_xor_sync(~0u, l[h], 1);
        l[h] += __shfl_xor_sync(~0u, l[h], 2);
    }
    const int64_t seg_rows = (int64_t)slot * P.B * P.H;
    if constexpr (!KEYS_SPLIT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if (!row_in[h]) continue;
            float* dst = P.part_o + (seg_rows + out_row[h]) * D;
#pragma unroll
            for (int n = 0; n < D / 8; ++n)
                *reinterpret_cast<float2*>(dst + n * 8 + (lane & 3) * 2) = make_float2(o[n][h * 2], o[n][h * 2 + 1]);
            if ((lane & 3) == 0) P.part_ml[seg_rows + out_row[h]] = make_float2(m[h], l[h]);
        }
    } else {
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

__device__ __forceinline__ int clamp_to(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }

template <int D>
__global__ void __launch_bounds__(kThreads) attention_kernel(const __grid_constant__ AttnParams P) {
    extern __shared__ __align__(128) char smem[];
    __shared__ int ids[kMaxIds];
    int block = blockIdx.x;
    if (block < P.prefix_blocks) {
        const int tile_slot = block % P.prefix_tiles;
        block /= P.prefix_tiles;
        const int kv_head = block % P.Hk, seg = block / P.Hk;
        // group g's tiles start at slot floor(offset_g r / 64) + g: at least as many slots as tiles for any sizes
        int lo = 0, hi = P.groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if ((int64_t)clamp_to(P.group_offsets[mid], 0, P.B) * P.r / 64 + mid <= tile_slot) lo = mid; else hi = mid - 1;
        }
        const int b0 = clamp_to(P.group_offsets[lo], 0, P.B), b1 = clamp_to(P.group_offsets[lo + 1], b0, P.B);
        const int tile = tile_slot - (int)((int64_t)b0 * P.r / 64 + lo), rows = (b1 - b0) * P.r;
        const int len = clamp_to(P.prefix_lens[lo], 0, P.max_prefix), begin = seg * P.prefix_seg, end = min(len, begin + P.prefix_seg);
        if (tile < 0 || tile * 64 >= rows || begin >= end) return;
        segment<D, false>(P, smem, ids, P.prefix_table + (int64_t)lo * P.prefix_width, P.prefix_width, begin, end, kv_head, tile * 64,
                          rows, b0, seg);
    } else {
        block -= P.prefix_blocks;
        const int tile = block % P.own_tiles;
        block /= P.own_tiles;
        const int kv_head = block % P.Hk;
        block /= P.Hk;
        const int b = block % P.B, seg = block / P.B;
        const int len = clamp_to(P.lens[b], 0, P.max_len), begin = seg * P.own_seg, end = min(len, begin + P.own_seg);
        if (begin >= end) return;
        segment<D, true>(P, smem, ids, P.block_table + (int64_t)b * P.own_width, P.own_width, begin, end, kv_head, tile * 16, P.r, b,
                         P.prefix_segs + seg);
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
    const int64_t want = 148 * 2 * 2;
    int64_t segs = units >= want ? 1 : (want + units - 1) / (units > 0 ? units : 1);
    const int64_t least = divide_up(longest, 4 * kTile);
    if (segs > least) segs = least;
    int64_t len = divide_up(divide_up(longest, segs), kTile) * (int64_t)kTile;
    if (len > most) len = most;
    const int64_t by_ids = (int64_t)(kMaxIds - 2) * page / kTile * kTile;
    return (int)(len < by_ids ? len : by_ids);
}

int plan(AttnParams& P) {
    P.own_tiles = divide_up(P.r, 16);
    P.prefix_tiles = P.groups > 0 ? (int)((int64_t)P.B * P.r / 64) + P.groups : 0;
    P.prefix_seg = plan_segment(P.max_prefix, (int64_t)P.Hk * (P.B * (int64_t)P.r / 64 > 0 ? P.B * (int64_t)P.r / 64 : 1), P.page, 16384);
    P.own_seg = plan_segment(P.max_len, (int64_t)P.B * P.Hk * P.own_tiles, P.page, 1024);
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

template <int D> int launch(const AttnParams& P, cudaStream_t s) {
    constexpr int kSmem = 4 * kTile * D * 2 + 16;
    static_assert(4 * kTile * D * 2 >= 4 * 16 * D * 4, "the warps' shares are joined in the tiles' room");
    const int bytes = kSmem + 4 * 16 * 8;
    if (cudaFuncSetAttribute(attention_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess) return RLCS_ERR_CUDA;
    const int64_t blocks = P.prefix_blocks + (int64_t)P.own_tiles * P.Hk * P.B * P.own_segs;
    if (blocks > 0) attention_kernel<D><<<(unsigned)blocks, kThreads, bytes, s>>>(P);
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
    const size_t rows = (size_t)(P.prefix_segs + P.own_segs) * P.B * P.H;
    P.part_o = static_cast<float*>(workspace);
    P.part_ml = reinterpret_cast<float2*>(P.part_o + rows * (P.d <= 64 ? 64 : 128));
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    return P.d <= 64 ? launch<64>(P, s) : launch<128>(P, s);
}

}  // extern "C"

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
    int tiles;                     // of 16 rows, a trajectory
};

struct Chunk {
    int first, count, start;       // first token of the step, tokens, place of the first in its trajectory (may be negative)
};

__device__ __forceinline__ Chunk chunk_of(const ChunkParams& C, int b) {
    Chunk c;
    c.first = clamp_to(C.offsets[b], 0, C.a.B);
    c.count = clamp_to(C.offsets[b + 1], c.first, C.a.B) - c.first;
    c.start = clamp_to(C.a.lens[b], 0, 0x7fffff00) - c.count;      // no sum with rows of a tile wraps
    c.count = min(c.count, C.max_new);
    return c;
}

// Keys that the rows below `rows` of a chunk see, at most.
__device__ __forceinline__ int keys_of(const ChunkParams& C, const Chunk& c, int rows) {
    return clamp_to(c.start + (rows + C.a.r - 1) / C.a.r, 0, C.a.max_len);
}

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
    if (begin >= end) return;
    segment<D, TMA, true>(P, &k_map, &v_map, raw, ids, bars, &gave_up, P.block_table + (int64_t)b * P.own_width, P.own_width, begin, end, kv_head,
                          first_row, rows, c.first, seg, c.start + 1 - begin);
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
    C.max_new = (int)(max_new < T ? max_new : T);
    if (T == 0 || H == 0 || seqs == 0 || C.max_new == 0) return RLCS_OK;
    if ((int64_t)C.max_new * P.r > (1 << 30)) return RLCS_ERR_SIZE;
    C.tiles = divide_up((int64_t)C.max_new * P.r, 16);
    P.own_seg = plan_segment(P.max_len, (int64_t)C.tiles * Hk * seqs, P.page, 1024);
    P.own_segs = divide_up(P.max_len, P.own_seg);
    if ((double)C.tiles * Hk * seqs * P.own_segs > 2147483647.0) return RLCS_ERR_SIZE;
    return RLCS_OK;
}

size_t workspace_of(const ChunkParams& C) {
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

template <int D> int launch(const ChunkParams& C, cudaStream_t s) {
    CUtensorMap k_map = {}, v_map = {};
    const AttnParams& P = C.a;
    const int64_t blocks = (int64_t)C.tiles * P.Hk * C.seqs * P.own_segs;
    if (blocks > 0) {
        const bool boxes = box_map(&k_map, P, P.k, kPart) && box_map(&v_map, P, P.v, kPart);
        const int st = boxes ? launch_chunk<D, true>(C, blocks, k_map, v_map, s) : launch_chunk<D, false>(C, blocks, k_map, v_map, s);
        if (st != RLCS_OK) return st;
    }
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
    if (workspace == nullptr || workspace_bytes < workspace_of(C)) return RLCS_ERR_WORKSPACE;
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

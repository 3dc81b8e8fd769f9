// Page tables, slot maps and positions of one step of a paged cache, from lengths that live on the GPU.
//
//   have_b = ceil(cached_b / page),  need_b = ceil((cached_b + added_b) / page)          pages of row b before and after
//   new pages come from the free list in row order: row b's i-th is free[sum_{c<b} (need_c - have_c) + i]
//   token number t of the step (rows one after the other) sits at position cached_b + t - sum_{c<b} added_c of its row b
//
// Two exclusive sums over the rows, then two outputs filled element by element.  Up to kFused rows every block makes the sums
// itself, in shared memory (2048 rows: about 2 us, what a second launch would cost), beyond one block makes them first.
// Small steps are bound by their launch (128 rows: 6 us on the GPU); 2048 prompts of 1024 tokens write 25 MB in 19 us, where the sums and
// one page lookup a token show (34 us with a token a thread, 64-bit divisions and two launches).
#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"

namespace {

struct TableParams {
    const int32_t* cached;
    const int32_t* added;
    const int32_t* free_pages;
    int32_t* table;
    int64_t* slots;
    int32_t* positions;
    int32_t* offsets;          // [B + 1] tokens before each row
    int32_t* page_offsets;     // [B + 1] new pages before each row
    int64_t num_slots;
    int32_t B, width, free_count, page;
    bool wide_slots, wide_positions, wide_table;       // 16-byte stores
};

struct Row {
    int have, fresh, cached, added;      // pages held and to be added (within the table's width), lengths
};

__device__ __forceinline__ Row row_of(const TableParams& P, int b) {
    const int cached = max(P.cached[b], 0), added = min(max(P.added[b], 0), 0x7fffffff - cached);
    const uint32_t page = P.page, width = P.width;
    const uint32_t have = min(((uint32_t)cached + page - 1) / page, width);      // page <= 2^24: no overflow
    const uint32_t need = min(((uint32_t)(cached + added) + page - 1) / page, width);
    return Row{(int)have, (int)(need - have), cached, added};
}

constexpr int kThreads = 256, kFused = 4096;

// Exclusive sums of (tokens, new pages) over all rows by the T threads of a block, to `offsets` and `pages` [B + 1].
template <int T> __device__ __forceinline__ void row_sums(const TableParams& P, int32_t* offsets, int32_t* pages) {
    __shared__ int2 part[T / 32];
    int2 carry = {0, 0};
    for (int base = 0; base < P.B; base += T) {
        const int b = base + threadIdx.x;
        int2 v = {0, 0};
        if (b < P.B) {
            const Row r = row_of(P, b);
            v = make_int2(r.added, r.fresh);
        }
        int2 s = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(~0u, s.x, o), y = __shfl_up_sync(~0u, s.y, o);
            if ((threadIdx.x & 31) >= o) { s.x += x; s.y += y; }
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 31) part[threadIdx.x >> 5] = s;
        __syncthreads();
        int2 all = {0, 0};
#pragma unroll 8
        for (int k = 0; k < T / 32; ++k) {
            if (k == (threadIdx.x >> 5)) { s.x += all.x; s.y += all.y; }
            all.x += part[k].x;
            all.y += part[k].y;
        }
        if (b < P.B) {
            offsets[b] = carry.x + s.x - v.x;
            pages[b] = carry.y + s.y - v.y;
        }
        carry.x += all.x;
        carry.y += all.y;
    }
    if (threadIdx.x == 0) {
        offsets[P.B] = carry.x;
        pages[P.B] = carry.y;
    }
}

__global__ void __launch_bounds__(1024) table_sums_kernel(const __grid_constant__ TableParams P) { row_sums<1024>(P, P.offsets, P.page_offsets); }

template <bool FUSED>
__global__ void __launch_bounds__(kThreads) table_fill_kernel(const __grid_constant__ TableParams P) {
    extern __shared__ int32_t sums[];
    const int32_t *offsets = P.offsets, *pages = P.page_offsets;
    if constexpr (FUSED) {
        row_sums<kThreads>(P, sums, sums + P.B + 1);
        __syncthreads();
        offsets = sums;
        pages = sums + P.B + 1;
        if (blockIdx.x == 0)
            for (int b = threadIdx.x; b <= P.B; b += kThreads) {
                P.offsets[b] = offsets[b];
                P.page_offsets[b] = pages[b];
            }
    }
    const int64_t step = (int64_t)gridDim.x * kThreads * 4, first = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    const int64_t cells = (int64_t)P.B * P.width;
    for (int64_t e = first; e < cells; e += step) {
        int b = cells <= 0x7fffffff ? (int)((uint32_t)e / (uint32_t)P.width) : (int)(e / P.width);
        int j = (int)(e - (int64_t)b * P.width);
        Row r = row_of(P, b);
        int32_t v[4];
        bool fresh[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            fresh[k] = false;
            v[k] = -1;
            if (e + k >= cells) continue;
            if (j == P.width) {
                j = 0;
                r = row_of(P, ++b);
            }
            fresh[k] = j >= r.have;
            if (fresh[k] && j < r.have + r.fresh) {
                const int at = pages[b] + j - r.have;
                if (at < P.free_count) v[k] = P.free_pages[at];
            }
            ++j;
        }
        if (P.wide_table && fresh[0] && fresh[1] && fresh[2] && fresh[3]) {
            *reinterpret_cast<int4*>(P.table + e) = make_int4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (fresh[k]) P.table[e + k] = v[k];
        }
    }
    const int total = offsets[P.B];
    for (int64_t t = first; t < P.num_slots; t += step) {
        long long slot[4] = {-1, -1, -1, -1};
        int pos[4] = {-1, -1, -1, -1};
        if (t < total) {
            int b = 0, hi = P.B - 1;                      // the last row that starts at or before t (empty rows skipped)
            while (b < hi) {
                const int mid = (b + hi + 1) >> 1;
                if (offsets[mid] <= t) b = mid; else hi = mid - 1;
            }
            Row r = row_of(P, b);
            int end = offsets[b + 1], at_page = -1, id = -1;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (t + k >= total) break;
                if (t + k >= end) {                       // on to the next row that has tokens
                    do end = offsets[++b + 1]; while (t + k >= end);
                    r = row_of(P, b);
                    at_page = -1;
                }
                pos[k] = r.cached + (int)(t + k - offsets[b]);
                const int j = (int)((uint32_t)pos[k] / (uint32_t)P.page);
                if (j != at_page) {
                    at_page = j;
                    id = -1;
                    if (j < r.have) {
                        id = P.table[(int64_t)b * P.width + j];
                    } else if (j < P.width) {
                        const int at = pages[b] + j - r.have;
                        if (at < P.free_count) id = P.free_pages[at];
                    }
                }
                if (id >= 0) slot[k] = (long long)id * P.page + (pos[k] - j * P.page);
            }
        }
        if (P.wide_slots && t + 3 < P.num_slots) {
            *reinterpret_cast<longlong2*>(P.slots + t) = make_longlong2(slot[0], slot[1]);
            *reinterpret_cast<longlong2*>(P.slots + t + 2) = make_longlong2(slot[2], slot[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (t + k < P.num_slots) P.slots[t + k] = slot[k];
        }
        if (P.wide_positions && t + 3 < P.num_slots) {
            *reinterpret_cast<int4*>(P.positions + t) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (t + k < P.num_slots) P.positions[t + k] = pos[k];
        }
    }
}

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

}  // namespace

extern "C" int rlcs_block_tables(const int32_t* cached, const int32_t* added, const int32_t* free_pages, int32_t* block_table,
                                 int64_t* slots, int32_t* positions, int32_t* offsets, int32_t* page_offsets, int64_t B,
                                 int64_t width, int64_t free_count, int64_t num_slots, int64_t page_size, void* cuda_stream) {
    const int64_t kMost = (int64_t(1) << 31) - 1;
    if (B < 0 || width < 0 || free_count < 0 || num_slots < 0 || page_size < 0) return RLCS_ERR_SIZE;
    if (B >= (int64_t(1) << 24) || width > (int64_t(1) << 24) || free_count > kMost || num_slots > kMost || page_size > (int64_t(1) << 24))
        return RLCS_ERR_SIZE;
    if (page_size == 0) return RLCS_ERR_ARG;
    if (offsets == nullptr || page_offsets == nullptr || (B > 0 && (cached == nullptr || added == nullptr)) ||
        (B > 0 && width > 0 && block_table == nullptr) || (free_count > 0 && free_pages == nullptr) ||
        (num_slots > 0 && (slots == nullptr || positions == nullptr)))
        return RLCS_ERR_NULL;
    const void* words[] = {cached, added, free_pages, block_table, positions, offsets, page_offsets};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    if (!aligned_to(slots, 8)) return RLCS_ERR_ALIGN;
    const TableParams P = {cached, added, free_pages, block_table, slots, positions, offsets, page_offsets, num_slots,
                           (int32_t)B, (int32_t)width, (int32_t)free_count, (int32_t)page_size, aligned_to(slots, 16), aligned_to(positions, 16),
                           aligned_to(block_table, 16)};
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const int64_t most = B * width > num_slots ? B * width : num_slots, sms = rlcs_device::limits().sms;
    int64_t blocks = (most + kThreads * 4 - 1) / (kThreads * 4);
    blocks = blocks < 1 ? 1 : blocks;
    if (B <= kFused) {
        if (blocks > 4 * sms) blocks = 4 * sms;
        table_fill_kernel<true><<<(unsigned)blocks, kThreads, 2 * (B + 1) * sizeof(int32_t), s>>>(P);
    } else {
        table_sums_kernel<<<1, 1024, 0, s>>>(P);
        if (blocks > 8 * sms) blocks = 8 * sms;
        table_fill_kernel<false><<<(unsigned)blocks, kThreads, 0, s>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

// Page tables, slot maps and positions of one step of a paged cache, from lengths that live on the GPU.
//
//   have_b = ceil(cached_b / page),  need_b = ceil((cached_b + added_b) / page)          pages of row b before and after
//   new pages come from the free list in row order: row b's i-th is free[sum_{c<b} (need_c - have_c) + i]
//   token number t of the step (rows one after the other) sits at position cached_b + t - sum_{c<b} added_c of its row b
//
// Two exclusive sums over the rows, then two outputs filled element by element.
#include <cstdint>

#include "../../include/rlcs.h"

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
};

struct Row {
    int have, fresh, cached, added;      // pages held and to be added (within the table's width), lengths
};

__device__ __forceinline__ Row row_of(const TableParams& P, int b) {
    const int cached = max(P.cached[b], 0), added = max(P.added[b], 0);
    const int64_t page = P.page;
    const int have = (int)min(((int64_t)cached + page - 1) / page, (int64_t)P.width);
    const int need = (int)min(((int64_t)cached + added + page - 1) / page, (int64_t)P.width);
    return Row{have, need - have, cached, added};
}

constexpr int kThreads = 256;

// Exclusive sums over all rows, by one block.
__global__ void __launch_bounds__(1024) table_sums_kernel(const __grid_constant__ TableParams P) {
    __shared__ int2 part[32];
    int2 carry = {0, 0};
    for (int base = 0; base < P.B; base += 1024) {
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
        for (int k = 0; k < 32; ++k) {
            if (k == (threadIdx.x >> 5)) { s.x += all.x; s.y += all.y; }
            all.x += part[k].x;
            all.y += part[k].y;
        }
        if (b < P.B) {
            P.offsets[b] = carry.x + s.x - v.x;
            P.page_offsets[b] = carry.y + s.y - v.y;
        }
        carry.x += all.x;
        carry.y += all.y;
    }
    if (threadIdx.x == 0) {
        P.offsets[P.B] = carry.x;
        P.page_offsets[P.B] = carry.y;
    }
}

__global__ void __launch_bounds__(kThreads) table_fill_kernel(const __grid_constant__ TableParams P) {
    const int64_t step = (int64_t)gridDim.x * kThreads, first = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    for (int64_t e = first; e < (int64_t)P.B * P.width; e += step) {
        const int b = (int)(e / P.width), j = (int)(e - (int64_t)b * P.width);
        const Row r = row_of(P, b);
        if (j < r.have) continue;
        const int at = P.page_offsets[b] + j - r.have;
        P.table[e] = j < r.have + r.fresh && at < P.free_count ? P.free_pages[at] : -1;
    }
    const int total = P.offsets[P.B];
    for (int64_t t = first; t < P.num_slots; t += step) {
        int64_t slot = -1;
        int pos = -1;
        if (t < total) {
            int lo = 0, hi = P.B - 1;                     // the last row that starts at or before t (empty rows skipped)
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (P.offsets[mid] <= t) lo = mid; else hi = mid - 1;
            }
            const Row r = row_of(P, lo);
            pos = r.cached + (int)(t - P.offsets[lo]);
            const int j = pos / P.page;
            if (j < P.width) {
                int id = -1;
                if (j < r.have) {
                    id = P.table[(int64_t)lo * P.width + j];
                } else {
                    const int at = P.page_offsets[lo] + j - r.have;
                    if (at < P.free_count) id = P.free_pages[at];
                }
                if (id >= 0) slot = (int64_t)id * P.page + (pos - j * P.page);
            }
        }
        P.slots[t] = slot;
        P.positions[t] = pos;
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
                           (int32_t)B, (int32_t)width, (int32_t)free_count, (int32_t)page_size};
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    table_sums_kernel<<<1, 1024, 0, s>>>(P);
    const int64_t most = B * width > num_slots ? B * width : num_slots;
    int64_t blocks = (most + kThreads - 1) / kThreads;
    if (blocks > 148 * 8) blocks = 148 * 8;
    if (blocks > 0) table_fill_kernel<<<(unsigned)blocks, kThreads, 0, s>>>(P);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

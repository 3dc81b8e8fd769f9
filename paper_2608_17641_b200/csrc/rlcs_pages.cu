// Pages of a paged cache: trajectories continued from others, copies of pages, and the pages that nobody names.
//
//   fork    new row i is the old row sources[i]: whole pages are shared, a part-filled last page stays with the first row that ends
//           in it, unless another has it whole, and is copied for the others, to pages taken from the free list in row order
//   copy    pages from[i] -> to[i] of keys and values
//   free    the numbers below num_pages that no live entry of the tables names, ascending
//
// What a page is shared by needs no counts: it is free when no table names it.
//
// Measured: 2048 rows forked and about 750 pages of 128 KB copied in both caches 77 us, of which the copies 65 (0.92 of the copy bandwidth),
// tables and numbers of all rows 12; 8 rows 8.3 us with their copies, a chain of a block's lookups; free pages among 9192 of 128 rows 6.8 us (one block), among 2.2 million of 4096 rows 22 us: 13 for 1.4 million
// marks in L2 (plain stores of bytes took 10 more), 8 for the list, whose counts every block makes itself instead of another launch.
#include <cooperative_groups.h>

#include <cstdint>

#include "../../include/rlcs.h"
#include "rlcs_device.cuh"

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256, kFused = 4096;

bool aligned_to(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// ---------------------------------------------------------------------------------------------- fork
// Who keeps a part-filled page goes by its number, not by the row that it comes from: branches share pages, and when they are cut back a
// page that is whole for one may be part-filled for another, or for both.  A table of the part-filled pages' numbers (open addressing, at
// most half full) has the first new row that ends in each, and whether a new row has it as a whole page; then nobody may write there.
struct ForkParams {
    const int32_t* table;
    const int32_t* lens;
    const int32_t* sources;
    const int32_t* free_pages;
    int32_t* out;
    int32_t* from;
    int32_t* to;
    int32_t* used;
    int32_t* keys;             // [slots] page numbers, -1: none                         } of large calls
    uint32_t* owner;           // [slots] first new row that ends there + 1, 0: nobody   }
    int32_t* number;           // [N] slot, then place in the free list; -1: none        }
    int32_t B, N, width, free_count, page;
    int32_t slots, shift;      // a power of two, and 32 - its logarithm
    bool fill;                 // whether fork_kernel writes whole tables
};

struct OldRow {
    int source, have, last;    // last: the page that a second row would copy, -1 without one
};

__device__ __forceinline__ uint32_t pages_of(int len, int page) { return ((uint32_t)max(len, 0) + page - 1) / (uint32_t)page; }      // page <= 2^24: no overflow

__device__ __forceinline__ OldRow old_row(const ForkParams& P, int i) {
    OldRow r = {P.sources[i], 0, -1};
    if (r.source < 0 || r.source >= P.B) { r.source = -1; return r; }
    const int len = max(P.lens[r.source], 0);
    const uint32_t need = pages_of(len, P.page);
    r.have = (int)min(need, (uint32_t)P.width);
    if (need <= (uint32_t)P.width && len % P.page != 0) r.last = P.table[(int64_t)r.source * P.width + r.have - 1];
    return r;
}

// Pages that a row of this length fills, of those that the table holds.
__device__ __forceinline__ int whole_of(const ForkParams& P, int len) { return min(max(len, 0) / P.page, P.width); }

__device__ __forceinline__ int slot_at(const ForkParams& P, int page) { return (int)((uint32_t)page * 2654435769u >> P.shift); }

__device__ __forceinline__ int find_slot(const ForkParams& P, const int32_t* keys, int page) {
    for (int h = slot_at(P, page);; h = (h + 1) & (P.slots - 1)) {      // half of the slots are free
        const int k = keys[h];
        if (k == page || k < 0) return k < 0 ? -1 : h;
    }
}

// Row i ends in `page`: its slot.
__device__ __forceinline__ int enter_page(const ForkParams& P, int32_t* keys, uint32_t* owner, int page, int i) {
    int h = slot_at(P, page);
    for (;; h = (h + 1) & (P.slots - 1)) {
        const int k = atomicCAS(keys + h, -1, page);
        if (k == -1 || k == page) break;
    }
    atomicMin(owner + h, (uint32_t)i + 1);
    return h;
}

// The page that row i takes from the free list.
__device__ __forceinline__ int taken(const ForkParams& P, int number) {
    return number >= 0 && number < P.free_count ? max(P.free_pages[number], -1) : -1;
}

// number[i] from slots to places in the free list, for every row that needs a page; the rest -1.  By the T threads of a block, four rows a
// thread at a time.
template <int T> __device__ __forceinline__ void fork_numbers(const ForkParams& P, const uint32_t* owner, int32_t* number, bool write) {
    constexpr int kRows = 4;
    __shared__ int part[kRows][T / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int carry = 0;
    for (int base = 0; base < P.N; base += kRows * T) {
        int slot[kRows];
        unsigned some[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int i = base + k * T + threadIdx.x;
            slot[k] = i < P.N ? number[i] : -1;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int i = base + k * T + threadIdx.x;
            some[k] = __ballot_sync(~0u, slot[k] >= 0 && owner[slot[k]] != (uint32_t)i + 1);
            if (lane == 0) part[k][warp] = __popc(some[k]);
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const int i = base + k * T + threadIdx.x;
            const int each = lane < T / 32 ? part[k][lane] : 0;
            const int before = carry + __reduce_add_sync(~0u, lane < warp ? each : 0);
            carry += __reduce_add_sync(~0u, each);
            if (i < P.N) number[i] = some[k] >> lane & 1 ? before + __popc(some[k] & ((1u << lane) - 1)) : -1;
        }
    }
    if (write && threadIdx.x == 0) *P.used = carry;
}

// The new tables as if nothing were copied, entries from `me` on.
__device__ __forceinline__ void gather_tables(const ForkParams& P, int64_t me, int64_t step) {
    const int64_t cells = (int64_t)P.N * P.width;
    for (int64_t e = me; e < cells; e += step) {
        const int i = cells <= 0x7fffffff ? (int)((uint32_t)e / (uint32_t)P.width) : (int)(e / P.width);
        const int j = (int)(e - (int64_t)i * P.width);
        const int s = P.sources[i];
        P.out[e] = s >= 0 && s < P.B && (uint32_t)j < pages_of(P.lens[s], P.page) ? P.table[(int64_t)s * P.width + j] : -1;
    }
}

// What row i copies, and its table's last entry where it does.
__device__ __forceinline__ void give_page(const ForkParams& P, int i, int number) {
    const int page = taken(P, number);
    P.to[i] = page;
    int from = -1;
    if (number >= 0) {
        const OldRow r = old_row(P, i);
        P.out[(int64_t)i * P.width + r.have - 1] = page;
        if (page >= 0) from = r.last;
    }
    P.from[i] = from;
}

constexpr int kWide = 1024;                  // threads where a block goes through all rows
constexpr int kMostWays = 8;                 // blocks that share the whole pages
constexpr int64_t kMostCells = 98304;        // entries of either table up to which they do (1024 rows of 64 15 us; 4096 of 64 36, and
                                             // 18 in launches of their own)

// Up to kFused rows and kMostCells entries: the table of pages in the shared memory of each block of one cluster.  All blocks enter all rows; each looks a share of
// the old tables' whole pages up, and tells the others what it finds (seldom anything); the numbers are again every block's own.
__global__ void __launch_bounds__(kWide) fork_kernel(const __grid_constant__ ForkParams P) {
    extern __shared__ int32_t held[];
    int32_t* const keys = held;
    uint32_t* const owner = reinterpret_cast<uint32_t*>(held + P.slots);
    int32_t* const number = held + 2 * P.slots;
    uint32_t* const continued = reinterpret_cast<uint32_t*>(number + P.N);      // a bit an old row
    const cg::cluster_group cluster = cg::this_cluster();
    const int ways = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), tid = threadIdx.x;
    auto sync = [&] { if (ways > 1) cluster.sync(); else __syncthreads(); };
    for (int h = tid; h < P.slots; h += kWide) { keys[h] = -1; owner[h] = ~0u; }
    for (int w = tid; w < (P.B + 31) / 32; w += kWide) continued[w] = 0;
    __syncthreads();
    for (int base = 0; base < P.N; base += 4 * kWide) {
        OldRow r[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = base + k * kWide + tid;
            r[k] = OldRow{-1, 0, -1};
            if (i < P.N) r[k] = old_row(P, i);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = base + k * kWide + tid;
            if (r[k].source >= 0) atomicOr(continued + (r[k].source >> 5), 1u << (r[k].source & 31));
            if (i < P.N) number[i] = r[k].last >= 0 ? enter_page(P, keys, owner, r[k].last, i) : -1;
        }
    }
    sync();
    const int64_t cells = (int64_t)P.B * P.width, step = (int64_t)ways * kWide, me = (int64_t)rank * kWide + tid;
    for (int64_t e = me; e < cells; e += 4 * step) {
        int id[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int64_t at = e + k * step;
            id[k] = -1;
            if (at >= cells) continue;
            const int s = cells <= 0x7fffffff ? (int)((uint32_t)at / (uint32_t)P.width) : (int)(at / P.width);
            if ((continued[s >> 5] >> (s & 31) & 1) && (int)(at - (int64_t)s * P.width) < whole_of(P, P.lens[s])) id[k] = P.table[at];
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (id[k] < 0 || find_slot(P, keys, id[k]) < 0) continue;
            for (int w = 0; w < ways; ++w) {                  // each block has its own order of the keys
                const int h = find_slot(P, cluster.map_shared_rank(keys, w), id[k]);
                if (h >= 0) cluster.map_shared_rank(owner, w)[h] = 0;
            }
        }
    }
    sync();
    fork_numbers<kWide>(P, owner, number, rank == 0);
    if (P.fill) gather_tables(P, me, step);
    sync();                                                   // the last entries below may be another block's
    for (int64_t i = me; i < P.N; i += step) give_page(P, (int)i, number[i]);
}

__global__ void __launch_bounds__(kThreads) fork_gather_kernel(const __grid_constant__ ForkParams P) {
    gather_tables(P, (int64_t)blockIdx.x * kThreads + threadIdx.x, (int64_t)gridDim.x * kThreads);
}

// The same for larger tables, the table of pages in the workspace or in place of outputs that are written later.
__global__ void __launch_bounds__(kThreads) fork_enter_kernel(const __grid_constant__ ForkParams P) {
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < P.N; i += gridDim.x * kThreads) {
        const int last = old_row(P, i).last;
        P.number[i] = last >= 0 ? enter_page(P, P.keys, P.owner, last, i) : -1;
    }
}

__global__ void __launch_bounds__(kThreads) fork_whole_kernel(const __grid_constant__ ForkParams P) {
    const int64_t cells = (int64_t)P.N * P.width;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < cells; e += (int64_t)gridDim.x * kThreads) {
        const int i = cells <= 0x7fffffff ? (int)((uint32_t)e / (uint32_t)P.width) : (int)(e / P.width), j = (int)(e - (int64_t)i * P.width);
        const int s = P.sources[i];
        if (s < 0 || s >= P.B || j >= whole_of(P, P.lens[s])) continue;
        const int id = P.table[(int64_t)s * P.width + j], h = id >= 0 ? find_slot(P, P.keys, id) : -1;
        if (h >= 0) P.owner[h] = 0;
    }
}

__global__ void __launch_bounds__(kWide) fork_numbers_kernel(const __grid_constant__ ForkParams P) { fork_numbers<kWide>(P, P.owner, P.number, true); }

__global__ void __launch_bounds__(kThreads) fork_give_kernel(const __grid_constant__ ForkParams P) {
    for (int i = blockIdx.x * kThreads + threadIdx.x; i < P.N; i += gridDim.x * kThreads) give_page(P, i, P.number[i]);
}

// Slots for the part-filled pages: twice as many as there can be, a power of two.
int64_t fork_slots(int64_t B, int64_t N) {
    const int64_t least = 2 * (B < N ? B : N);
    int64_t slots = 2;
    while (slots < least) slots *= 2;
    return slots;
}

// ---------------------------------------------------------------------------------------------- copy
struct CopyParams {
    char* cache[2];
    const int32_t* from;
    const int32_t* to;
    int64_t pages, page_stride, token_stride, head_stride;      // strides in bytes
    int32_t N, caches, page, Hk, row;                           // row: bytes of one head of one token
    int64_t page_bytes;                                         // of a page without gaps, else 0
};

constexpr int kPairs = 1024, kCopyBlocks = 4, kPiece = kThreads * 16 * 4;        // bytes a block copies at a time

__global__ void __launch_bounds__(kThreads, kCopyBlocks) copy_kernel(const __grid_constant__ CopyParams P) {
    __shared__ int2 pairs[kPairs];
    __shared__ int counts[kPairs / 32];
    static_assert(kPairs == 32 * 32, "a lane a count");
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t bytes = (int64_t)P.page * P.Hk * P.row, pieces = (bytes + kPiece - 1) / kPiece;
    for (int base = 0; base < P.N; base += kPairs) {
        // the pairs that are there, in their order: every block has the same list
        const int most = min(P.N - base, kPairs);
        int2 p[kPairs / kThreads];
        unsigned some[kPairs / kThreads];
        __syncthreads();                                      // the last list has been read
#pragma unroll
        for (int k = 0; k < kPairs / kThreads; ++k) {
            const int i = k * kThreads + threadIdx.x;
            p[k] = i < most ? make_int2(P.from[base + i], P.to[base + i]) : make_int2(-1, -1);
        }
#pragma unroll
        for (int k = 0; k < kPairs / kThreads; ++k) {
            some[k] = __ballot_sync(~0u, p[k].x >= 0 && p[k].x < P.pages && p[k].y >= 0 && p[k].y < P.pages && p[k].x != p[k].y);
            if (lane == 0) counts[k * (kThreads / 32) + warp] = __popc(some[k]);
        }
        __syncthreads();
        const int each = counts[lane], count = __reduce_add_sync(~0u, each);
#pragma unroll
        for (int k = 0; k < kPairs / kThreads; ++k) {
            const int before = __reduce_add_sync(~0u, lane < k * (kThreads / 32) + warp ? each : 0);
            if (some[k] >> lane & 1) pairs[before + __popc(some[k] & ((1u << lane) - 1))] = p[k];
        }
        __syncthreads();
        const int64_t items = (int64_t)count * pieces * P.caches;
        for (int64_t w = blockIdx.x; w < items; w += gridDim.x) {
            const int2 p = pairs[w / (pieces * P.caches)];
            const int64_t rest = w % (pieces * P.caches), piece = rest % pieces;
            char* cache = P.cache[rest / pieces];
            const char* src = cache + p.x * P.page_stride;
            char* dst = cache + p.y * P.page_stride;
            uint4 v[4];
            int64_t at[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int64_t o = piece * kPiece + (k * kThreads + threadIdx.x) * 16;
                at[k] = -1;
                if (o < bytes) {
                    if (P.page_bytes) {
                        at[k] = o;
                    } else {                                   // tokens, heads, pieces of a head
                        const int64_t unit = o / P.row;
                        at[k] = unit / P.Hk * P.token_stride + unit % P.Hk * P.head_stride + o % P.row;
                    }
                    v[k] = *reinterpret_cast<const uint4*>(src + at[k]);
                }
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (at[k] >= 0) *reinterpret_cast<uint4*>(dst + at[k]) = v[k];
        }
    }
}

// ---------------------------------------------------------------------------------------------- free
struct FreeParams {
    const int32_t* table[2];
    const int32_t* lens[2];
    int32_t rows[2], width[2];
    uint32_t* bits;            // of the pages that are named
    int32_t* out;
    int32_t* count;
    int32_t pages, words, page;
};

// Marks what a table names, a warp a row, four entries a lane at a time.
__device__ __forceinline__ void mark_rows(const FreeParams& P, int t, uint32_t* bits, int first, int warps) {
    const int lane = threadIdx.x & 31;
    for (int b = first; b < P.rows[t]; b += warps) {
        const uint32_t need = ((uint32_t)max(P.lens[t][b], 0) + P.page - 1) / (uint32_t)P.page;
        const int have = (int)min(need, (uint32_t)P.width[t]);
        const int32_t* row = P.table[t] + (int64_t)b * P.width[t];
        for (int j = lane; j < have; j += 128) {
            int id[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) id[k] = j + k * 32 < have ? row[j + k * 32] : -1;
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (id[k] >= 0 && id[k] < P.pages) atomicOr(bits + (id[k] >> 5), 1u << (id[k] & 31));
        }
    }
}

__global__ void __launch_bounds__(kThreads) free_mark_kernel(const __grid_constant__ FreeParams P) {
#pragma unroll 1
    for (int t = 0; t < 2; ++t) mark_rows(P, t, P.bits, blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32));
}

// Free pages among the 32 of a word; the words behind the last are a whole vector's, and 0.
__device__ __forceinline__ uint32_t spare_of(const FreeParams& P, uint32_t bits, int word) {
    if (word >= P.words) return 0u;
    return ~bits & (word == P.words - 1 && (P.pages & 31) ? ~(~0u << (P.pages & 31)) : ~0u);
}

constexpr int kList = 1024;

// The list of words [begin, end), and this block's share of the -1 behind the list: every block counts the free pages before its own
// words, and of all of them, itself, sixteen words a thread at a time.
__device__ __forceinline__ void list_words(const FreeParams& P, const uint32_t* bits, int begin, int end, int block, int blocks) {
    __shared__ int part[2][kList / 32], totals[kList / 32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int before = 0, all = 0;                                  // of whole vectors: `begin` is a multiple of four
    const uint4* quads = reinterpret_cast<const uint4*>(bits);
    const int n = (P.words + 3) / 4;
    for (int w = threadIdx.x; w < n; w += 4 * kList) {
        uint4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = w + k * kList < n ? quads[w + k * kList] : make_uint4(~0u, ~0u, ~0u, ~0u);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = w + k * kList;
            int spare = __popc(~v[k].x) + __popc(~v[k].y) + __popc(~v[k].z) + __popc(~v[k].w);
            if (at == n - 1)                                  // words and bits behind the last page count as marked
                spare = __popc(spare_of(P, v[k].x, at * 4)) + __popc(spare_of(P, v[k].y, at * 4 + 1)) + __popc(spare_of(P, v[k].z, at * 4 + 2)) +
                        __popc(spare_of(P, v[k].w, at * 4 + 3));
            all += spare;
            before += at * 4 < begin ? spare : 0;
        }
    }
    before = __reduce_add_sync(~0u, before);
    all = __reduce_add_sync(~0u, all);
    const int share = (end - begin + kList / 32 - 1) / (kList / 32), w0 = min(begin + warp * share, end), w1 = min(w0 + share, end);
    int mine = 0;
    for (int w = w0 + lane; w < w1; w += 32) mine += __popc(spare_of(P, bits[w], w));
    mine = __reduce_add_sync(~0u, mine);
    if (lane == 0) { part[0][warp] = before; part[1][warp] = all; totals[warp] = mine; }
    __syncthreads();
    before = __reduce_add_sync(~0u, part[0][lane] + (lane < warp ? totals[lane] : 0));
    all = __reduce_add_sync(~0u, part[1][lane]);
    for (int w = w0; w < w1; ++w) {
        const uint32_t spare = spare_of(P, bits[w], w);
        if (spare >> lane & 1) P.out[before + __popc(spare & ((1u << lane) - 1))] = w * 32 + lane;
        before += __popc(spare);
    }
    if (block == 0 && threadIdx.x == 0) *P.count = all;
    for (int64_t i = all + (int64_t)block * kList + threadIdx.x; i < P.pages; i += (int64_t)blocks * kList) P.out[i] = -1;
}

__global__ void __launch_bounds__(kList) free_list_kernel(const __grid_constant__ FreeParams P) {
    const int per = ((P.words + gridDim.x - 1) / gridDim.x + 3) / 4 * 4, begin = min((int)blockIdx.x * per, (P.words + 3) / 4 * 4);
    list_words(P, P.bits, begin, min(begin + per, P.words), blockIdx.x, gridDim.x);
}

// Small caches and tables: one block, the marks in shared memory.  A warp a row up to 256 rows (128 rows of 64: 6.8 us, 8.1 the other way),
// an entry a thread wherever its row is beyond (1401 rows of three: 12 us, 30 the other way).
constexpr int kAlonePages = 65536, kAloneEntries = 32768;

__global__ void __launch_bounds__(kList) free_alone_kernel(const __grid_constant__ FreeParams P) {
    __shared__ __align__(16) uint32_t bits[kAlonePages / 32 + 4];
    for (int w = threadIdx.x; w < (P.words + 3) / 4 * 4; w += kList) bits[w] = 0;
    __syncthreads();
#pragma unroll 1
    for (int t = 0; t < 2; ++t) {
        if (P.rows[t] <= 256) {
            mark_rows(P, t, bits, threadIdx.x >> 5, kList / 32);
            continue;
        }
        const int cells = P.rows[t] * P.width[t];             // at most kAloneEntries
        for (int e = threadIdx.x; e < cells; e += 4 * kList) {
            int id[4], len[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int at = e + k * kList;
                id[k] = at < cells ? P.table[t][at] : -1;
                len[k] = at < cells ? P.lens[t][at / P.width[t]] : 0;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t need = ((uint32_t)max(len[k], 0) + P.page - 1) / (uint32_t)P.page;
                if ((uint32_t)(e + k * kList) % (uint32_t)P.width[t] < need && id[k] >= 0 && id[k] < P.pages) atomicOr(bits + (id[k] >> 5), 1u << (id[k] & 31));
            }
        }
    }
    __syncthreads();
    list_words(P, bits, 0, P.words, 0, 1);
}

}  // namespace

extern "C" {

size_t rlcs_fork_block_tables_workspace_bytes(int64_t B, int64_t N) {
    if (B <= 0 || N <= 0 || (B <= kFused && N <= kFused) || B >= (int64_t(1) << 24) || N >= (int64_t(1) << 24)) return 0;
    return (size_t)(2 * fork_slots(B, N) + N) * sizeof(int32_t);
}

int rlcs_fork_block_tables(const int32_t* block_table, const int32_t* lens, const int32_t* sources, const int32_t* free_pages,
                           int32_t* new_table, int32_t* copy_from, int32_t* copy_to, int32_t* pages_used, int64_t B, int64_t N,
                           int64_t width, int64_t free_count, int64_t page_size, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    const int64_t kMost = (int64_t(1) << 31) - 1;
    if (B < 0 || N < 0 || width < 0 || free_count < 0 || page_size < 0) return RLCS_ERR_SIZE;
    if (B >= (int64_t(1) << 24) || N >= (int64_t(1) << 24) || width > (int64_t(1) << 24) || free_count > kMost || page_size > (int64_t(1) << 24))
        return RLCS_ERR_SIZE;
    if (page_size == 0) return RLCS_ERR_ARG;
    if (pages_used == nullptr || (N > 0 && (sources == nullptr || copy_from == nullptr || copy_to == nullptr || (width > 0 && new_table == nullptr))) ||
        (N > 0 && B > 0 && (lens == nullptr || (width > 0 && block_table == nullptr))) || (free_count > 0 && free_pages == nullptr))
        return RLCS_ERR_NULL;
    const void* words[] = {block_table, lens, sources, free_pages, new_table, copy_from, copy_to, pages_used};
    for (const void* p : words)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    const size_t need = rlcs_fork_block_tables_workspace_bytes(B, N);
    if (need > 0) {
        if (workspace == nullptr || workspace_bytes < need) return RLCS_ERR_WORKSPACE;
        if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    if (B == 0 || N == 0) {                                       // nothing to continue, or nobody who does
        if (cudaMemsetAsync(pages_used, 0, sizeof(int32_t), s) != cudaSuccess) return RLCS_ERR_CUDA;
        if (N > 0 && (cudaMemsetAsync(copy_from, 0xff, (size_t)N * sizeof(int32_t), s) != cudaSuccess ||
                      cudaMemsetAsync(copy_to, 0xff, (size_t)N * sizeof(int32_t), s) != cudaSuccess ||
                      (width > 0 && cudaMemsetAsync(new_table, 0xff, (size_t)(N * width) * sizeof(int32_t), s) != cudaSuccess)))
            return RLCS_ERR_CUDA;
        return RLCS_OK;
    }
    const int64_t slots = fork_slots(B, N);
    int32_t* const keys = static_cast<int32_t*>(workspace);
    ForkParams P = {block_table, lens, sources, free_pages, new_table, copy_from, copy_to, pages_used, keys, nullptr, nullptr,
                    (int32_t)B, (int32_t)N, (int32_t)width, (int32_t)free_count, (int32_t)page_size, (int32_t)slots, 32, false};
    for (int64_t n = slots; n > 1; n /= 2) --P.shift;
    const int64_t cells = N * width, sms = rlcs_device::limits().sms;
    auto blocks_for = [&](int64_t items) { const int64_t n = (items + kThreads - 1) / kThreads; return (unsigned)(n < 1 ? 1 : n < 8 * sms ? n : 8 * sms); };
    const bool own_launches = need > 0 || (width >= 8 && (B > N ? B : N) * width > kMostCells);
    if (!own_launches) {
        static bool granted[64];
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return RLCS_ERR_CUDA;
        if (!granted[dev]) {
            const int most = (2 * (int)fork_slots(kFused, kFused) + kFused + kFused / 32) * (int)sizeof(int32_t);
            if (cudaFuncSetAttribute(fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most) != cudaSuccess) return RLCS_ERR_CUDA;
            granted[dev] = true;
        }
        // one block while every thread has an entry at most, else eight; tables of more than two entries a thread of those are written by
        // a launch of their own
        const int ways = B * width > kWide || cells > kWide ? kMostWays : 1;
        P.fill = cells <= 2 * kMostWays * kWide;
        if (!P.fill) fork_gather_kernel<<<blocks_for(cells), kThreads, 0, s>>>(P);
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)ways);
        cfg.blockDim = dim3(kWide);
        cfg.dynamicSmemBytes = (size_t)(2 * slots + N + (B + 31) / 32) * sizeof(int32_t);
        cfg.stream = s;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = ways;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaLaunchKernelEx(&cfg, fork_kernel, P) != cudaSuccess) return RLCS_ERR_CUDA;
    } else {
        // without a workspace the table of pages lies where the new table is written afterwards (2 * slots < 8 * N), and the numbers where the
        // copies are: each is read before it is overwritten
        if (need == 0) P.keys = new_table;
        P.owner = reinterpret_cast<uint32_t*>(P.keys + slots);
        P.number = need == 0 ? copy_to : P.keys + 2 * slots;
        if (cudaMemsetAsync(P.keys, 0xff, (size_t)slots * 2 * sizeof(int32_t), s) != cudaSuccess) return RLCS_ERR_CUDA;
        fork_enter_kernel<<<blocks_for(N), kThreads, 0, s>>>(P);
        if (cells > 0) fork_whole_kernel<<<blocks_for(cells), kThreads, 0, s>>>(P);
        fork_numbers_kernel<<<1, kWide, 0, s>>>(P);
        if (cells > 0) fork_gather_kernel<<<blocks_for(cells), kThreads, 0, s>>>(P);
        fork_give_kernel<<<blocks_for(N), kThreads, 0, s>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

int rlcs_copy_pages_bf16(uint16_t* k_cache, uint16_t* v_cache, int64_t pages, int64_t page_stride, int64_t token_stride, int64_t head_stride,
                         const int32_t* copy_from, const int32_t* copy_to, int64_t N, int64_t page_size, int64_t Hk, int64_t d,
                         void* cuda_stream) {
    if (N < 0 || pages < 0 || page_size < 0 || Hk < 0 || d < 0) return RLCS_ERR_SIZE;
    if (N > (1 << 30) || pages > (int64_t(1) << 31) - 1 || page_size > (1 << 24) || Hk > 4096 || d > (1 << 16) || d % 8 != 0) return RLCS_ERR_SIZE;
    if (page_stride < 0 || token_stride < 0 || head_stride < 0) return RLCS_ERR_SIZE;
    if (N == 0 || pages == 0 || page_size == 0 || Hk == 0 || d == 0) return RLCS_OK;
    if (k_cache == nullptr || copy_from == nullptr || copy_to == nullptr) return RLCS_ERR_NULL;
    if (!aligned_to(k_cache, 16) || !aligned_to(v_cache, 16) || !aligned_to(copy_from, 4) || !aligned_to(copy_to, 4)) return RLCS_ERR_ALIGN;
    if (page_stride % 8 || token_stride % 8 || head_stride % 8) return RLCS_ERR_ALIGN;
    // a page's tokens and heads, one after the other in either order
    const bool tight = (head_stride == d || Hk == 1) && (token_stride == Hk * d || page_size == 1);
    const bool heads_first = (token_stride == d || page_size == 1) && (head_stride == page_size * d || Hk == 1);
    const int64_t bytes = page_size * Hk * d * 2;
    CopyParams P = {};
    P.cache[0] = reinterpret_cast<char*>(k_cache);
    P.cache[1] = reinterpret_cast<char*>(v_cache);
    P.from = copy_from;
    P.to = copy_to;
    P.pages = pages;
    P.page_stride = page_stride * 2;
    P.token_stride = token_stride * 2;
    P.head_stride = head_stride * 2;
    P.N = (int32_t)N;
    P.caches = v_cache != nullptr ? 2 : 1;
    P.page = (int32_t)page_size;
    P.Hk = (int32_t)Hk;
    P.row = (int32_t)(d * 2);
    P.page_bytes = tight || heads_first ? bytes : 0;
    const int64_t sms = rlcs_device::limits().sms, items = N * P.caches * ((bytes + kPiece - 1) / kPiece);
    copy_kernel<<<(unsigned)(items < kCopyBlocks * sms ? items : kCopyBlocks * sms), kThreads, 0, static_cast<cudaStream_t>(cuda_stream)>>>(P);
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

size_t rlcs_free_pages_workspace_bytes(int64_t num_pages) {
    return num_pages <= 0 || num_pages > (int64_t(1) << 31) - 1 ? 0 : (size_t)((num_pages + 127) / 128) * 16;      // whole vectors of marks
}

int rlcs_free_pages(const int32_t* block_table, const int32_t* lens, const int32_t* prefix_table, const int32_t* prefix_lens,
                    int32_t* free_pages, int32_t* free_count, int64_t B, int64_t width, int64_t groups, int64_t prefix_width,
                    int64_t num_pages, int64_t page_size, void* workspace, size_t workspace_bytes, void* cuda_stream) {
    if (B < 0 || width < 0 || groups < 0 || prefix_width < 0 || num_pages < 0 || page_size < 0) return RLCS_ERR_SIZE;
    if (B >= (int64_t(1) << 24) || groups >= (int64_t(1) << 24) || width > (int64_t(1) << 24) || prefix_width > (int64_t(1) << 24) ||
        num_pages > (int64_t(1) << 31) - 64 || page_size > (int64_t(1) << 24))
        return RLCS_ERR_SIZE;
    if (page_size == 0) return RLCS_ERR_ARG;
    if (free_count == nullptr || (num_pages > 0 && free_pages == nullptr) || (B > 0 && (lens == nullptr || (width > 0 && block_table == nullptr))) ||
        (groups > 0 && (prefix_lens == nullptr || (prefix_width > 0 && prefix_table == nullptr))))
        return RLCS_ERR_NULL;
    const void* all[] = {block_table, lens, prefix_table, prefix_lens, free_pages, free_count};
    for (const void* p : all)
        if (!aligned_to(p, 4)) return RLCS_ERR_ALIGN;
    const size_t need = rlcs_free_pages_workspace_bytes(num_pages);
    if (need > 0) {
        if (workspace == nullptr || workspace_bytes < need) return RLCS_ERR_WORKSPACE;
        if (!aligned_to(workspace, 16)) return RLCS_ERR_ALIGN;
    }
    const cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    FreeParams P = {{block_table, prefix_table}, {lens, prefix_lens}, {(int32_t)B, (int32_t)groups}, {(int32_t)width, (int32_t)prefix_width},
                    static_cast<uint32_t*>(workspace), free_pages, free_count, (int32_t)num_pages, (int32_t)((num_pages + 31) / 32),
                    (int32_t)page_size};
    if (num_pages <= kAlonePages && B * width + groups * prefix_width <= kAloneEntries) {
        free_alone_kernel<<<1, kList, 0, s>>>(P);
    } else {
        const int64_t sms = rlcs_device::limits().sms, rows = B > groups ? B : groups, blocks = (rows + kThreads / 32 - 1) / (kThreads / 32);
        if (need > 0 && cudaMemsetAsync(workspace, 0, need, s) != cudaSuccess) return RLCS_ERR_CUDA;
        if (rows > 0) free_mark_kernel<<<(unsigned)(blocks < 8 * sms ? blocks : 8 * sms), kThreads, 0, s>>>(P);
        const int64_t parts = (P.words + kThreads - 1) / kThreads;
        free_list_kernel<<<(unsigned)(parts < 1 ? 1 : parts < sms ? parts : sms), kList, 0, s>>>(P);
    }
    return cudaGetLastError() == cudaSuccess ? RLCS_OK : RLCS_ERR_CUDA;
}

}  // extern "C"

// Internal declarations of the moves whose index map is data (include/ttc_moves.h), shared by the host part
// (ttc_moves.cpp) and the kernels (ttc_route.hip, ttc_pages.hip).
#pragma once

#include <cstdint>

#include "ttc_internal.h"
#include "ttc_moves.h"

struct ttc_route_s {
    int      dtype;
    int64_t  width;
    int      topk, experts;
    int64_t  first;
    int      align, id_bytes;
    float    alpha, beta;
};

struct ttc_pages_s {
    int      dtype, cache_dtype;
    int64_t  heads, dim, page, pages;
    int64_t  stride_head, stride_slot, stride_page;    // elements
    int64_t  span;                                     // elements from the first to the last of the cache, inclusive
    ttc::FastDiv page_div;
};

namespace ttc {

constexpr int kMoveThreads = 256;          // workgroup of the row moves
constexpr int kSortThreads = 1024;         // largest workgroup of the sort
constexpr int kSortBlocks = 8;             // ids a lane of the sort holds at most
constexpr int kSortOneBlocks = 2;          // and where one workgroup sorts alone: 2048 ids in 4.7 us, two kernels of two workgroups 3.4 + 3.2 and the
                                           // way from one to the other; 4000 ids the other way round (7.5 us alone)
constexpr int kSortOne = kSortOneBlocks * kSortThreads;
// Chunks up to which a lane takes no more ids, and counts (chunks times experts) up to which every workgroup adds up those of the others by
// itself; beyond them a kernel between does it.  us for 1,048,576 ids of 64 and 256 experts with 128, 256 and 512 chunks 25, 18, 20 and 34, 24, 34;
// 262,144 ids of 256 experts (256 chunks) 14 without the kernel between, 17 with it; 524,288 ids of 1024 experts 28 (128 chunks) and 23.
constexpr int64_t kSortChunks = 256, kSortCounts = 1 << 16;
inline bool sort_adds(int64_t chunks, int experts) { return chunks * experts <= kSortCounts; }

inline int elem_bytes(int dtype) { return dtype == TTC_F32 ? 4 : dtype == TTC_F8 ? 1 : 2; }

// How a sort of n assignments is cut: `blocks` ids per lane, `chunk` assignments per workgroup.
struct SortShape {
    int      threads, blocks;
    int64_t  chunk, chunks;
};
SortShape sort_shape(int64_t n, int experts);

// Kernel launchers; the callers have checked every argument.  They return TTC_OK or TTC_ERR_HIP; the row moves TTC_ERR_OVERFLOW, with nothing
// launched, where tokens times pieces of a row (64 vectors) exceed 2^31-1, which takes a tensor of 1 TB.
struct SortArgs {
    const void* ids;
    int64_t     ld_ids;
    int64_t     first;
    int32_t    *offsets, *counts, *position, *source;
    int32_t*    hist;                      // [chunks][experts], then [experts] totals (three-kernel form only)
    uint32_t    n, rows;                   // assignments, rows of a sorted tensor
    int32_t     topk, experts, align, id_bytes;
    FastDiv     topk_div;
};
int launch_sort(const SortArgs& a, const SortShape& s, void* stream);

struct RowArgs {
    const void    *x;                      // tokens' side, read (gather: x, grad: dy)
    const void    *rows;                   // sorted side, read (combine, grad)
    void          *y;                      // written (gather: rows, combine: y, grad: drows)
    const float   *weights;
    const int32_t *position, *offsets, *counts;
    float         *dweights;
    int64_t        ld_x, ld_rows, ld_y;
    float          alpha, beta;
    uint32_t       tokens, width, row_count;
    int32_t        topk, experts, align, dtype;
};
int launch_gather(const RowArgs& a, void* stream);
int launch_combine(const RowArgs& a, void* stream);
int launch_combine_grad(const RowArgs& a, void* stream);

struct MapArgs {
    const int32_t *first, *cached, *fresh, *free_list;
    int32_t       *table, *starts, *page_starts, *slots, *positions, *owner;
    int64_t        ld_table;
    int32_t        requests, free_count, tokens;
    uint32_t       pages;
    FastDiv        page;
};
int launch_map(const MapArgs& a, void* stream);

struct SlotArgs {
    const int32_t *slots;
    const void    *k, *v;                  // write: packed; read: cache
    void          *k_out, *v_out;          // write: cache; read: packed
    const float   *k_scale, *v_scale;
    int64_t        ld_k, ld_v;
    int64_t        stride_head, stride_slot, stride_page;
    uint32_t       tokens, slot_count, heads, dim;
    FastDiv        page;
    int32_t        dtype, cache_dtype;
};
int launch_write(const SlotArgs& a, void* stream);
int launch_read(const SlotArgs& a, void* stream);

}  // namespace ttc

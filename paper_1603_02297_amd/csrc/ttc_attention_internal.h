// Internal declarations of the heads and the attention (include/ttc_attention.h), shared by the host part (ttc_attention.cpp) and the
// kernels (ttc_heads.hip, ttc_attend*.hip).
#pragma once

#include <atomic>

#include "ttc_attention.h"
#include "ttc_moves_internal.h"

struct ttc_heads_s {
    int      dtype;
    int64_t  q_heads, kv_heads, dim, rotated;
    int      paired, norm;
    float    eps;
    uint64_t turns[TTC_HEADS_MAX_ROTATED / 2];         // angles in units of 2^-64 of a turn: products with a position wrap at whole turns
};

struct ttc_attend_s {
    int      dtype, cache_dtype;
    int64_t  q_heads, heads, dim, page, pages, vec, span;
    int64_t  stride_head, stride_slot, stride_page;    // as of the cache
    float    scale;
    int64_t  window;
    ttc::FastDiv page_div;
};

namespace ttc {

constexpr int kHeadsThreads = 256;
// Workgroups of a launch at most: four on each compute unit, each over many tokens, so that angles and weights are fetched once (512 to 16384: none faster).
constexpr int kHeadsGroups = 1024, kGradGroups = 512;
// Units of a lane where heads go element by element: 64 lanes have the 256 pairs of the longest head.
constexpr int kHeadsRounds = 4;

// Queries, keys and values of one call.  A head is cut into units of two vectors of V elements, the two sides of V rotations; `lanes` lanes
// of a wavefront have one head, 64 / lanes heads at a time are a group, and `splits` wavefronts share a token's groups.
struct HeadsArgs {
    const void    *q, *k, *v;              // null: not wanted (v: only on the way into a cache)
    void          *q_out, *k_out, *v_out;  // k_out, v_out: packed, or the cache
    const float   *q_weight, *k_weight, *k_scale, *v_scale;
    const int32_t *positions, *slots;
    int64_t        ld_q, ld_k, ld_v, ld_qo, ld_ko;
    int64_t        stride_head, stride_slot, stride_page;
    uint32_t       tokens, q_heads, kv_heads, dim, rotated, slot_count;
    FastDiv        page, split_div;
    int32_t        dtype, cache_dtype;     // cache_dtype -1: packed results
    int32_t        paired, norm;
    float          eps;
    int32_t        lanes_log, full;        // full: every unit of every lane has elements of its own in every group
    uint32_t       q_groups, k_groups, v_groups, per_wave;
    // the backward pass: q, k are the inputs, and beside them
    const void    *dq_out, *dk_out;
    int64_t        ld_dqo, ld_dko;
    float         *dq_weight, *dk_weight, *partial;
    uint64_t       turns[TTC_HEADS_MAX_ROTATED / 2];
};
int launch_heads(const HeadsArgs& a, void* stream);
int launch_heads_grad(const HeadsArgs& a, void* stream);

// How the work of a call is cut, on the host and for the workspace.
struct HeadsShape {
    int      vec;                          // elements of a vector: 16 bytes, 8 elements into records, or 1
    int      groups;                       // workgroups
    uint32_t splits;
};
HeadsShape cut_heads(HeadsArgs& a, int groups);          // sets what the cut says of a, too

// The exponentials' reference is the maximum less this many powers of 2, and they are multiplied in fp16 by up to 2^(7 + 8): it holds less than 2^16.  Its smallest step is then
// 2^-31 of the largest, and a million positions that it rounds away are less than the rounding of the result.  Relative to the maximum itself, positions below 2^-25 of it
// were in the sum but not in the products: 32,768 of them 0.1 % of all weights.
constexpr int attend_lift(int dtype) { return dtype == TTC_F16 ? 7 : 0; }

// Of a partial result: the exponent of 2 that its exponentials are relative to, and their sum.  In one number, their logarithm, a part's weight would be off by
// the rounding of that: 2^-24 of the whole score.
struct PartSum {
    float top, sum;
};

// Attention.  The rows of a request are its new tokens' query heads that share a head of the cache, token by token; a workgroup has `tile` rows of them
// and a part of the positions that they see.
struct AttendArgs {
    const void    *q, *k_cache, *v_cache;
    void          *out;
    float         *lse, *partial;                      // partial results: rows of dim elements
    PartSum       *partial_sums;
    int32_t       *parts;                              // [token][q_head][2]: the first of its partial results, and how many there are
    const float   *k_scale, *v_scale;
    const int32_t *starts, *cached, *table;
    int64_t        ld_q, ld_o, ld_table;
    int64_t        stride_head, stride_slot, stride_page;
    uint32_t       tokens, requests, q_heads, heads, group, dim, pages, splits, slots_of_tiles;
    uint32_t       partial_rows;
    uint32_t       join_step, join_back;               // part i > 0 of a row lies i * step - back behind its first
    uint32_t       window;                             // 0: none
    FastDiv        page, group_div;
    float          scale;                              // with log2(e)
    int32_t        dtype, cache_dtype;
};

constexpr int kTileMany = 128;             // rows of a workgroup at most: four wavefronts'; where there are few, 16 or 32, every wavefront with other positions
constexpr int kAttendMaxSplits = 32;
// What the kernels are compiled for: dims up to these; and narrow caches of one of them, few rows, in the form that keeps keys out of LDS.
constexpr int attend_dim(int dim) { return dim <= 32 ? 32 : dim <= 64 ? 64 : dim <= 96 ? 96 : dim <= 128 ? 128 : dim <= 192 ? 192 : 256; }
constexpr bool attend_own(int bytes, int cache_bytes, int dim, int tile) { return bytes == 2 && cache_bytes == 1 && dim == attend_dim(dim) && tile < 128; }
// Workgroups that share a compute unit, by registers and LDS.
constexpr int attend_resident(int bytes, bool own, bool records, int dim, int tile)
{
    return bytes == 4 || dim > 128 ? 1 : own && records && tile == 16 ? 3 : 2;
}
// Whether there are tiles of 32 rows: their results, the queries and a tile of the cache on its way have to fit the registers.
constexpr bool attend_half(int bytes, bool records, int dim) { return bytes == 4 ? dim <= 128 : dim <= 192 || records; }
constexpr uint32_t kAttendUnit = 128, kAttendMaxParts = 128;     // positions that are not shared among workgroups; results that a row may have to be joined from

struct AttendShape {
    uint32_t tile, slots, splits;          // rows of a tile, tiles at most, parts of the positions at most
    uint32_t shares;                       // workgroups, where rows are few
    int64_t  partial_rows;                 // 0: every row's positions are one workgroup's
};
AttendShape attend_shape(const ttc_attend_s* a, int64_t requests, int64_t tokens, int64_t longest);

int launch_attend(const AttendArgs& a, const AttendShape& s, void* stream);
// The kernel of a type, and what it needs; one file each.
struct AttendKernel {
    const void* fn;
    int         threads, lds;
    std::atomic<uint64_t>* raised;         // bit d: its LDS has been asked for on device d
};
AttendKernel attend_kernel_f32(int cache_dtype, int dim, int rows);
AttendKernel attend_kernel_bf16(int cache_dtype, int dim, int rows);
AttendKernel attend_kernel_f16(int cache_dtype, int dim, int rows);

}  // namespace ttc

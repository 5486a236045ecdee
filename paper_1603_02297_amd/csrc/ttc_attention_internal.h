// Internal declarations of the heads and the attention (include/ttc_attention.h), shared by the host part (ttc_attention.cpp) and the
// kernels (ttc_heads.hip, ttc_attend*.hip).
#pragma once

#include "ttc_attention.h"
#include "ttc_moves_internal.h"

struct ttc_heads_s {
    int      dtype;
    int64_t  q_heads, kv_heads, dim, rotated;
    int      paired, norm;
    float    eps;
    uint64_t turns[TTC_HEADS_MAX_ROTATED / 2];         // angles in units of 2^-64 of a turn: products with a position wrap at whole turns
};

namespace ttc {

constexpr int kHeadsThreads = 256;
// Workgroups of a launch at most: four on each compute unit, each over many tokens, so that angles and weights are fetched once.
constexpr int kHeadsGroups = 1024;

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
    int32_t        lanes_log;
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
HeadsShape cut_heads(HeadsArgs& a);          // sets what the cut says of a, too

}  // namespace ttc

// Checks of tensors that the entry points of the moves by data and of the attention share (ttc_moves.cpp, ttc_attention.cpp).  No HIP here.
#pragma once

#include <climits>

#include "ttc_moves_internal.h"

namespace ttc {

inline bool row_type(int dtype) { return dtype == TTC_F32 || dtype == TTC_BF16 || dtype == TTC_F16; }

// Bytes from the first to the last element of `cols` columns of `len` elements, ld apart; false if that is no size.
inline bool span_bytes(int64_t cols, int64_t ld, int64_t len, int bytes, uint64_t* out)
{
    if (cols == 0 || len == 0) { *out = 0; return true; }
    int64_t n;
    if (__builtin_mul_overflow(cols - 1, ld, &n) || __builtin_add_overflow(n, len, &n) || n > (INT64_MAX >> 4)) return false;
    *out = (uint64_t)n * (uint64_t)bytes;
    return true;
}

// One tensor of a call: where it is, how long, and whether the call writes it.
struct Operand {
    const void* p;
    uint64_t    bytes;
    int         align;
    bool        written;
};

// Every pointer aligned to its element, nothing written overlaps anything else.  A tensor without elements overlaps nothing, wherever it points.
template <int N> int check_operands(const Operand (&o)[N])
{
    for (int i = 0; i < N; ++i)
        if (o[i].p && (uintptr_t)o[i].p % (uintptr_t)o[i].align) return TTC_ERR_MISALIGNED;
    for (int i = 0; i < N; ++i)
        for (int j = 0; j < N; ++j) {
            if (i == j || !o[i].written || !o[i].p || !o[j].p || !o[i].bytes || !o[j].bytes) continue;
            const uintptr_t a = (uintptr_t)o[i].p, b = (uintptr_t)o[j].p;
            if (a < b + o[j].bytes && b < a + o[i].bytes) return TTC_ERR_ALIAS;
        }
    return TTC_OK;
}

// Keys and values are written by one call and may be parts of one tensor, so that their spans interleave: whether two tensors of one layout,
// `apart` bytes from each other, share a byte.  Levels go from the largest stride down, each stride no smaller than all that lies below it
// spans, so that only the two steps next to apart / stride bring them that close.
struct Level {
    int64_t stride, extent;                 // bytes, entries
};
inline bool share(int64_t apart, const Level* l, int levels, int64_t bytes)
{
    if (levels == 0) return -bytes < apart && apart < bytes;
    const int64_t step = apart / l->stride - (apart % l->stride < 0);
    for (int64_t t = step; t <= step + 1; ++t)
        if (-l->extent < t && t < l->extent && share(apart - t * l->stride, l + 1, levels - 1, bytes)) return true;
    return false;
}
inline bool share(const void* a, const void* b, uint64_t span, const Level* l, int levels, int64_t bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    if ((x < y ? y - x : x - y) >= span) return false;
    return share((int64_t)(y - x), l, levels, bytes);
}

}  // namespace ttc

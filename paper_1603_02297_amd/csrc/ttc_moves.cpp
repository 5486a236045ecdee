// Host part of the moves whose index map is data (include/ttc_moves.h): handles, sizes, and the checks of every call.
// No HIP here: what passes these checks goes to the launchers in ttc_route.hip and ttc_pages.hip.
#include <algorithm>
#include <climits>
#include <new>

#include "ttc_moves_internal.h"

namespace ttc {

SortShape sort_shape(int64_t n, int experts)
{
    SortShape s;
    s.threads = kSortThreads;
    s.blocks = 1;
    if (n <= kSortThreads) {                // as few wavefronts as hold the ids; a thread for every expert
        const int64_t need = std::max<int64_t>(std::max<int64_t>(n, experts), 1);
        s.threads = (int)((need + kWave - 1) / kWave * kWave);
    } else if (n <= kSortOne) {
        s.blocks = kSortOneBlocks;
    } else {                                // several workgroups, a lane with as few ids as kSortChunks allows
        while (s.blocks < kSortBlocks && (n + s.blocks * s.threads - 1) / (s.blocks * s.threads) > kSortChunks) s.blocks *= 2;
    }
    s.chunk = (int64_t)s.threads * s.blocks;
    s.chunks = std::max<int64_t>(1, (n + s.chunk - 1) / s.chunk);
    return s;
}

namespace {

// Bytes from the first to the last element of `cols` columns of `len` elements, ld apart; false if that is no size.
bool span_bytes(int64_t cols, int64_t ld, int64_t len, int bytes, uint64_t* out)
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
bool share(int64_t apart, const Level* l, int levels, int64_t bytes)
{
    if (levels == 0) return -bytes < apart && apart < bytes;
    const int64_t step = apart / l->stride - (apart % l->stride < 0);
    for (int64_t t = step; t <= step + 1; ++t)
        if (-l->extent < t && t < l->extent && share(apart - t * l->stride, l + 1, levels - 1, bytes)) return true;
    return false;
}
bool share(const void* a, const void* b, uint64_t span, const Level* l, int levels, int64_t bytes)
{
    const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
    if ((x < y ? y - x : x - y) >= span) return false;
    return share((int64_t)(y - x), l, levels, bytes);
}

int64_t route_rows(const ttc_route_s* r, int64_t tokens)
{
    if (tokens < 0) return -TTC_ERR_INVALID_VALUE;
    int64_t n, pad;
    if (__builtin_mul_overflow(tokens, (int64_t)r->topk, &n) || n > INT32_MAX) return -TTC_ERR_OVERFLOW;
    pad = std::min<int64_t>(n, r->experts) * (r->align - 1);
    return n + pad > INT32_MAX ? -TTC_ERR_OVERFLOW : n + pad;
}

int64_t route_workspace(const ttc_route_s* r, int64_t tokens)
{
    const SortShape s = sort_shape(tokens * r->topk, r->experts);
    if (s.chunks <= 1) return 0;
    return (s.chunks + (sort_adds(s.chunks, r->experts) ? 0 : 1)) * r->experts * (int64_t)sizeof(int32_t);
}

// What the three row moves share: the token count, and the offsets that padding needs.
int check_route(const ttc_route_s* r, int64_t tokens, int64_t* rows)
{
    if (!r) return TTC_ERR_NULL_POINTER;
    *rows = route_rows(r, tokens);
    return *rows < 0 ? (int)-*rows : TTC_OK;
}

RowArgs row_args(const ttc_route_s* r, int64_t tokens, int64_t rows)
{
    RowArgs a = {};
    a.tokens = (uint32_t)tokens;
    a.width = (uint32_t)r->width;
    a.row_count = (uint32_t)rows;
    a.topk = r->topk;
    a.experts = r->experts;
    a.align = r->align;
    a.dtype = r->dtype;
    a.alpha = r->alpha;
    a.beta = r->beta;
    return a;
}

bool row_type(int dtype) { return dtype == TTC_F32 || dtype == TTC_BF16 || dtype == TTC_F16; }

}  // namespace
}  // namespace ttc

using namespace ttc;

extern "C" {

ttc_route_t ttc_route_create(int dtype, int64_t width, int topk, int experts, int64_t first, int align, int id_bytes,
                             const float* alpha, const float* beta)
{
    int st = TTC_OK;
    if (!row_type(dtype)) st = TTC_ERR_UNSUPPORTED_DTYPE;
    else if (width < 1 || topk < 1 || topk > TTC_ROUTE_MAX_TOPK || experts < 1 || experts > TTC_ROUTE_MAX_EXPERTS || first < 0 || align < 1 ||
             align > TTC_ROUTE_MAX_ALIGN || (id_bytes != 4 && id_bytes != 8))
        st = TTC_ERR_INVALID_VALUE;
    else if (width > INT32_MAX / 2 || first > INT64_MAX - experts) st = TTC_ERR_OVERFLOW;
    ttc_route_s* r = st == TTC_OK ? new (std::nothrow) ttc_route_s : nullptr;
    if (st == TTC_OK && !r) st = TTC_ERR_ALLOC;
    if (r) *r = {dtype, width, topk, experts, first, align, id_bytes, alpha ? *alpha : 1.f, beta ? *beta : 0.f};
    set_last_status(st);
    return r;
}

int ttc_route_destroy(ttc_route_t route)
{
    delete route;
    return TTC_OK;
}

int64_t ttc_route_rows(ttc_route_t route, int64_t tokens)
{
    return route ? route_rows(route, tokens) : -TTC_ERR_NULL_POINTER;
}

int64_t ttc_route_workspace(ttc_route_t route, int64_t tokens)
{
    if (!route) return -TTC_ERR_NULL_POINTER;
    const int64_t rows = route_rows(route, tokens);
    return rows < 0 ? rows : route_workspace(route, tokens);
}

int ttc_route_sort(ttc_route_t route, int64_t tokens, const void* ids, int64_t ld_ids, int32_t* offsets, int32_t* counts,
                   int32_t* position, int32_t* source, void* workspace, void* stream)
{
    int64_t rows;
    int st = check_route(route, tokens, &rows);
    if (st != TTC_OK) return st;
    if (ld_ids < route->topk) return TTC_ERR_INVALID_VALUE;
    const int64_t n = tokens * route->topk, work = route_workspace(route, tokens);
    if (!offsets || !counts || (n && (!ids || !position)) || (work && !workspace)) return TTC_ERR_NULL_POINTER;
    uint64_t id_span;
    if (!span_bytes(tokens, ld_ids, route->topk, route->id_bytes, &id_span)) return TTC_ERR_OVERFLOW;
    st = check_operands({Operand{ids, id_span, route->id_bytes, false}, {offsets, 4 * (uint64_t)(route->experts + 1), 4, true},
                         {counts, 4 * (uint64_t)route->experts, 4, true}, {position, 4 * (uint64_t)n, 4, true},
                         {source, 4 * (uint64_t)rows, 4, true}, {work ? workspace : nullptr, (uint64_t)work, 4, true}});
    if (st != TTC_OK) return st;
    SortArgs a = {};
    a.ids = ids; a.ld_ids = ld_ids; a.first = route->first;
    a.offsets = offsets; a.counts = counts; a.position = position; a.source = source;
    a.hist = static_cast<int32_t*>(workspace);
    a.n = (uint32_t)n; a.rows = (uint32_t)rows;
    a.topk = route->topk; a.experts = route->experts; a.align = route->align; a.id_bytes = route->id_bytes;
    a.topk_div = make_fastdiv((uint32_t)route->topk);
    return launch_sort(a, sort_shape(n, route->experts), stream);
}

int ttc_route_gather(ttc_route_t route, int64_t tokens, const void* x, int64_t ldx, const float* weights, const int32_t* position,
                     const int32_t* offsets, const int32_t* counts, void* rows, int64_t ld_rows, void* stream)
{
    int64_t n_rows;
    int st = check_route(route, tokens, &n_rows);
    if (st != TTC_OK) return st;
    if (ldx < route->width || ld_rows < route->width) return TTC_ERR_INVALID_VALUE;
    if (tokens == 0) return TTC_OK;
    if (!x || !position || !rows || (route->align > 1 && (!offsets || !counts))) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(route->dtype);
    const uint64_t n = (uint64_t)tokens * route->topk;
    uint64_t bx, br;
    if (!span_bytes(tokens, ldx, route->width, eb, &bx) || !span_bytes(n_rows, ld_rows, route->width, eb, &br)) return TTC_ERR_OVERFLOW;
    st = check_operands({Operand{x, bx, eb, false}, {rows, br, eb, true}, {weights, 4 * n, 4, false}, {position, 4 * n, 4, false},
                         {offsets, 4 * (uint64_t)(route->experts + 1), 4, false}, {counts, 4 * (uint64_t)route->experts, 4, false}});
    if (st != TTC_OK) return st;
    RowArgs a = row_args(route, tokens, n_rows);
    a.x = x; a.ld_x = ldx; a.y = rows; a.ld_y = ld_rows;
    a.weights = weights; a.position = position; a.offsets = offsets; a.counts = counts;
    return launch_gather(a, stream);
}

int ttc_route_combine(ttc_route_t route, int64_t tokens, const void* rows, int64_t ld_rows, const float* weights, const int32_t* position,
                      void* y, int64_t ldy, void* stream)
{
    int64_t n_rows;
    int st = check_route(route, tokens, &n_rows);
    if (st != TTC_OK) return st;
    if (ldy < route->width || ld_rows < route->width) return TTC_ERR_INVALID_VALUE;
    if (tokens == 0) return TTC_OK;
    if (!rows || !position || !y) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(route->dtype);
    const uint64_t n = (uint64_t)tokens * route->topk;
    uint64_t by, br;
    if (!span_bytes(tokens, ldy, route->width, eb, &by) || !span_bytes(n_rows, ld_rows, route->width, eb, &br)) return TTC_ERR_OVERFLOW;
    st = check_operands({Operand{rows, br, eb, false}, {y, by, eb, true}, {weights, 4 * n, 4, false}, {position, 4 * n, 4, false}});
    if (st != TTC_OK) return st;
    RowArgs a = row_args(route, tokens, n_rows);
    a.rows = rows; a.ld_rows = ld_rows; a.y = y; a.ld_y = ldy;
    a.weights = weights; a.position = position;
    return launch_combine(a, stream);
}

int ttc_route_combine_grad(ttc_route_t route, int64_t tokens, const void* dy, int64_t ld_dy, const void* rows, int64_t ld_rows,
                           const float* weights, const int32_t* position, const int32_t* offsets, const int32_t* counts,
                           void* drows, int64_t ld_drows, float* dweights, void* stream)
{
    int64_t n_rows;
    int st = check_route(route, tokens, &n_rows);
    if (st != TTC_OK) return st;
    if (ld_dy < route->width || (drows && ld_drows < route->width) || (dweights && ld_rows < route->width)) return TTC_ERR_INVALID_VALUE;
    if (tokens == 0) return TTC_OK;
    if (!dy || !position || (!drows && !dweights) || (dweights && !rows) || (drows && route->align > 1 && (!offsets || !counts)))
        return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(route->dtype);
    const uint64_t n = (uint64_t)tokens * route->topk;
    uint64_t bx, br = 0, bd = 0;
    if (!span_bytes(tokens, ld_dy, route->width, eb, &bx) || (drows && !span_bytes(n_rows, ld_drows, route->width, eb, &bd)) ||
        (dweights && !span_bytes(n_rows, ld_rows, route->width, eb, &br)))
        return TTC_ERR_OVERFLOW;
    st = check_operands({Operand{dy, bx, eb, false}, {dweights ? rows : nullptr, br, eb, false}, {drows, bd, eb, true}, {dweights, 4 * n, 4, true},
                         {weights, 4 * n, 4, false}, {position, 4 * n, 4, false}, {offsets, 4 * (uint64_t)(route->experts + 1), 4, false},
                         {counts, 4 * (uint64_t)route->experts, 4, false}});
    if (st != TTC_OK) return st;
    RowArgs a = row_args(route, tokens, n_rows);
    a.x = dy; a.ld_x = ld_dy; a.rows = dweights ? rows : nullptr; a.ld_rows = ld_rows; a.y = drows; a.ld_y = ld_drows;
    a.weights = weights; a.position = position; a.offsets = offsets; a.counts = counts; a.dweights = dweights;
    return launch_combine_grad(a, stream);
}

ttc_pages_t ttc_pages_create(int dtype, int cache_dtype, int64_t heads, int64_t dim, int64_t page, int64_t pages, const int64_t* strides)
{
    int st = TTC_OK;
    ttc_pages_s p = {};
    p.dtype = dtype; p.cache_dtype = cache_dtype; p.heads = heads; p.dim = dim; p.page = page; p.pages = pages;
    int64_t slots, token;
    if (!row_type(dtype) || (cache_dtype != dtype && cache_dtype != TTC_F8)) st = TTC_ERR_UNSUPPORTED_DTYPE;
    else if (heads < 1 || dim < 1 || page < 1 || pages < 1) st = TTC_ERR_INVALID_VALUE;
    else if (__builtin_mul_overflow(page, pages, &slots) || slots > INT32_MAX || __builtin_mul_overflow(heads, dim, &token) || token > INT32_MAX / 2)
        st = TTC_ERR_OVERFLOW;
    if (st == TTC_OK) {
        p.stride_head = strides ? strides[0] : dim;
        p.stride_slot = strides ? strides[1] : heads * dim;
        p.stride_page = strides ? strides[2] : page * heads * dim;
        // from the smallest stride up, every index steps over all that lies below it: no two elements share a place
        struct { int64_t stride, extent; } index[3] = {{p.stride_head, heads}, {p.stride_slot, page}, {p.stride_page, pages}};
        std::sort(index, index + 3, [](const auto& a, const auto& b) { return a.stride < b.stride; });
        int64_t span = dim;
        for (const auto& i : index) {
            if (i.extent == 1) continue;
            if (i.stride < span) { st = TTC_ERR_INVALID_VALUE; break; }
            int64_t n;
            if (__builtin_mul_overflow(i.stride, i.extent - 1, &n) || __builtin_add_overflow(span, n, &span) || span > (INT64_MAX >> 4)) { st = TTC_ERR_OVERFLOW; break; }
        }
        p.span = span;
        // an index of one entry is never stepped along; whatever its stride says is not read
        if (heads == 1) p.stride_head = 0;
        if (page == 1) p.stride_slot = 0;
        if (pages == 1) p.stride_page = 0;
        p.page_div = make_fastdiv((uint32_t)page);
    }
    ttc_pages_s* out = st == TTC_OK ? new (std::nothrow) ttc_pages_s(p) : nullptr;
    if (st == TTC_OK && !out) st = TTC_ERR_ALLOC;
    set_last_status(st);
    return out;
}

int ttc_pages_destroy(ttc_pages_t pages)
{
    delete pages;
    return TTC_OK;
}

int ttc_pages_map(ttc_pages_t pages, int64_t requests, const int32_t* first, const int32_t* cached, const int32_t* fresh,
                  int32_t* table, int64_t ld_table, const int32_t* free_list, int64_t free_count, int64_t tokens, int32_t* starts,
                  int32_t* page_starts, int32_t* slots, int32_t* positions, int32_t* owner, void* stream)
{
    if (!pages) return TTC_ERR_NULL_POINTER;
    if (requests < 0 || ld_table < 0 || free_count < 0 || tokens < 0) return TTC_ERR_INVALID_VALUE;
    uint64_t table_bytes;
    if (requests > INT32_MAX / 2 || free_count > INT32_MAX || tokens > INT32_MAX || !span_bytes(requests, ld_table, ld_table, 4, &table_bytes))
        return TTC_ERR_OVERFLOW;
    if (!starts || !page_starts || (tokens && !slots) || (requests && (!cached || !fresh || (ld_table && !table))) || (free_count && !free_list))
        return TTC_ERR_NULL_POINTER;
    const uint64_t per_request = 4 * (uint64_t)requests, per_token = 4 * (uint64_t)tokens;
    const int st = check_operands({Operand{first, per_request, 4, false}, {cached, per_request, 4, false}, {fresh, per_request, 4, false},
                                   {table, table_bytes, 4, true}, {free_list, 4 * (uint64_t)free_count, 4, false}, {starts, per_request + 4, 4, true},
                                   {page_starts, per_request + 4, 4, true}, {slots, per_token, 4, true}, {positions, per_token, 4, true},
                                   {owner, per_token, 4, true}});
    if (st != TTC_OK) return st;
    MapArgs a = {};
    a.first = first; a.cached = cached; a.fresh = fresh; a.free_list = free_list;
    a.table = table; a.starts = starts; a.page_starts = page_starts; a.slots = slots; a.positions = positions; a.owner = owner;
    a.ld_table = ld_table;
    a.requests = (int32_t)requests; a.free_count = (int32_t)free_count; a.tokens = (int32_t)tokens;
    a.pages = (uint32_t)pages->pages;
    a.page = pages->page_div;
    return launch_map(a, stream);
}

// write: packed tensors in, cache out; read: the other way round
static int move_slots(ttc_pages_t pages, bool write, int64_t tokens, const int32_t* slots, const void* k, int64_t ldk, const void* v, int64_t ldv,
                      const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale, void* stream)
{
    if (!pages) return TTC_ERR_NULL_POINTER;
    const int64_t row = pages->heads * pages->dim;
    if (tokens < 0 || ldk < row || (v && ldv < row)) return TTC_ERR_INVALID_VALUE;
    if ((k_scale || v_scale) && pages->cache_dtype != TTC_F8) return TTC_ERR_INVALID_VALUE;
    if (tokens > INT32_MAX) return TTC_ERR_OVERFLOW;
    if (tokens == 0) return TTC_OK;
    if (!slots || !k || !k_cache || !v != !v_cache) return TTC_ERR_NULL_POINTER;
    const int eb = elem_bytes(pages->dtype), cb = elem_bytes(pages->cache_dtype);
    uint64_t bk, bv = 0;
    if (!span_bytes(tokens, ldk, row, eb, &bk) || (v && !span_bytes(tokens, ldv, row, eb, &bv))) return TTC_ERR_OVERFLOW;
    const uint64_t bc = (uint64_t)pages->span * cb, bs = 4 * (uint64_t)pages->heads;
    // keys and values may be parts of one tensor, on either side: they are checked against the other side, for being the same, and where they
    // are written for sharing elements
    if (v && (k == v || k_cache == v_cache)) return TTC_ERR_ALIAS;
    int st = check_operands({Operand{k, bk, eb, !write}, {k_cache, bc, cb, write}, {slots, 4 * (uint64_t)tokens, 4, false}, {k_scale, bs, 4, false}, {v_scale, bs, 4, false}});
    if (st == TTC_OK && v) {
        st = check_operands({Operand{v, bv, eb, !write}, {v_cache, bc, cb, write}, {slots, 4 * (uint64_t)tokens, 4, false}, {k_scale, bs, 4, false}, {v_scale, bs, 4, false}});
        if (st == TTC_OK) st = check_operands({Operand{k, bk, eb, !write}, {v_cache, bc, cb, write}});
        if (st == TTC_OK) st = check_operands({Operand{v, bv, eb, !write}, {k_cache, bc, cb, write}});
        Level level[3];
        int levels = 0;
        bool shared;
        if (write) {
            for (const Level& l : {Level{pages->stride_head, pages->heads}, {pages->stride_slot, pages->page}, {pages->stride_page, pages->pages}})
                if (l.extent > 1) level[levels++] = {l.stride * cb, l.extent};
            std::sort(level, level + levels, [](const Level& a, const Level& b) { return a.stride > b.stride; });
            shared = share(k_cache, v_cache, bc, level, levels, pages->dim * cb);
        } else {
            if (tokens > 1) level[levels++] = {ldk * eb, tokens};
            // rows of two different distances in one span: taken to meet
            shared = ldk == ldv || tokens == 1 ? share(k, v, bk, level, levels, row * eb) : (uintptr_t)k < (uintptr_t)v + bv && (uintptr_t)v < (uintptr_t)k + bk;
        }
        if (st == TTC_OK && shared) st = TTC_ERR_ALIAS;
    }
    if (st != TTC_OK) return st;
    SlotArgs a = {};
    a.slots = slots;
    a.k = write ? k : k_cache; a.v = write ? v : v_cache;
    a.k_out = const_cast<void*>(write ? k_cache : k); a.v_out = const_cast<void*>(write ? v_cache : v);
    a.k_scale = k_scale; a.v_scale = v_scale;
    a.ld_k = ldk; a.ld_v = ldv;
    a.stride_head = pages->stride_head; a.stride_slot = pages->stride_slot; a.stride_page = pages->stride_page;
    a.tokens = (uint32_t)tokens; a.slot_count = (uint32_t)(pages->page * pages->pages);
    a.heads = (uint32_t)pages->heads; a.dim = (uint32_t)pages->dim;
    a.page = pages->page_div;
    a.dtype = pages->dtype; a.cache_dtype = pages->cache_dtype;
    return write ? launch_write(a, stream) : launch_read(a, stream);
}

int ttc_pages_write(ttc_pages_t pages, int64_t tokens, const int32_t* slots, const void* k, int64_t ldk, const void* v, int64_t ldv,
                    void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, void* stream)
{
    return move_slots(pages, true, tokens, slots, k, ldk, v, ldv, k_cache, v_cache, k_scale, v_scale, stream);
}

int ttc_pages_read(ttc_pages_t pages, int64_t tokens, const int32_t* slots, const void* k_cache, const void* v_cache,
                   const float* k_scale, const float* v_scale, void* k, int64_t ldk, void* v, int64_t ldv, void* stream)
{
    return move_slots(pages, false, tokens, slots, k, ldk, v, ldv, k_cache, v_cache, k_scale, v_scale, stream);
}

}  // extern "C"

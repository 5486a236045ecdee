/*
 * ttc_moves.h -- C ABI of the moves whose index map is data.
 *
 * ttc.h moves a tensor by a permutation that is known when the plan is made.  Here the map is computed on the
 * GPU from what a model decided a moment ago, and then used by the moves that follow:
 *
 *   ttc_route_*   rows (tokens) sorted by the expert that a router chose for them, and back, weighted and added up;
 *                 with the gradients
 *   ttc_pages_*   block tables, packed offsets and slots from request lengths, and the moves of keys and values into
 *                 and out of a paged cache by those slots
 *
 * Conventions as in ttc.h: column-major (leftmost index has stride 1), DEVICE pointers owned by the caller, integer
 * status codes, nothing throws or aborts across this boundary.  A handle is made once for what stays (types, widths,
 * scalars), touches no device, may be used from several streams at a time, and is freed by its destroy function.
 * Every other call is asynchronous: it enqueues a few kernels (mostly one) on `stream` (hipStream_t as void*, NULL is the
 * default stream), allocates nothing, never synchronises and can be captured into a graph.
 *
 * Maps are checked on the GPU before they are followed: an entry that points outside its tensor counts as "nowhere",
 * whatever it is, so no map makes a kernel leave its tensors.  Leading dimensions (ld*) count elements between
 * neighbouring columns, as lda in ttc.h; every column starts wherever its ld puts it (element alignment suffices).
 * Sums run in 32 bits in a fixed order and are rounded once: the same inputs give the same bits.
 */
#ifndef TTC_MOVES_H_
#define TTC_MOVES_H_

#include "ttc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types beside TTC_F32 that these moves take (ttc_plan_create takes none of them).  TTC_F8 is the 8-bit format
 * with four exponent and three mantissa bits, largest value 448, no infinities; it is a type of the cache only.
 * So is TTC_Q4: a vector of `dim` elements (a multiple of 8, at most 512) is a record of 4 + dim/2 bytes, a step and a minimum in bf16 (in this order) and the
 * codes, element 2i in the low and 2i+1 in the high half of byte i; element = minimum + code * step.  Written are the largest
 * minimum of bf16 that is no larger than the vector's, the smallest step of bf16 that reaches its maximum with code 15, and the nearest codes (to the even one in the middle), all three
 * from differences and quotients in 32 bits: no element is off by more than half a step and that rounding.  A vector with a NaN, an infinity, an element beyond the range of bf16, or
 * elements further apart than 32 bits can say becomes all NaN. */
enum { TTC_BF16 = 8, TTC_F16 = 9, TTC_F8 = 10, TTC_Q4 = 11 };

/* Limits of a handle (TTC_ERR_INVALID_VALUE beyond them). */
enum { TTC_ROUTE_MAX_EXPERTS = 1024, TTC_ROUTE_MAX_TOPK = 64, TTC_ROUTE_MAX_ALIGN = 65536 };

/* ---- rows sorted by expert, and back ------------------------------------------------------------------------- */

typedef struct ttc_route_s* ttc_route_t;

/*
 * A handle for one layer of experts.
 *   dtype       TTC_F32, TTC_BF16 or TTC_F16: the type of every row.
 *   width       elements of a row.
 *   topk        experts chosen per token (1 .. TTC_ROUTE_MAX_TOPK).
 *   experts     experts that live here, numbered first .. first+experts-1 in the router's ids (1 .. TTC_ROUTE_MAX_EXPERTS).
 *   align       every expert's segment of the sorted rows starts at a multiple of `align` rows and is padded to one
 *               (the rows of a matrix tile; 1 = no padding).
 *   id_bytes    4 or 8: the ids are int32 or int64.
 *   alpha, beta HOST pointers to one float each; NULL means alpha = 1, beta = 0.  Copied.
 * Returns NULL on error; ttc_last_status() says why.
 */
ttc_route_t ttc_route_create(int dtype, int64_t width, int topk, int experts, int64_t first, int align, int id_bytes,
                             const float* alpha, const float* beta);
int ttc_route_destroy(ttc_route_t route);

/* Rows of a sorted tensor that suffice whatever the router chose: tokens*topk + min(tokens*topk, experts)*(align-1).
 * Every sorted tensor has that many.  A negative status on error. */
int64_t ttc_route_rows(ttc_route_t route, int64_t tokens);
/* Bytes of workspace for ttc_route_sort (0 where it needs none), or a negative status. */
int64_t ttc_route_workspace(ttc_route_t route, int64_t tokens);

/*
 * The sort.  Assignment a = topk*t + k is token t's k-th choice.
 *   ids        [topk, tokens], ld_ids >= topk: the chosen experts.  An id outside first .. first+experts-1 is nowhere:
 *              an expert of another rank, or a token that is padding.
 *   offsets    [experts+1] int32, out: the first row of every expert's segment; offsets[experts] is where the last ends.
 *   counts     [experts] int32, out: rows of the segment that hold a token; the others are padding.
 *   position   [topk, tokens] int32, out: the row of every assignment, -1 for nowhere.  Within a segment rows keep the
 *              order of the assignments (the sort is stable).
 *   source     [ttc_route_rows] int32, out, may be NULL: the assignment of every row, -1 for padding and past the end.
 *   workspace  ttc_route_workspace bytes, aligned to 4; contents are of no interest before or after.
 */
int ttc_route_sort(ttc_route_t route, int64_t tokens, const void* ids, int64_t ld_ids, int32_t* offsets, int32_t* counts,
                   int32_t* position, int32_t* source, void* workspace, void* stream);

/*
 * Tokens to their rows:  rows[:, position[k,t]] <- weights[k,t] * x[:, t].
 *   x         [width, tokens], ldx >= width.
 *   weights   [topk, tokens] float, or NULL: copied bit for bit.
 *   offsets, counts as ttc_route_sort left them; padding rows become 0.  Needed if align > 1, else they may be NULL.
 *   rows      [width, ttc_route_rows], ld_rows >= width; rows past offsets[experts] are not touched.
 */
int ttc_route_gather(ttc_route_t route, int64_t tokens, const void* x, int64_t ldx, const float* weights, const int32_t* position,
                     const int32_t* offsets, const int32_t* counts, void* rows, int64_t ld_rows, void* stream);

/*
 * Rows back to their tokens:  y[:, t] <- alpha * sum_k weights[k,t] * rows[:, position[k,t]]  +  beta * y[:, t].
 * Choices that are nowhere add nothing (a token with no other becomes beta * y); weights NULL: all 1.  The sum runs
 * over k in order; with beta == 0 y is never read.  By a handle with alpha = 1 and beta = 0, whatever those of the layer's own
 * handle are, this is the gradient of ttc_route_gather: with weights NULL, or of the weighted one with its weights.
 */
int ttc_route_combine(ttc_route_t route, int64_t tokens, const void* rows, int64_t ld_rows, const float* weights, const int32_t* position,
                      void* y, int64_t ldy, void* stream);

/*
 * The gradients of ttc_route_combine:
 *   drows[:, position[k,t]] <- (alpha * weights[k,t]) * dy[:, t]       (padding rows 0, rows past the end not touched)
 *   dweights[k,t]           <- alpha * sum_i dy[i, t] * rows[i, position[k,t]]        (0 where the choice is nowhere)
 * dweights NULL: no gradient of the weights; rows is not read then and may be NULL.  drows NULL: that of the weights only
 * (with x as dy and the gradient of ttc_route_gather's rows as rows, by a handle with alpha = 1, its weights' gradient).  weights
 * NULL: all 1.
 */
int ttc_route_combine_grad(ttc_route_t route, int64_t tokens, const void* dy, int64_t ld_dy, const void* rows, int64_t ld_rows,
                           const float* weights, const int32_t* position, const int32_t* offsets, const int32_t* counts,
                           void* drows, int64_t ld_drows, float* dweights, void* stream);

/* ---- pages of a cache ----------------------------------------------------------------------------------------- */

typedef struct ttc_pages_s* ttc_pages_t;

/*
 * A handle for a cache of `pages` pages with `page` slots each; a slot holds `heads` vectors of `dim` elements (keys or
 * values of one token).  Slot s is place s % page of page s / page.
 *   dtype        type of keys and values outside the cache: TTC_F32, TTC_BF16 or TTC_F16.
 *   cache_dtype  the same, or TTC_F8, or TTC_Q4.
 *   strides      HOST array of three: elements (TTC_Q4: bytes) between neighbouring heads, slots and pages in the cache (elements of a
 *                vector are neighbours).  NULL: [dim, heads, page, pages] dense, with records in the place of vectors for TTC_Q4.  No two elements may share a place.
 * Returns NULL on error; ttc_last_status() says why.
 */
ttc_pages_t ttc_pages_create(int dtype, int cache_dtype, int64_t heads, int64_t dim, int64_t page, int64_t pages, const int64_t* strides);
int ttc_pages_destroy(ttc_pages_t pages);

/*
 * Block tables and slots from request lengths.  Request r holds cached[r] tokens and gets fresh[r] more; the call gives it
 * the pages that these need and lists the positions first[r] .. cached[r]+fresh[r]-1 of all requests, packed.
 *   first      [requests] int32 or NULL: first position to list; NULL means cached (the new tokens only), larger
 *              values count as cached[r].
 *   cached, fresh [requests] int32; negative counts as 0, and cached[r]+fresh[r] is cut at 2^31-1.
 *   table      [ld_table, requests] int32, in and out: entry b of request r is the page of its positions b*page ...
 *              Entries below ceil(cached/page) are read, those from there to ceil((cached+fresh)/page) are written, each with
 *              the first token of its page (so not those of tokens past the end of `slots`).
 *   free_list  [free_count] int32: pages to take, in order; request 0's come first.
 *   tokens     length of slots, positions and owner (a step's buffers; >= 0).
 *   starts     [requests+1] int32, out: where every request's listed positions start; starts[requests] is their number,
 *              also where it exceeds `tokens` (cut at 2^31-1).
 *   page_starts [requests+1] int32, out: the same for the pages taken; page_starts[requests] > free_count says that there
 *              were too few: entries without a page become -1.  Pages are counted for every block that a request needs, those past
 *              the table's width, which nothing will point to, among them.
 *   slots      [tokens] int32, out: the slot of every listed position; -1 past the end, where the table has no entry
 *              (position >= ld_table*page), and where the entry is no page (0 .. pages-1).
 *   positions, owner [tokens] int32, out, each may be NULL: position within its request, and the request; -1 past the end.
 */
int ttc_pages_map(ttc_pages_t pages, int64_t requests, const int32_t* first, const int32_t* cached, const int32_t* fresh,
                  int32_t* table, int64_t ld_table, const int32_t* free_list, int64_t free_count, int64_t tokens, int32_t* starts,
                  int32_t* page_starts, int32_t* slots, int32_t* positions, int32_t* owner, void* stream);

/*
 * Keys and values into the cache:  k_cache[:, h, slots[i]] <- k[:, h, i], and v likewise.
 *   k, v       [dim, heads, tokens], ldk, ldv >= heads*dim elements between tokens (parts of one fused projection).
 *              v and v_cache NULL: one tensor only.
 *   k_scale, v_scale [heads] float or NULL (1): with TTC_F8 the cache holds k / k_scale[h], cut at +-448 and rounded to
 *              nearest even; a NaN stays one.  Refused (TTC_ERR_INVALID_VALUE) with another cache type.
 * A token whose slot is nowhere (negative, or past the cache) is left out.  Two tokens must not have one slot.
 * k_cache and v_cache may be parts of one tensor, their vectors between each other's; sharing an element is TTC_ERR_ALIAS.
 */
int ttc_pages_write(ttc_pages_t pages, int64_t tokens, const int32_t* slots, const void* k, int64_t ldk, const void* v, int64_t ldv,
                    void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, void* stream);

/*
 * And out of it:  k[:, h, i] <- k_cache[:, h, slots[i]] (* k_scale[h]), 0 where the slot is nowhere.
 * k and v may be parts of one tensor, with ldk == ldv where one lies within the other's rows; sharing an element is TTC_ERR_ALIAS.
 */
int ttc_pages_read(ttc_pages_t pages, int64_t tokens, const int32_t* slots, const void* k_cache, const void* v_cache,
                   const float* k_scale, const float* v_scale, void* k, int64_t ldk, void* v, int64_t ldv, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TTC_MOVES_H_ */

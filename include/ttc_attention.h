/*
 * ttc_attention.h -- C ABI of the way of a layer's queries, keys and values around the paged cache of ttc_moves.h.
 *
 *   ttc_heads_*        norms of queries and keys for each head, with the rotation by position in the same pass; with the gradients
 *   ttc_pages_append   the same on the way of new tokens into the cache
 *   ttc_attend_*       attention of new tokens over the pages of their requests
 *
 * Conventions as in ttc_moves.h: column-major, DEVICE pointers owned by the caller, integer status codes, nothing throws or aborts
 * across this boundary; handles are made once, touch no device, may be used from several streams at a time; every other
 * call enqueues a few kernels on `stream`, allocates nothing, never synchronises and can be captured into a graph.  A call works on the
 * current device, which its tensors and its stream belong to.  A workspace belongs to the calls of one stream (or of one graph) at a time.
 * Entries of slots, tables and lengths are checked on the GPU before they are followed.  Sums run in 32 bits in a fixed order: the same
 * inputs give the same bits.
 */
#ifndef TTC_ATTENTION_H_
#define TTC_ATTENTION_H_

#include "ttc_moves.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Limits of a handle (TTC_ERR_INVALID_VALUE beyond them). */
enum { TTC_HEADS_MAX_DIM = 512, TTC_HEADS_MAX_ROTATED = 256, TTC_ATTEND_MAX_DIM = 256 };

/* ---- norms of the heads, and their rotation ------------------------------------------------------------------ */

typedef struct ttc_heads_s* ttc_heads_t;

/*
 * A handle for the heads of one layer.  For a vector x of `dim` elements at position p, with weights w:
 *     u = x / sqrt(mean(x^2) + eps) * w            (norm != 0; else u = x)
 *     y = u with its first `rotated` elements turned, pair i by the angle p * angles[i]:
 *         (y_a, y_b) = (u_a cos - u_b sin, u_b cos + u_a sin)
 * where pair i is elements (i, i + rotated/2), or its neighbours (2i, 2i+1) if paired != 0.
 *   dtype      TTC_F32, TTC_BF16 or TTC_F16: the type of every tensor but weights.  Everything between is 32 bits, rounded once.
 *   q_heads, kv_heads  heads of queries and of keys.
 *   dim        1 .. TTC_HEADS_MAX_DIM.
 *   rotated    even, 0 .. min(dim, TTC_HEADS_MAX_ROTATED).
 *   angles     HOST array of rotated/2 doubles (radians for each position, finite), copied; NULL if rotated is 0.  Products with the position
 *              are exact to 2^-31 of a turn, however far the position.
 *   eps        >= 0, finite; not read without norm.
 * Returns NULL on error; ttc_last_status() says why.
 */
ttc_heads_t ttc_heads_create(int dtype, int64_t q_heads, int64_t kv_heads, int64_t dim, int64_t rotated, int paired, const double* angles,
                             int norm, float eps);
int ttc_heads_destroy(ttc_heads_t heads);

/*
 * Queries and keys of packed tokens:  q_out <- y(q), k_out <- y(k).
 *   positions  [tokens] int32; a token with a negative one is padding, whose results are left as they were.  NULL only if nothing is rotated.
 *   q, k       [dim, heads, tokens], ldq, ldk >= heads*dim elements between tokens (parts of one fused projection).  k and k_out NULL: queries
 *              only; q and q_out NULL: keys only.
 *   q_weight, k_weight  [dim] float, or NULL (1).  Refused (TTC_ERR_INVALID_VALUE) without norm.
 *   q_out, k_out  as q and k; each may be the tensor that it is made of, in its place (same address, same distance).
 */
int ttc_heads_rotate(ttc_heads_t heads, int64_t tokens, const int32_t* positions, const void* q, int64_t ldq, const void* k, int64_t ldk,
                     const float* q_weight, const float* k_weight, void* q_out, int64_t ld_qo, void* k_out, int64_t ld_ko, void* stream);

/* Bytes of workspace for ttc_heads_rotate_grad (0 where it needs none), or a negative status. */
int64_t ttc_heads_workspace(ttc_heads_t heads, int64_t tokens);

/*
 * The gradients of ttc_heads_rotate, from those of its results (dq_out, dk_out) and its inputs:
 *     du = dy turned back,  dw = sum over tokens and heads of x/s * du,  g = du * w,  dx = g/s - x * mean(g * x) / s^3,   s = sqrt(mean(x^2) + eps)
 *   q, k       not read, and may be NULL, without norm.
 *   dq, dk     as dq_out and dk_out; each may be its tensor of gradients, in its place.  Padding is left as it was and adds nothing.
 *   dq_weight, dk_weight  [dim] float, each may be NULL; refused without norm.  0 where no token is left.
 *   workspace  ttc_heads_workspace bytes, aligned to 4; not used, and may be NULL, where neither is wanted.
 */
int ttc_heads_rotate_grad(ttc_heads_t heads, int64_t tokens, const int32_t* positions, const void* dq_out, int64_t ld_dqo, const void* dk_out,
                          int64_t ld_dko, const void* q, int64_t ldq, const void* k, int64_t ldk, const float* q_weight, const float* k_weight,
                          void* dq, int64_t ld_dq, void* dk, int64_t ld_dk, float* dq_weight, float* dk_weight, void* workspace, void* stream);

/* ---- new tokens into the cache -------------------------------------------------------------------------------- */

/*
 * q_out <- y(q),  k_cache[:, h, slots[i]] <- y(k)[:, h, i],  v_cache[:, h, slots[i]] <- v[:, h, i]
 * in one pass, for a cache and heads of one type, one dim and one number of kv_heads.  What goes into 8 or 4 bits is y itself, rounded once; scales as for
 * ttc_pages_write.  A token with a negative position is left out; one whose slot is nowhere gets its queries only.  q and q_out may both be NULL; q_out may be q
 * in its place.  Two tokens must not have one slot.  A cache in 4 bits takes vectors whose rotated part is a multiple of 16 (TTC_ERR_INVALID_VALUE: rotate first, then
 * ttc_pages_write).
 */
int ttc_pages_append(ttc_pages_t pages, ttc_heads_t heads, int64_t tokens, const int32_t* slots, const int32_t* positions, const void* q, int64_t ldq,
                     const void* k, int64_t ldk, const void* v, int64_t ldv, const float* q_weight, const float* k_weight, void* q_out, int64_t ld_qo,
                     void* k_cache, void* v_cache, const float* k_scale, const float* v_scale, void* stream);

/* ---- attention over the cache ---------------------------------------------------------------------------------- */

typedef struct ttc_attend_s* ttc_attend_t;

/*
 * A handle for attention over caches like that of `pages` (what it says is copied), dim 1 .. TTC_ATTEND_MAX_DIM.
 *   q_heads    a multiple of the cache's heads: query head h reads head h / (q_heads / heads).
 *   scale      finite, what the products of queries and keys are multiplied with.
 *   window     0: every position up to the query's own; else the last `window` of them, its own among them.
 * Returns NULL on error; ttc_last_status() says why.
 */
ttc_attend_t ttc_attend_create(ttc_pages_t pages, int64_t q_heads, double scale, int64_t window);
int ttc_attend_destroy(ttc_attend_t attend);

/* Bytes of workspace for ttc_attend_pages with tables of ld_table entries (0 where it needs none), or a negative status: -TTC_ERR_OVERFLOW, as the call itself then, where
 * requests or tokens*q_heads are 2^29 or more, tokens*q_heads and requests * the cache's heads together 2^31 or more, or a table of a request has more than 2^40 entries. */
int64_t ttc_attend_workspace(ttc_attend_t attend, int64_t requests, int64_t tokens, int64_t ld_table);

/*
 * out[:, h, i] <- sum_j softmax_j(scale * <q[:, h, i], k_j>) v_j  over the positions j that token i sees.
 *   q          [dim, q_heads, tokens], ldq >= q_heads*dim: the packed new tokens.
 *   starts     [requests+1] int32 as ttc_pages_map left it for them: request r has the tokens starts[r] .. starts[r+1]-1.  Tokens before starts[0] and from
 *              starts[requests] on are left as they were.
 *   cached     [requests] int32: positions that request r held before them (negative counts as 0); its token i stands at cached[r] + i - starts[r], and its keys and
 *              values, those of the new tokens among them, are in the cache already.
 *   table      [ld_table, requests] int32 as for ttc_pages_map.  Positions past the table (>= ld_table*page) and those whose entry is no page are not there.
 *   k_cache, v_cache, k_scale, v_scale   as for ttc_pages_read.
 *   out        as q; must not overlap it.
 *   lse        [q_heads, tokens] float or NULL: the logarithm of the sum of exponentials, -inf where a token sees nothing.
 *   workspace  ttc_attend_workspace bytes, aligned to 16.
 * A token that sees nothing, or scores of -inf only, gets 0.  What a position that is not seen holds (NaN, infinities) has no effect.  Scores, exponentials and their sums are
 * 32 bits; with 16-bit queries the exponentials (over a cache in 4 bits: times the values' steps) are rounded to that type for their products with the values, once; in fp16
 * those below 2^-21 of a row's largest to multiples of 2^-31 of it at most.  Values are added up before they are divided by the sum of the exponentials: those above 2^116 / (positions seen)
 * may become infinite on the way.
 */
int ttc_attend_pages(ttc_attend_t attend, int64_t requests, int64_t tokens, const void* q, int64_t ldq, const int32_t* starts, const int32_t* cached,
                     const int32_t* table, int64_t ld_table, const void* k_cache, const void* v_cache, const float* k_scale, const float* v_scale,
                     void* out, int64_t ldo, float* lse, void* workspace, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* TTC_ATTENTION_H_ */

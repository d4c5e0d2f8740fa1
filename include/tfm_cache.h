/*
 * tfm_cache.h — C ABI of contexts kept in 8 bits on MI355X (gfx950): keys and values appended to a
 * paged cache of e4m3 codes with a power of two for each block of rows and head, attention of query
 * rows over it, and the forward-only layer calls of tfm_layer.h with such a cache in place of the
 * bfloat16 one.
 *
 * Conventions: the caller owns every buffer and the library allocates nothing; calls are
 * asynchronous on `stream` (a hipStream_t, NULL = the null stream) of the current device and may
 * be captured into a graph; pointers are device pointers, aligned to their elements (pools and
 * workspaces to 16 bytes); on a negative return (the codes of tfm_layer.h) nothing was launched and
 * tfm_last_error() describes the error.  Sums run in a fixed order: the same call gives the same
 * bits again.  Calls that run at the same time need workspaces of their own, and only calls that
 * read a pool may run at the same time on it.
 */
#ifndef TFM_CACHE_H
#define TFM_CACHE_H

#include "tfm_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- the pool ---------------------------------------------------------------------------------
 * n_pages pages of `page` rows (16, 32, 64, 128 or 256) of `heads` key/value heads of d channels
 * (16, 32, 64 or 128).  A pool holds, one after another,
 *
 *   keys    [n_pages][heads][page][d]   e4m3 codes (OCP: bias 7, largest 448, 0x7f and 0xff NaN)
 *   values  [n_pages][heads][d][page]   e4m3 codes
 *   powers  [n_pages][heads][2]         bytes e of the keys and of the values
 *
 * and a code c of a block (page, head) stands for c 2^(e - 127), 79 <= e <= 175 (a byte outside is
 * read as the nearest of these).
 *
 * Sequence b's row r is row r % page of the page pages[b][r / page] (pages: int32 [B][max_pages],
 * or null: page b max_pages + r / page).  A page index outside [0, n_pages) is absent: its rows are
 * neither written nor seen.  Pages may be shared by sequences that only read them; a page that an
 * append writes must belong to one sequence and stand in its table once.
 * Limits: 1 <= heads <= 4096, 1 <= n_pages <= 2^31 - 1, at most 2^46 bytes. */
typedef struct {
  int32_t heads, d, page, n_pages;
} tfm_cache8;

/* Bytes of the pool (0 on invalid arguments). */
size_t tfm_cache8_bytes(const tfm_cache8* c);

/* ---- appending ---------------------------------------------------------------------------------
 * Rows i < n_new[b] (null: L) of k and v become rows lens[b] + i (null: 0) of sequence b; lens is
 * not changed.  n_new is cut to [0, L] and lens to [0, max_pages page]; rows past the sequence's
 * last page are left out.  Row (b, i, h) of k is the d elements from element b stride_k[0] +
 * i stride_k[1] + h stride_k[2] on (v alike).
 *
 * A block's power is the least e in [79, 175] with |x| <= 448 2^(e - 127) for its rows, and codes are
 * x 2^(127 - e) rounded to the nearest, halves to even.  Where a block has rows already (those before
 * lens[b]) its power does not fall; where it grows, the codes of these rows are rounded again to the
 * new power.  NaN, infinities and values above 448 2^48 do not count for the power and become NaN
 * codes.  Everything else of the pool is left as it was.
 * Limits: B, L, max_pages >= 0, B max_pages <= 2^31 - 1, max_pages page <= 2^30; strides in
 * [0, 2^40], the last row at most 2^48 elements from the first.  k, v and the pool must not share
 * memory. */
typedef struct {
  int32_t B, L, max_pages;
  int32_t dtype;                    /* tfm_dtype of k and v */
  int64_t stride_k[3], stride_v[3]; /* elements between sequences, rows, heads */
} tfm_cache8_rows;

int tfm_cache8_append(const tfm_cache8* c, const tfm_cache8_rows* r, const void* k, const void* v,
                      const int32_t* pages, const int32_t* lens, const int32_t* n_new, void* pool,
                      size_t pool_bytes, void* stream);

/* ---- attention ----------------------------------------------------------------------------------
 * Query row i < n_rows[b] (null: L) of head h attends to the rows j of sequence b's cache with
 * j < lens[b] and, if causal, j < lens[b] - n_rows[b] + i + 1 (the query rows are the last rows of
 * their sequence), at key/value head h / (heads / cache heads):
 *
 *   out_i = sum_j p_j V_j,  p = softmax over those j of scale q_i K_j,  lse_i = log of its sum
 *
 * (natural logarithm; lse nullable, float32 [B][L][heads]).  A row that attends to nothing gets
 * out = 0 and lse = -inf; rows i >= n_rows[b] of out and lse are left as they were.  NaN codes show
 * in the rows that attend to them and in no others.  lens is cut to [0, max_len] (0: no such cut) and
 * to [0, max_pages page], n_rows to [0, L].  max_len is a promise that no sequence is longer: it
 * chooses how the rows of a cache are split over workgroups.
 *
 * Scores, statistics and sums are held in float32, as is scale log2(e).  Codes are exact as bfloat16
 * (keys) and half (values of blocks less than 2^22 below the row's largest); a float32 query goes in
 * three bfloat16 parts whose sum it is (subnormal ones may be lost).  Weights are rounded to half (by
 * 2^-11 of each, or 2^-33 of the row's largest where that is more), with a float32 output to two halves
 * (2^-23).
 *
 * Rows of q and out (dtype both) lie by their strides as above; out's rows must not overlap.  out may
 * be q itself (with equal strides: in place); it shares no element with q otherwise, and none with
 * the pool, lse and the workspace.  A query row with elements of 2^112 and more, infinite or NaN, or
 * with a score of 2^127 and more has undefined outputs, others not.
 * Limits: B, L >= 0, heads a multiple of the cache's with at most 2^16 of them, L heads <= 2^26,
 * B L heads <= 2^31 - 1; max_pages, strides as above; scale in [-2^64, 2^64]. */
typedef struct {
  int32_t B, L, max_pages, max_len;
  int32_t heads, causal;
  int32_t dtype;                      /* tfm_dtype of q and out */
  float scale;
  int64_t stride_q[3], stride_out[3]; /* elements between sequences, rows, heads */
} tfm_cache8_query;

/* Bytes of scratch of tfm_cache8_attend (may be 0; 0 on invalid arguments too). */
size_t tfm_cache8_attend_workspace_bytes(const tfm_cache8* c, const tfm_cache8_query* a);

int tfm_cache8_attend(const tfm_cache8* c, const tfm_cache8_query* a, const void* q,
                      const int32_t* pages, const int32_t* lens, const int32_t* n_rows,
                      const void* pool, size_t pool_bytes, void* out, float* lse, void* workspace,
                      size_t workspace_bytes, void* stream);

/* ---- forward-only layer calls ---------------------------------------------------------------------
 * tfm_layer_fwd_context and tfm_layer_fwd_query with the item axis' keys and values kept in 8 bits:
 *
 *   tfm_layer_fwd_context8  the context call (the same Y and kv_cache), after which the train rows'
 *       keys and values are appended to cache8.  kv_cache is scratch here (tfm_infer_cache_bytes of
 *       the context's dims): one serves every layer of a stack.
 *   tfm_layer_fwd_query8    the query call against cache8.  Each query row's answer depends on itself
 *       and the context alone, up to the order of sums, which goes by dims and context_rows.
 *
 * cache8 (tfm_infer_cache8_bytes of the context's dims, opaque layout) is a pool of pages of 64 rows
 * with a power of two for each page and head: half the bfloat16 cache's bytes, but for a column's last
 * page, and three bits of fraction.
 * Limits and conditions are those of the two calls; tfm_infer8_workspace_bytes is the scratch of
 * query8 (dims->R: the query rows), tfm_infer_workspace_bytes that of context8. */
size_t tfm_infer_cache8_bytes(const tfm_dims* dims);
size_t tfm_infer8_workspace_bytes(const tfm_dims* dims, int32_t context_rows);

int tfm_layer_fwd_context8(const tfm_dims* dims, const int32_t* n_train, const uint8_t* cell_mask,
                           const void* X, const float* params, void* Y, void* kv_cache,
                           size_t cache_bytes, void* cache8, size_t cache8_bytes, void* workspace,
                           size_t workspace_bytes, void* stream);

int tfm_layer_fwd_query8(const tfm_dims* dims, int32_t context_rows, const int32_t* n_train,
                         const uint8_t* cell_mask, const void* X, const float* params,
                         const void* cache8, size_t cache8_bytes, void* Y, void* workspace,
                         size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TFM_CACHE_H */

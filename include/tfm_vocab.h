/*
 * tfm_vocab.h — C ABI of the operators over discrete values at the two ends of the stack on
 * MI355X (gfx950): category or token ids in (an embedding table and its gradient), a teacher's
 * top logits as training signal (distillation), classes drawn from logits out (sampling).  They
 * stand beside the encoders and the decoder of tfm_ends.h:
 *
 *     X      = encode(x) + embed(ids)         tfm_encode_fwd, tfm_embed_fwd (accumulate)
 *     logits = decode(blocks(X))              tfm_layer_fwd per block, tfm_decode_fwd
 *     loss, dlogits                           tfm_distill_loss
 *     dY, decoder grads                       tfm_decode_bwd
 *     dX, block grads                         tfm_layer_bwd per block
 *     encoder grads, dtable                   tfm_encode_bwd, tfm_embed_bwd
 *     answers                                 tfm_sample
 *
 * Conventions: the caller owns every buffer and the library allocates nothing; calls are
 * asynchronous on `stream` (a hipStream_t, NULL = the null stream) of the current device and may
 * be captured into a graph; pointers are device pointers, aligned to their elements (workspaces to
 * 16 bytes); sums run in a fixed order (the same call gives the same bits again; the last bits of a
 * distillation may differ between buffers that lie otherwise to 16 bytes); on a negative return
 * (the codes of tfm_layer.h) nothing was launched and tfm_last_error() describes the error.  dtype
 * fields are tfm_dtype values.  Sums, softmax statistics and losses are held in 32 or 64 bits and
 * each bfloat16 output is rounded once.  Calls that run at the same time need workspaces of their
 * own.  Ids and class indices outside their range are absent: they are skipped as described, and
 * never read or written through.
 */
#ifndef TFM_VOCAB_H
#define TFM_VOCAB_H

#include "tfm_layer.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- embedding ------------------------------------------------------------------------------
 * ids: int32 [n0][n1][n2], an id in [0, V) or absent (any other value).  Row (i, j, k) of the
 * activations is the E elements from element i stride[0] + j stride[1] + k stride[2] of out (dout)
 * on; elements between the rows are left as they were.  Rows side by side: n = {1, 1, N}, stride =
 * {0, 0, E}.  The first n2 cells of every data row of a stack input X[B][R][C+1][E]: n = {B, R - T,
 * n2}, stride = {R (C+1) E, (C+1) E, E}, out = X + T (C+1) E.  table: [V][E], side by side.
 *
 *   tfm_embed_fwd   out row = scale table[id], 0 for an absent id; with accumulate != 0 it adds
 *                   scale table[id] to the row instead and leaves the rows of absent ids as they
 *                   were.
 *   tfm_embed_bwd   dtable[V][E] (float32) = scale times the sum, over the positions that hold the
 *                   id, of dout's rows, in the order of the positions up to how the sum is split
 *                   (a split that depends on the ids, sizes and dtype alone, not on strides or
 *                   where the buffers lie); rows of ids that do not occur are 0; with accumulate
 *                   != 0 it is added to dtable and those rows are left as they were.
 *
 * Limits: every n >= 0 and their product at most 2^27; 1 <= V <= 2^24; 1 <= E <= 2^16; strides in
 * [0, 2^40], the last row at most 2^48 elements from the first.  The forward's rows must not
 * overlap: in order of their strides, each axis longer than one must step past all that the ones
 * before it reach (the backward only reads its rows: any strides, 0 for a broadcast gradient).
 * out and table (dtable, dout and workspace) must not share memory. */
typedef struct {
  int32_t n[3];        /* shape of ids */
  int32_t E, V;        /* row width; table rows */
  int32_t dtype;       /* of out and dout */
  int32_t table_dtype; /* of table (forward; dtable is float32) */
  float scale;         /* finite */
  int64_t stride[3];   /* elements */
} tfm_embed;

/* Bytes of scratch of tfm_embed_bwd (0 on invalid arguments). */
size_t tfm_embed_workspace_bytes(const tfm_embed* e);

int tfm_embed_fwd(const tfm_embed* e, const int32_t* ids, const void* table, void* out,
                  int accumulate, void* stream);
int tfm_embed_bwd(const tfm_embed* e, const int32_t* ids, const void* dout, float* dtable,
                  int accumulate, void* workspace, size_t workspace_bytes, void* stream);

/* ---- distillation from a teacher's top logits ------------------------------------------------
 * Row n has the student's logits s[0 .. V), of which the classes [0, n_class[n]) count (n_class
 * nullable: all V; a value is cut to [0, V]), and the teacher's entries (top_idx[n][j],
 * top_logit[n][j]), j < k, in any order; an entry whose index is outside the row's classes is
 * absent, and of a repeated index the first entry counts.  With tau = temperature, J the classes of
 * the entries and q = softmax(s / tau) over the row's classes:
 *
 *   tail == 0   p_j = softmax of top_logit / tau over the entries; p_t = 0
 *   tail == 1   p_j = exp(top_logit_j / tau - top_lse[n]), top_lse[n] being the log-sum-exp of all
 *               of the teacher's logits / tau; p_t = max(0, 1 - sum p_j) stands for all classes
 *               outside J together (0 where no class outside J has a logit above -inf)
 *   D = sum_j p_j (log p_j - log q_j) + p_t (log p_t - log sum_{v not in J} q_v)
 *   L = alpha tau^2 D + (1 - alpha) (log sum_v exp(s_v) - s_label)
 *
 * The last term is left out where labels[n] is absent (labels may be null if alpha == 1).  The
 * outputs are
 *
 *   row_loss[n] = L (nullable),  loss[0] = sum_n w_n L_n / sum_n w_n  (weights null: all 1; 0 if
 *   the weights sum to 0),  dlogits = the gradient of loss with respect to the logits (nullable:
 *   loss alone), 0 in [n_class[n], V).
 *
 * Rows of weight 0, rows without a class and rows whose classes all have a logit of -inf are left
 * out: row_loss and dlogits are 0 whatever else they hold (the weight of the latter two still
 * counts).  A -inf logit has q = 0 and no gradient but -p; a NaN or +inf logit, and a teacher's
 * logit that is NaN or +inf, give that row a loss that is not finite and undefined gradients
 * (alpha == 0 without a label leaves L no term: 0).  Teacher's -inf logits have p = 0.
 *
 * logits and dlogits: rows of V elements ld apart, the elements between rows untouched; dlogits
 * may be logits itself (in place) but must not overlap it otherwise (from the first element of the
 * first row to the last of the last: rows that lie between the other's rows are refused too).
 * Limits: 0 <= N <= 2^27, 1 <= V <= 2^18, 1 <= k <= 256, V <= ld <= 2^40, N ld <= 2^48,
 * temperature in [2^-20, 2^20] (D is held to about 2^-22, so the loss's error grows with tau^2),
 * 0 <= alpha <= 1. */
typedef struct {
  int32_t N, V, k;
  int32_t dtype; /* of logits and dlogits */
  int32_t tail;  /* 0 or 1 */
  float temperature, alpha;
  int64_t ld;
} tfm_distill;

/* Bytes of scratch of tfm_distill_loss (0 on invalid arguments). */
size_t tfm_distill_workspace_bytes(const tfm_distill* d);

int tfm_distill_loss(const tfm_distill* d, const void* logits, const int32_t* top_idx,
                     const float* top_logit, const float* top_lse, const int32_t* labels,
                     const float* weights, const int32_t* n_class, float* loss, float* row_loss,
                     void* dlogits, void* workspace, size_t workspace_bytes, void* stream);

/* ---- sampling ---------------------------------------------------------------------------------
 * Draws one class per row from the logits s[0 .. V), of which the classes [0, n_class[n]) count
 * (nullable as above), with settings per row (each nullable: off) and a given uniform number.
 * With x_v = (s_v - max s) / temperature and the classes ordered by falling logit, the lower index
 * first among equals, the kept classes are the longest run from the front that every rule allows:
 *
 *   top_k   at most top_k classes                                   (off: <= 0)
 *   top_p   a class while the ones before it hold less than top_p of the probability of the first
 *           top_k classes                                           (off: >= 1 or NaN)
 *   min_p   a class while exp(x_v) >= min_p                         (off: <= 0 or NaN)
 *
 * The first class is always kept.  token[n] is the first kept class, in order of class index, at
 * which the running sum of exp(x) over the kept classes exceeds u[n] times its total;
 * logprob[n] (nullable) = x_token - log(total).  temperature null: 1; temperature <= 0 or NaN:
 * the first class of the order.  u below 0 or NaN counts as 0, u >= 1 as the largest float32 below
 * 1.  -inf and NaN logits are never drawn; among +inf logits x = 0, and other classes have
 * probability 0.  A row without a class that can be drawn gets token -1 and logprob -inf.
 *
 * The weights exp(x) are rounded to multiples of 2^-51 (2^-44 at V = 2^18) and summed exactly, so a
 * draw depends on its row alone and neither on the order of summation nor on the batch.
 * Limits: 0 <= N <= 2^27, 1 <= V <= 2^18, V <= ld <= 2^40 (rows ld elements apart), N ld <= 2^48. */
typedef struct {
  int32_t N, V;
  int32_t dtype; /* of logits */
  int64_t ld;
} tfm_sampling;

int tfm_sample(const tfm_sampling* s, const void* logits, const int32_t* n_class,
               const float* temperature, const int32_t* top_k, const float* top_p,
               const float* min_p, const float* u, int32_t* token, float* logprob, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* TFM_VOCAB_H */

/*
 * liblda: operators of neural word models on one AMD Instinct MI355X.
 *
 * A word model predicts the words of a document from a vector of its topics:
 * layer norm, a gated layer, and a softmax over the whole vocabulary, whose
 * loss is the negative log-likelihood per token that lda_loglik reports for
 * the fitted counts (there in base 2).  A model that reads the words themselves
 * in order embeds them and runs a gated recurrence over each document, and may
 * learn from a teacher's most likely words.  Each operator has its forward and
 * its backward pass.
 *
 * Conventions for every call:
 *   - All data pointers are device memory of the current device, owned by the
 *     caller.  The work is enqueued on `stream` (a hipStream_t; NULL = the
 *     null stream) and the call returns without waiting for it.
 *   - Matrices are row-major with unit column stride; ld* is the row stride
 *     in elements.  Inputs may overlap or repeat rows (any ld >= 0); outputs
 *     need ld >= columns and must not overlap anything else of the call.
 *     Pointers need the alignment of their element type only.  Matrices whose
 *     rows start at multiples of 16 bytes and hold a multiple of 16 bytes are
 *     read where they lie; others are slower (the products copy them into the
 *     workspace first).
 *   - Sums, softmax statistics and row statistics are kept in 32 bits or more; an
 *     output is rounded once to its type.  Every sum has one order: results
 *     are the same bits on every run.
 *   - `workspace` is device scratch of at least the size that the operator's
 *     *_workspace call gives for the same arguments (256-byte aligned; NULL if
 *     that size is 0).  It may be reused by later work on the same stream.
 *   - Nothing throws across this boundary; nothing is allocated.  Calls return
 *     LDA_E_ARG (NULL pointer, negative size, unknown type, stride or
 *     workspace too small), LDA_E_RANGE (a size limit below), LDA_E_DEVICE
 *     (a launch failed); lda_last_error(NULL) has the message for the calling
 *     thread.
 */
#ifndef LDA_OPS_H
#define LDA_OPS_H

#include "lda.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of the matrices of a call. */
typedef enum { LDA_F32 = 0, LDA_BF16 = 1, LDA_F16 = 2 } lda_dtype;

/* Activation of the gated layer: a*sigmoid(a), a*Phi(a) with the normal
 * distribution function Phi, sigmoid(a). */
typedef enum { LDA_SILU = 0, LDA_GELU = 1, LDA_SIGMOID = 2 } lda_act;

/* Most rows, columns or words of one call. */
#define LDA_OPS_MAX_ROWS 16777216
#define LDA_OPS_MAX_COLS 1048576
#define LDA_OPS_MAX_VOCAB 16777216
/* Most tiles of 128 x 128 of a product's result (logits, gated layer, weight
 * gradient): a call on more rows is made in parts. */
#define LDA_OPS_MAX_TILES 8388608
/* Most bytes of an embedding's gradient, and most parts of 512 rows by 1,024 bytes
 * that it is summed from. */
#define LDA_OPS_MAX_EMBED_BYTES 273804165120
#define LDA_OPS_MAX_EMBED_PARTS 67108860
/* Most words that a teacher lists for a row, and most of all rows of a call
 * (rows times top). */
#define LDA_OPS_MAX_TOP 256
#define LDA_OPS_MAX_LISTED 268435456
/* Rows from one kept state of a recurrence to the next. */
#define LDA_OPS_RECUR_ROWS 16

/*
 * Layer norm of each row of x [rows][cols]:
 *   mean = sum x / cols, rstd = 1 / sqrt(sum (x - mean)^2 / cols + eps)
 *   y = (x - mean) * rstd * weight + bias
 * weight and bias [cols] are given together or both NULL (1 and 0).
 * mean and rstd [rows] are always in 32 bits.  eps must be finite and >= 0.
 *
 * The backward pass takes dy and the forward's mean and rstd:
 *   g = dy * weight, h = (x - mean) * rstd
 *   dx = rstd * (g - mean(g) - h * mean(g h))
 *   dweight = sum over rows of dy h, dbias = sum over rows of dy
 * dweight and dbias are given together or both NULL (not computed).  With
 * rows = 0 they are set to zero.
 */
typedef struct {
  int32_t dtype; /* lda_dtype of x, weight, bias, y, dy, dx, dweight, dbias */
  int64_t rows;
  int32_t cols; /* >= 1 */
  float eps;
  const void *x;
  int64_t ldx;
  const void *weight, *bias;
  void *y; /* forward */
  int64_t ldy;
  float *mean, *rstd; /* written by the forward, read by the backward pass */
  const void *dy;     /* backward */
  int64_t lddy;
  void *dx;
  int64_t lddx;
  void *dweight, *dbias;
  void *workspace; /* backward */
  size_t workspace_bytes;
  void *stream;
} lda_norm_args;

lda_status lda_layer_norm(const lda_norm_args *a);
lda_status lda_layer_norm_backward_workspace(const lda_norm_args *a, size_t *bytes);
lda_status lda_layer_norm_backward(const lda_norm_args *a);

/*
 * Gated layer: x [rows][width], w_gate and w_value [hidden][width],
 *   a = x w_gate^T, b = x w_value^T, h = act(a) * b   [rows][hidden]
 * in one kernel; a and b stay in registers.  The backward pass recomputes
 * them from x:
 *   da = dh * b * act'(a), db = dh * act(a)
 *   dx = da w_gate + db w_value, dw_gate = da^T x, dw_value = db^T x
 * da and db are rounded to the type of the matrices, as operands of the three
 * products; in half precision times a power of two for each row, so that they
 * may pass the type's range where the gradients do not (a row's part of the
 * weights' gradients loses bits where max |dh| max |x| |x|, |x| the row's length,
 * is more than some 2^29 below the largest row's).  With rows = 0 the weights'
 * gradients are set to zero.
 */
typedef struct {
  int32_t dtype, act; /* lda_dtype, lda_act */
  int64_t rows;
  int32_t width, hidden; /* >= 1 */
  const void *x;
  int64_t ldx;
  const void *w_gate;
  int64_t ld_gate;
  const void *w_value;
  int64_t ld_value;
  void *h; /* forward */
  int64_t ldh;
  const void *dh; /* backward */
  int64_t lddh;
  void *dx;
  int64_t lddx;
  void *dw_gate, *dw_value; /* row stride width */
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} lda_gated_args;

lda_status lda_gated_workspace(const lda_gated_args *a, size_t *bytes);
lda_status lda_gated(const lda_gated_args *a);
lda_status lda_gated_backward_workspace(const lda_gated_args *a, size_t *bytes);
lda_status lda_gated_backward(const lda_gated_args *a);

/*
 * Softmax cross entropy over a vocabulary, without keeping the logits:
 * x [rows][width], weight [vocab][width], bias [vocab] in 32 bits or NULL,
 *   z = x weight^T + bias, lse_i = log sum_v exp z_iv
 *   loss_i = lse_i - z[i][label_i]
 * A label outside [0, vocab) leaves its row out: loss 0, no gradient,
 * whatever the row of x holds.  A bias of -inf masks a word: its probability
 * is 0, and so is that of a row whose words are all masked (lse -inf); the
 * loss of a masked label is +inf.
 *
 * The backward pass takes dloss [rows] and the forward's lse, recomputes the
 * logits in pieces of the vocabulary (as many words as take 256 MiB, but at
 * least 1,024) and keeps one piece of
 *   G_iv = dloss_i * (exp(z_iv - lse_i) - [v = label_i])
 * (0 for rows left out and rows without words) in the workspace:
 *   dx = G weight, dweight = G^T x, dbias = sum over rows of G
 * As an operand of the first two products, in 16-bit types, G is kept without
 * dloss and rounded to the type of the matrices (dbias is summed before); dloss
 * multiplies dx in 32 bits, and x, rounded once more, for dweight (in half
 * precision a row's part of dweight loses bits where its |x dloss| is more than
 * some 2^28 times below the largest).  Rows of weight must be finite also where
 * their word is masked.  dbias is NULL if and only if bias is.  With rows = 0,
 * dweight and dbias are set to zero.
 */
typedef struct {
  int32_t dtype;
  int64_t rows;
  int32_t width, vocab; /* >= 1 */
  const void *x;
  int64_t ldx;
  const void *weight;
  int64_t ld_weight;
  const float *bias;
  const int32_t *labels;
  float *loss; /* forward */
  float *lse;  /* written by the forward, read by the backward pass */
  const float *dloss; /* backward */
  void *dx;
  int64_t lddx;
  void *dweight; /* row stride width */
  float *dbias;
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} lda_xent_args;

lda_status lda_softmax_xent_workspace(const lda_xent_args *a, size_t *bytes);
lda_status lda_softmax_xent(const lda_xent_args *a);
lda_status lda_softmax_xent_backward_workspace(const lda_xent_args *a, size_t *bytes);
lda_status lda_softmax_xent_backward(const lda_xent_args *a);

/*
 * Word embedding: words [rows], weight [vocab][width],
 *   y_i = scale * weight[word_i]
 * and 0 for a word outside [0, vocab).  The backward pass takes dy:
 *   dweight_v = scale * sum of dy_i over the rows with word_i = v
 * (0 for a word that no row has; rows outside the vocabulary have no part in
 * it, whatever their dy holds).  The rows are sorted by word and a word's are
 * summed in their order, in pieces of a fixed length: in 32 bits for 16-bit types,
 * in 64 bits for single precision, so that dweight is off by its own rounding
 * alone however many rows a word has.  scale must be finite.
 */
typedef struct {
  int32_t dtype; /* of weight, y, dy, dweight */
  int64_t rows;
  int32_t width, vocab; /* >= 1 */
  float scale;
  const int32_t *words;
  const void *weight; /* forward */
  int64_t ld_weight;
  void *y;
  int64_t ldy;
  const void *dy; /* backward */
  int64_t lddy;
  void *dweight; /* row stride width */
  void *workspace; /* backward */
  size_t workspace_bytes;
  void *stream;
} lda_embed_args;

lda_status lda_embedding(const lda_embed_args *a);
lda_status lda_embedding_backward_workspace(const lda_embed_args *a, size_t *bytes);
lda_status lda_embedding_backward(const lda_embed_args *a);

/*
 * Gated linear recurrence over documents: x and gate [rows][cols]; document s
 * has the rows offsets[s] .. offsets[s + 1] - 1, and begins with its row of
 * state [docs][cols] (32 bits; NULL = 0):
 *   f_t = sigmoid(gate_t), h_t = f_t h_{t-1} + (1 - f_t) x_t
 *   last_s = h of its last row, of an empty document its state
 * in each column by itself; h is rounded to the type of the matrices, the state
 * that goes on is not.  Rows of no document are 0 in h and in the gradients,
 * whatever x, gate and dh hold there, and no document's values, infinities and
 * NaN included, reach another one.  offsets [docs + 1] are device memory and not
 * checked: they must not decrease (values are unspecified if they do, no access
 * is out of range) and what lies outside [0, rows] is cut off.  A call has at most
 * LDA_OPS_MAX_TILES / 2 parts of 256 rows by 64 columns.
 *
 * kept [ceil(rows / LDA_OPS_RECUR_ROWS)][cols] are the states before every
 * LDA_OPS_RECUR_ROWS-th row, for the backward pass.  It takes dh and dlast
 * [docs][cols] (NULL = 0):
 *   g_t = dh_t + f_{t+1} g_{t+1}; the last row's is dh + dlast
 *   dx_t = (1 - f_t) g_t, dgate_t = g_t (h_{t-1} - x_t) f_t (1 - f_t)
 *   dstate_s = f g of its first row, of an empty document dlast_s
 * dstate is NULL if and only if state is.
 *
 * The step is one row more of each of `rows` documents: x, gate and h
 * [rows][cols], state and last [rows][cols], which may be the same memory.  It
 * has no offsets, kept and workspace; docs must be rows.
 */
typedef struct {
  int32_t dtype; /* of x, gate, h, dh, dx, dgate */
  int64_t rows;
  int32_t cols; /* >= 1 */
  int64_t docs; /* at most LDA_OPS_MAX_ROWS */
  const int64_t *offsets;
  const void *x;
  int64_t ldx;
  const void *gate;
  int64_t ld_gate;
  const float *state;
  void *h; /* forward and step */
  int64_t ldh;
  float *last;
  float *kept;    /* written by the forward, read by the backward pass */
  const void *dh; /* backward */
  int64_t lddh;
  const float *dlast;
  void *dx;
  int64_t lddx;
  void *dgate;
  int64_t ld_dgate;
  float *dstate;
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} lda_recur_args;

lda_status lda_recurrence_workspace(const lda_recur_args *a, size_t *bytes);
lda_status lda_recurrence(const lda_recur_args *a);
lda_status lda_recurrence_backward_workspace(const lda_recur_args *a, size_t *bytes);
lda_status lda_recurrence_backward(const lda_recur_args *a);
lda_status lda_recurrence_step(const lda_recur_args *a);

/*
 * Distillation over a vocabulary: how far the softmax over x weight^T + bias is
 * from a teacher that lists up to `top` words and their scores (logits, or
 * logarithms of probabilities) for each row, both softened by the temperature,
 * without keeping the logits:
 *   z = (x weight^T + bias) / temperature, lse_i = log sum_v exp z_iv
 *   p_i = softmax of the row's scores / temperature over its listed words
 *   loss_i = sum_j p_ij (log p_ij - (z[i][word_ij] - lse_i))
 * words and scores are [rows][top]; a word outside [0, vocab) is an empty place,
 * whatever its score.  A word listed twice counts with both places.  A row
 * without listed words, or whose scores are all -inf, is left out: loss 0, no
 * gradient, whatever its x holds.  A score of -inf has p = 0 and no part in the
 * loss; a listed word with p > 0 that the bias masks (-inf) makes it +inf.
 * logits [rows][top] are the z of the listed words (0 at empty places), kept for
 * the backward pass:
 *   G_iv = dloss_i / temperature * (exp(z_iv - lse_i) - p_iv)
 *   dx = G weight, dweight = G^T x, dbias = sum over rows of G
 * p_iv being the p of the row's places with word v (0 for rows left out and rows
 * without words).  As for the softmax cross entropy the logits are recomputed in
 * pieces of the vocabulary, one piece of G is kept, without the power of two in
 * dloss / temperature and in 16-bit types rounded to them (up to 128 rows with what
 * the rounding left beside it), and rows of weight must be finite; in half precision
 * a row's part of dweight loses bits as there.  dbias is NULL if and only if bias is.
 * temperature and its reciprocal must be finite and positive.
 */
typedef struct {
  int32_t dtype;
  int64_t rows;
  int32_t width, vocab, top; /* >= 1 */
  float temperature;
  const void *x;
  int64_t ldx;
  const void *weight;
  int64_t ld_weight;
  const float *bias;
  const int32_t *words;
  int64_t ld_words;
  const float *scores;
  int64_t ld_scores;
  float *loss;        /* forward */
  float *lse;         /* written by the forward, read by the backward pass */
  float *logits;      /* the same; row stride top */
  const float *dloss; /* backward */
  void *dx;
  int64_t lddx;
  void *dweight; /* row stride width */
  float *dbias;
  void *workspace;
  size_t workspace_bytes;
  void *stream;
} lda_distill_args;

lda_status lda_softmax_distill_workspace(const lda_distill_args *a, size_t *bytes);
lda_status lda_softmax_distill(const lda_distill_args *a);
lda_status lda_softmax_distill_backward_workspace(const lda_distill_args *a, size_t *bytes);
lda_status lda_softmax_distill_backward(const lda_distill_args *a);

#ifdef __cplusplus
}
#endif
#endif

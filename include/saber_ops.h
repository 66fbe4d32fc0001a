/*
 * saber_ops.h - operators of a head that is trained on a topic model's features (gfx950): layer norm, softmax cross
 * entropy together with its projection onto the vocabulary, and activation checkpoints in 8 bits; and of one that
 * answers: root-mean-square norm of a residual stream, rows in 8 bits and their product, words drawn from logits.
 *
 * The head takes features of every token (its topic of saber_get_z, its document's row of A, an embedding of the word
 * before) through a norm to logits over the sampler's own vocabulary and scores the token's word, or draws one.
 *
 * Conventions
 *   - Every pointer to data is a DEVICE pointer (tensors stay where they are); the caller owns all of them, the work
 *     space included.  Pointers must be aligned to their elements, the work space to 256 bytes.
 *   - A matrix is rows of `cols` consecutive elements that lie `stride` elements apart (stride >= cols); outputs are
 *     contiguous.  Rows may start at any element: what is not aligned to 16 bytes costs time, nothing else.  Outputs
 *     must not overlap inputs.
 *   - Every call only enqueues kernels on `stream` (a hipStream_t of the current device, null: the default stream): it
 *     allocates nothing, waits for nothing and may be captured into a graph.
 *   - Element types: binary32, binary16, bfloat16.  Sums, statistics and losses are binary32 in every case; results are
 *     rounded once, to nearest even.  The same inputs give the same bits.
 *   - Every function returns SABER_OK or a negative saber_status (saber.h) and never throws;
 *     saber_ops_last_error() has the message of the calling thread's last failure.
 *   - Limits: fewer than 2^31 rows and words, at most 2^20 columns; cross entropy: at most 2^26 - 16 rows, and
 *     fewer than 2^40 values of the features in its backward pass; products of 8-bit rows: at most 2^17 - 1 columns and
 *     2^24 tiles of 256 x 256 logits; drawing: fewer than 2^31 words (ERANGE).
 */
#ifndef SABER_OPS_H
#define SABER_OPS_H

#include "saber.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum saber_dtype {
    SABER_F32 = 0,
    SABER_F16 = 1,
    SABER_BF16 = 2
} saber_dtype;

/* Message of the calling thread's last failed call of this header (static storage, never NULL). */
const char *saber_ops_last_error(void);

/*
 * Layer norm of every row: m = mean x, v = mean (x - m)^2, y = (x - m) / sqrt(v + eps) * weight + bias.
 *   x [rows][cols] of dtype; weight, bias [cols] of wtype, either may be NULL (ones, zeros)
 *   y [rows][cols] of dtype; mean, rstd [rows]: m and 1 / sqrt(v + eps), what the backward pass needs
 *   q, scale       both NULL, or a checkpoint of x (saber_checkpoint8_save) that is written in the same pass
 * Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_layer_norm_forward(const void *x, int64_t x_stride, const void *weight, const void *bias, int64_t rows,
                             int64_t cols, int dtype, int wtype, float eps, void *y, float *mean, float *rstd, int8_t *q,
                             float *scale, void *stream);

/* Bytes of work space that saber_layer_norm_backward needs for dweight or dbias. */
int saber_layer_norm_backward_workspace(int64_t rows, int64_t cols, int64_t *bytes);

/*
 * Gradients of the above: with h = (x - m) rstd and g = dy * weight
 *   dx = rstd (g - mean(g) - h mean(g h)),  dweight = sum over rows of dy h,  dbias = sum over rows of dy
 *   dy [rows][cols] of dtype; x as in the forward pass, or NULL with a checkpoint of it in q and scale: the values that
 *                 the checkpoint stands for then take the place of x in h, with m and rstd of x itself (an approximation,
 *                 half a step of the checkpoint off at most; h then has not exactly mean 0 and variance 1)
 *   dx [rows][cols] of dtype, dweight and dbias [cols] of wtype; any of them may be NULL (not computed)
 *   workspace     needed for dweight or dbias
 * No rows give zeros for dweight and dbias.  Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, const int8_t *q,
                              const float *scale, const float *mean, const float *rstd, const void *weight, int64_t rows,
                              int64_t cols, int dtype, int wtype, void *dx, void *dweight, void *dbias, void *workspace,
                              int64_t workspace_bytes, void *stream);

/*
 * An activation in 8 bits.  Every 128 columns of a row (the last block may be shorter) share a step
 * c = max|x| / 127 (binary32, and at most the largest c of which 127 c is finite); an element is held as round(x / c), ties
 * to even, within -127 .. 127, and restored as that number times c: at most half a step off where c is a normal number
 * (below, c itself is rounded coarsely).  A block of zeros has step 0.  A block with an infinity or NaN is
 * restored as NaN.
 *   q [rows][cols], scale [rows][ceil(cols / 128)]
 */
int saber_checkpoint8_save(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int dtype, int8_t *q,
                           float *scale, void *stream);
int saber_checkpoint8_restore(const int8_t *q, const float *scale, int64_t rows, int64_t cols, int dtype, void *x,
                              void *stream);

/*
 * Softmax cross entropy of x weight^T: lse_n = log sum_v exp(x_n . W_v), loss_n = lse_n - x_n . W_target(n).  The logits
 * are never held: the work space is packed operands where they are needed (of the weight at most 256 MB at a time) and
 * a maximum and a sum per row and tile of words.
 *   x [rows][cols], weight [vocab][cols] of dtype; target [rows]: int32, or int64 if target64
 *   A negative target leaves the row out: its loss is 0 (lse is still the row's).  One of vocab or more gives NaN.
 *   loss, lse [rows]
 *   workspace, workspace_bytes   with workspace NULL the bytes needed are stored there and nothing else is done;
 *                                otherwise *workspace_bytes is what the work space holds.  (The need depends on sizes,
 *                                strides, types and the 16-byte alignment of x and weight.)
 * Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_linear_xent_forward(const void *x, int64_t x_stride, const void *weight, int64_t w_stride, const void *target,
                              int target64, int64_t rows, int64_t vocab, int64_t cols, int dtype, float *loss, float *lse,
                              void *workspace, int64_t *workspace_bytes, void *stream);

/*
 * Gradients for dloss [rows]: with d_nv = dloss_n (exp(x_n . W_v - lse_n) - [v = target(n)])
 *   dx_n = sum_v d_nv W_v,  dweight_v = sum_n d_nv x_n
 *   lse as the forward pass gave it; dx [rows][cols], dweight [vocab][cols] of dtype, either may be NULL
 * Between the products d is held in the type of x, for one piece of the vocabulary at a time; binary32 keeps its 24
 * bits.  The work space does not grow with the vocabulary: d of a piece takes 256 MB at most and so do its packed words
 * (256 words make a piece whatever the sizes), beside copies of the features and partial sums of dx.  Rows left out have zeros in dx and add nothing to dweight, whatever x and lse
 * hold there; no rows give zeros for dweight.  workspace as above.  Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_linear_xent_backward(const float *dloss, const void *x, int64_t x_stride, const void *weight, int64_t w_stride,
                               const void *target, int target64, const float *lse, int64_t rows, int64_t vocab,
                               int64_t cols, int dtype, void *dx, void *dweight, void *workspace,
                               int64_t *workspace_bytes, void *stream);

/*
 * Root-mean-square norm of every row of a residual stream: s = x + residual, rounded to the stream's type,
 * r = 1 / sqrt(mean s^2 + eps), y = s r weight.  The norm is of the sum as it is held.
 *   x [rows][cols] of dtype; residual [rows][cols] of rtype (dtype or SABER_F32), or NULL: then s = x, rtype is dtype and
 *                 sum is NULL
 *   weight [cols] of wtype, or NULL (ones)
 *   sum [rows][cols] of rtype: s
 *   y [rows][cols] of dtype; or y NULL and q, q_stride, scale: y in 8 bits (saber_rows8_save).  With t = s weight in
 *                 binary32, c = max|t| / 127 of the row: q = round(t / c), scale = c r
 *   rstd [rows]: r, what the backward pass needs; or NULL
 * Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_rms_norm_forward(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride,
                           const void *weight, int64_t rows, int64_t cols, int dtype, int rtype, int wtype, float eps,
                           void *sum, void *y, float *rstd, int8_t *q, int64_t q_stride, float *scale, void *stream);

/* Bytes of work space that saber_rms_norm_backward needs for dweight. */
int saber_rms_norm_backward_workspace(int64_t rows, int64_t cols, int64_t *bytes);

/*
 * Gradients of the above (of y, not of its form in 8 bits): with h = s r and g = dy * weight
 *   ds = r (g - h mean(g h)) + dsum,  dweight = sum over rows of dy h
 *   dy [rows][cols] of dtype; dsum [rows][cols] of rtype, the gradient of the sum as the stream goes on with it, or NULL
 *   s [rows][cols] of rtype: the sum (x, where there was no residual)
 *   dx of dtype, dresidual of rtype, both [rows][cols]: ds, rounded to either type; dweight [cols] of wtype; any may be NULL
 *   workspace     needed for dweight
 * No rows give zeros for dweight.  Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_rms_norm_backward(const void *dy, int64_t dy_stride, const void *dsum, int64_t dsum_stride, const void *s,
                            int64_t s_stride, const float *rstd, const void *weight, int64_t rows, int64_t cols, int dtype,
                            int rtype, int wtype, void *dx, void *dresidual, void *dweight, void *workspace,
                            int64_t workspace_bytes, void *stream);

/*
 * Rows in 8 bits, the operands of saber_linear8: a row has one step c = max|x| / 127 (binary32, and at most the largest c
 * of which 127 c is finite), an element is held as round(x / c), ties to even, and restored as that number times c.  A row
 * of zeros has step 0; one with an infinity or NaN is restored as NaN.
 *   q: rows of cols bytes that start at multiples of 16 bytes, q_stride bytes apart (a multiple of 16); those up to the next
 *      multiple of 16 are zeros (written by saber_rows8_save)
 *   scale [rows]: the steps
 */
int saber_rows8_save(const void *x, int64_t x_stride, int64_t rows, int64_t cols, int dtype, int8_t *q, int64_t q_stride,
                     float *scale, void *stream);
int saber_rows8_restore(const int8_t *q, int64_t q_stride, const float *scale, int64_t rows, int64_t cols, int dtype,
                        void *x, void *stream);

/*
 * Logits from rows in 8 bits: out_nv = (sum over k of x_nk weight_vk) x_scale_n w_scale_v.  The sums are int32 and exact; then
 * a sum is rounded to binary32, multiplied by either scale in this order, each product rounded to binary32, and the result
 * to dtype.
 *   x [rows][cols], weight [words][cols] as above; values -128 .. 127; out [rows][words] of dtype
 * Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_linear8(const int8_t *x, int64_t x_stride, const float *x_scale, const int8_t *weight, int64_t w_stride,
                  const float *w_scale, int64_t rows, int64_t words, int64_t cols, int dtype, void *out, void *stream);

/*
 * Draws a word for every row of logits l by the row's random number u: with z = (l - max l) / temperature and the words in
 * falling order of their logits, equal ones in the order of their numbers, these are left:
 *   the first top_k (0 or less: all), of them the fewest that hold top_p of their sum of exp z (1 or more: all), of them
 *   those of exp z >= min_p; always the first one
 * and the first word, by number, is taken at which the sum of exp z of the words left exceeds u times that of all of them.
 * The masses are sums of whole multiples of 2^-45 (of 2^(ceil(log2 words) - 62) beyond 2^17 words) of the likeliest
 * word's: what is below half of that has none, also where there are so many such words that together they would have
 * some.  The limits are compared in 64 bits; a share of the whole counts as held from 2^-40 of the whole below it.
 * u is a binary32, so of 24 bits where torch's rand or the like makes it: a word of less than 2^-24 of the mass left is
 * drawn only if a multiple of 2^-24 falls on it.
 *   logits [rows][words] of dtype; -inf leaves a word out, infinite ones share all of the mass
 *   temperatures, top_ks (int32, or int64 if top_k64), top_ps, min_ps [rows]: a value per row, or NULL: then temperature,
 *                 top_k, top_p, min_p hold for all rows (and are checked: one below 0 is refused).  A temperature of 0 (as
 *                 a value per row also less, or NaN) takes the first word of the largest logit, whatever the limits.
 *                 As values per row a top_p or min_p below 0 counts as 0, beyond 1 as 1, and NaN as no limit.
 *   u [rows]: within [0, 1); what is outside counts as the next number within, NaN as 0
 *   word [rows], p [rows]: the word and its share of the mass left.  A row of which nothing is left (all -inf): -1 and 0.
 *                 One with a NaN: -1 and NaN.
 * Errors: EINVAL, ERANGE, EDEVICE.
 */
int saber_sample(const void *logits, int64_t stride, int64_t rows, int64_t words, int dtype, const float *u,
                 const float *temperatures, float temperature, const void *top_ks, int top_k64, int64_t top_k,
                 const float *top_ps, float top_p, const float *min_ps, float min_p, int64_t *word, float *p, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* SABER_OPS_H */

/*
 * saber_ops.h - operators of a head that is trained on a topic model's features (gfx950): layer norm, softmax cross
 * entropy together with its projection onto the vocabulary, and activation checkpoints in 8 bits.
 *
 * The head takes features of every token (its topic of saber_get_z, its document's row of A, an embedding of the word
 * before) through a norm to logits over the sampler's own vocabulary and scores the token's word.
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
 *     fewer than 2^40 values of the features in its backward pass (ERANGE).
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

#ifdef __cplusplus
}
#endif
#endif /* SABER_OPS_H */

/* Layers of networks whose gradients are aggregated by CodedReduce, on one AMD MI355X (gfx950).
 *
 * Coded aggregation (codedreduce.h) recovers the exact full gradient from what redundant workers form, on three conditions on the network
 * whose gradients are handed to it: its loss is a SUM over data points; a point's gradient depends on that point alone, whatever else its
 * holder has; and every holder of a point forms the same gradient.  These are the layers of a network that keep them (the last up to
 * rounding, as the conventions say):
 *
 *     cr_group_norm_*     normalisation within a data point, with an activation
 *     cr_dropout_*        dropout whose mask is a function of the data point's index, not of who draws it or when; with bias and residual
 *     cr_softmax_loss     the loss over several classes (of two: CR_LOGISTIC), and its gradient
 *
 * A worker computes its own points with them, or one call serves all: gradients of parameters come once per RUN of consecutive points, so
 * that a slab gradient (codedreduce.h) is the sum of the runs between its rows, and what several workers hold in common is formed once.
 *
 * Conventions (beside those of codedreduce.h: plain C ABI, cr_status, the text of the last error on the calling thread from
 * cr_layers_last_error)
 *   - an activation is `points` data points of `positions` rows of `channels` values, channels last.  The channels of a row are
 *     contiguous; points and positions have strides, in elements, zero or more (inputs may be broadcast; rows of outputs must not
 *     overlap).  Storage is fp32 or bf16 (enum cr_xdtype); parameters, their gradients and statistics are fp32, contiguous.  Any
 *     alignment that the element has will do.
 *   - all pointers but the structs and `bounds` are device addresses.  The caller owns everything; nothing is allocated.
 *   - a call enqueues kernel launches on hip_stream (NULL = the default stream) of the current device and returns without waiting: no copy,
 *     no memset, so that it may be captured in a HIP graph.  A workspace is scratch of one call: calls that overlap in time must not share it.
 *   - an output may be the very tensor of an input (same address, same strides) where this is said; other overlaps are errors that are
 *     not looked for.
 *   - sums, statistics and exponentials are held in 32 bits or more; a result is rounded once, to its type.  Every sum has a fixed order:
 *     the same call on the same inputs gives the same bits.  Between calls that have a point among other points, a row of the loss and what
 *     dropout makes of a point are the same bits too; what a group norm makes of it may differ by rounding, since the order of its sums goes
 *     by the number of points, as it does for gradients of parameters.
 *   - no points: CR_OK, gradients of parameters are zero.
 */
#ifndef CODEDREDUCE_LAYERS_H
#define CODEDREDUCE_LAYERS_H

#include "codedreduce.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cr_layer_shape {
    int64_t points, positions, channels; /* points >= 0; positions, channels >= 1; points and positions < 2^31, channels <= 2^24 */
    int32_t dtype;                       /* enum cr_xdtype of the activations */
} cr_layer_shape_t;

typedef struct cr_layer_view {           /* element (n, p, c) is at dev + (n * point_stride + p * position_stride + c) elements; strides up to 2^40, */
                                         /* points * point_stride + positions * position_stride + channels up to 2^60 */
    void *dev;
    int64_t point_stride, position_stride;
} cr_layer_view_t;

enum cr_activation { CR_ACT_NONE = 0, CR_ACT_RELU = 1, CR_ACT_SILU = 2 }; /* z; max(z, 0); z sigmoid(z) */

/* The text of the last error of a call of this header on the calling thread. */
const char *cr_layers_last_error(void);

/* ---- group norm with an activation -------------------------------------------------------------------------------------------------
 * The channels are cut into `groups` equal consecutive groups; over the M = positions * channels / groups values of a group of a point,
 *     mean = sum(x) / M,   rstd = 1 / sqrt(sum((x - mean)^2) / M + eps),   h = (x - mean) rstd,   y = act(gamma h + beta).
 *   gamma, beta   `channels` floats each, or NULL: 1 and 0
 *   y             may be x itself
 *   mean, rstd    points x groups floats each, what the gradient needs; NULL (both) where none will be asked for
 *   eps           >= 0
 * A point with a NaN or an infinity in a group has NaN there (mean and rstd of that group included) and nowhere else.
 * Distances from the mean of 10^18 and more have squares that 32 bits do not hold: rstd may be 0 there, and h with it.
 *
 * cr_group_norm_backward: from dy and what the forward pass was given and left,
 *     dz = dy act'(gamma h + beta),   dbeta = sum dz,   dgamma = sum dz h   (over the points of a run and their positions),
 *     dx = rstd (gamma dz - sum_group(gamma dz) / M - h sum_group(gamma dz h) / M).
 *   bounds        host, runs + 1 ascending indices, from 0 to `points`: run r is points [bounds[r], bounds[r+1]), which may be none.
 *                 NULL: one run of all points (runs = 1)
 *   dx            may be dy or x itself; NULL: not wanted
 *   dgamma, dbeta runs x channels floats each; NULL: not wanted (each by itself)
 * act' of CR_ACT_RELU is 0 at 0.
 * cr_group_norm_workspace_bytes: what a call on this shape needs (256-byte aligned), whichever strides and pointers it has; may be 0.
 * A point that no workgroup holds is cut into pieces of 2 000 values or more, and in the gradient every piece leaves 8 bytes a channel there.
 * That is little beside the activations but for points of few positions and wide groups: of one position and more than 4 096 channels a group
 * (2 048 of fp32), or of two to eight and half as many, it is 8 bytes a channel and point (16 384 points of 8 192 channels: 1.1 GB).  Points with 2^31 pieces between them (4 * 10^12 values or more: inputs that
 * are broadcast) are refused by cr_group_norm_workspace_bytes and cr_group_norm_backward. */
int cr_group_norm_workspace_bytes(const cr_layer_shape_t *shape, int groups, const int64_t *bounds, int runs, size_t *forward_bytes,
                                  size_t *backward_bytes);
int cr_group_norm_forward(const cr_layer_shape_t *shape, const cr_layer_view_t *x, const float *gamma, const float *beta, int groups,
                          float eps, int activation, const cr_layer_view_t *y, float *mean, float *rstd, void *workspace,
                          size_t workspace_bytes, void *hip_stream);
int cr_group_norm_backward(const cr_layer_shape_t *shape, const cr_layer_view_t *dy, const cr_layer_view_t *x, const float *mean,
                           const float *rstd, const float *gamma, const float *beta, int groups, int activation, const int64_t *bounds,
                           int runs, const cr_layer_view_t *dx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes,
                           void *hip_stream);

/* ---- bias, dropout, residual ---------------------------------------------------------------------------------------------------------
 *     y = residual + (kept ? (x + bias) * scale : 0)
 * with a mask that is drawn again wherever it is needed and never stored.  The draw for channel c at position p of the data point with
 * index i is 16 bits, the (c mod 4)-th from below, of output number
 *     (i * positions + p) * ceil(channels / 4) + c / 4       (modulo 2^64)
 * of the splitmix64 stream started at `key`, which is output number `draw` (+ *draw_dev) of the stream started at `seed`.  A value is kept
 * where its draw is at least T = floor(rate * 65536 + 0.5); scale = 65536 / (65536 - T), so that the expectation is exact for the rate
 * that is really drawn.  What is not kept has no influence on y, be it infinite or NaN. */
typedef struct cr_dropout {
    double rate;               /* 0 <= rate, T < 65536 */
    uint64_t seed, draw;       /* a draw for every layer and step: say step * layers + layer */
    const uint64_t *draw_dev;  /* device, one number added to `draw` when the kernel runs, for calls that are captured and replayed; or NULL */
    int64_t first_point;       /* the call's points have the indices first_point, first_point + 1, ... */
    const int64_t *point_dev;  /* device, `points` numbers: or these indices; NULL */
} cr_dropout_t;

/*   bias      `channels` floats or NULL;   residual  or NULL;   y  may be x or residual itself
 * cr_dropout_backward:  dx = kept ? dy * scale : 0,  dbias = sum of dx (before rounding) over the points of a run and their positions; the
 * residual's gradient is dy.
 *   dx        may be dy itself; NULL: not wanted;   bounds, runs  as above;   dbias  runs x channels floats, or NULL: not wanted */
int cr_dropout_workspace_bytes(const cr_layer_shape_t *shape, const int64_t *bounds, int runs, size_t *backward_bytes);
int cr_dropout_forward(const cr_layer_shape_t *shape, const cr_layer_view_t *x, const float *bias, const cr_layer_view_t *residual,
                       const cr_dropout_t *dropout, const cr_layer_view_t *y, void *hip_stream);
int cr_dropout_backward(const cr_layer_shape_t *shape, const cr_layer_view_t *dy, const cr_dropout_t *dropout, const cr_layer_view_t *dx,
                        const int64_t *bounds, int runs, float *dbias, void *workspace, size_t workspace_bytes, void *hip_stream);

/* ---- softmax loss ------------------------------------------------------------------------------------------------------------------------
 * Row by row, with x the row's logits, t its target and w its weight:
 *     lse = log(sum_j exp(x_j)),   loss = w (lse - x_t),   dlogits_j = w (exp(x_j - lse) - [j = t])
 * and the loss of a batch is their sum.
 * The loss is formed from the logits' distances to the largest one, not from lse, so that it is as good beside large logits as beside small ones.
 *   logits    rows x classes of `dtype` (enum cr_xdtype), contiguous classes, row_stride elements apart
 *   targets   `rows` int64.  Negative: the row counts for nothing (loss and gradient 0, whatever its logits).  At least `classes`: no class;
 *             loss and gradient are NaN
 *   weights   `rows` floats or NULL: 1
 *   loss      `rows` floats;   lse  `rows` floats or NULL (also for rows without a target)
 *   dlogits   like logits, may be logits itself; NULL: not wanted
 * A logit of -infinity is a class that cannot be: its share and its gradient are 0 (its gradient -w where it is the target, the loss
 * infinite).  In a row of nothing else lse is -infinity, the loss +infinity (times w) and the gradient 0.  A row with a NaN or +infinity has
 * NaN in all outputs.
 * Limits: rows < 2^31, classes 1 to 2^28. */
int cr_softmax_loss_workspace_bytes(int64_t rows, int64_t classes, int dtype, size_t *bytes);
int cr_softmax_loss(int64_t rows, int64_t classes, int dtype, const void *logits, int64_t row_stride, const int64_t *targets,
                    const float *weights, float *loss, float *lse, void *dlogits, int64_t dlogits_row_stride, void *workspace,
                    size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CODEDREDUCE_LAYERS_H */

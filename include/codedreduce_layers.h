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
 * and for networks over tokens
 *
 *     cr_embedding_*      rows of a table looked up by tokens; the table's gradient, added up in the tokens' order
 *     cr_log_probs*       log probabilities of tokens, with the entropy and the most probable alternatives; the gradient of the first two
 *     cr_distill_loss     the loss against a teacher's alternatives, and its gradient
 *
 * A worker computes its own points with them, or one call serves all: gradients of parameters come once per RUN of consecutive points, so
 * that a slab gradient (codedreduce.h) is the sum of the runs between its rows, and what several workers hold in common is formed once.
 *
 * Conventions (beside those of codedreduce.h: plain C ABI, cr_status, the text of the last error on the calling thread from
 * cr_layers_last_error)
 *   - an activation is `points` data points of `positions` rows of `channels` values, channels last.  The channels of a row are
 *     contiguous; points and positions have strides, in elements, zero or more (inputs may be broadcast; rows of outputs must not
 *     overlap).  Storage is fp32 or bf16 (enum cr_xdtype); parameters (but tables of tokens), their gradients and statistics are fp32,
 *     contiguous.  Any alignment that the element has will do.
 *   - all pointers but the structs and `bounds` are device addresses.  The caller owns everything; nothing is allocated.
 *   - a call enqueues kernel launches on hip_stream (NULL = the default stream) of the current device and returns without waiting: no copy,
 *     no memset, so that it may be captured in a HIP graph.  A workspace is scratch of one call: calls that overlap in time must not share it.
 *   - an output may be the very tensor of an input (same address, same strides) where this is said; other overlaps are errors that are
 *     not looked for.
 *   - sums, statistics and exponentials are held in 32 bits or more; a result is rounded once, to its type.  Every sum has a fixed order:
 *     the same call on the same inputs gives the same bits.  Between calls that have a point among other points, a row of the losses and log
 *     probabilities, what dropout makes of a point and what is looked up for it are the same bits too; what a group norm makes of it may differ by rounding, since the order of its sums goes
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

/* ---- token embedding ---------------------------------------------------------------------------------------------------------------------
 *     y(n, p, :) = scale table[t(n, p), :]
 *   tokens        view of int64 without channels: t(n, p) is at dev + (n * point_stride + p * position_stride) elements, 8-byte aligned.
 *                 Negative: no token; y is 0 there.  At least `vocabulary`: no row of the table; y is NaN there
 *   table         vocabulary x channels of table_dtype (enum cr_xdtype), contiguous
 *   scale         a finite number
 *   shape         of y, dtype that of y.  Limits: points * positions < 2^31, vocabulary 1 to 2^28
 *
 * cr_embedding_backward:
 *     dtable[r][v][:] = scale sum dy(n, p, :)   over the points n of run r and the positions p with t(n, p) = v
 *   every row is written, rows of tokens that a run does not have with 0; where there is no token, or no row, dy has no influence, be it
 *   infinite or NaN.  A run's terms are added up in the order of their points and positions, in pieces that go by the call's shape and
 *   its tokens; the pieces' sums meet in 64 bits, in a fixed order.
 *   shape         of dy, dtype that of dy;   bounds, runs  as above
 *   dtable        runs x vocabulary x channels floats
 * cr_embedding_workspace_bytes: what the gradient needs (256-byte aligned): 16 bytes a position (17 of more than one run), two rows of floats for
 * each piece (16 to 256 positions), a byte for each row of up to 128 runs, 2 KB for each of up to 256 workgroups that sort; each of these up to 256 bytes more. */
int cr_embedding_workspace_bytes(const cr_layer_shape_t *shape, int64_t vocabulary, const int64_t *bounds, int runs, size_t *backward_bytes);
int cr_embedding_forward(const cr_layer_shape_t *shape, const cr_layer_view_t *tokens, const void *table, int table_dtype, int64_t vocabulary,
                         float scale, const cr_layer_view_t *y, void *hip_stream);
int cr_embedding_backward(const cr_layer_shape_t *shape, const cr_layer_view_t *dy, const cr_layer_view_t *tokens, int64_t vocabulary,
                          float scale, const int64_t *bounds, int runs, float *dtable, void *workspace, size_t workspace_bytes,
                          void *hip_stream);

/* ---- log probabilities -------------------------------------------------------------------------------------------------------------------
 * Row by row, with x the row's logits and t its token:
 *     c = max_j x_j,   L = log(sum_j exp(x_j - c)),   l_j = x_j - c - L,   logp = l_t,   entropy = -sum_j exp(l_j) l_j
 * and the `top` classes of the largest logits in descending order, of equal ones the lowest first, with their l_j.  (Where neither entropy nor alternatives are
 * wanted, cr_softmax_loss has logp as a loss of weight -1, and its gradient, with the weights -dlogp, in the same call.)
 *   logits        rows x classes of `dtype` (enum cr_xdtype), contiguous classes, row_stride elements apart
 *   tokens, logp  `rows` int64 and floats, or NULL (both).  Negative: no token, logp is 0.  At least `classes`: no class, logp is NaN
 *   entropy       `rows` floats or NULL
 *   top_index, top_logp   rows x top int64 and floats (top 0: NULL).  Places for which there is no class (a logit of -infinity is a class that
 *                 cannot be) have index -1 and -infinity
 *   largest, log_sum      `rows` floats each, c and L, what the gradient needs; NULL (both) where none will be asked for
 * A class that cannot be adds nothing to the entropy; as a token it has logp -infinity.  In a row of nothing else c, L and every logp are
 * -infinity, the entropy is 0.  A row with a NaN or +infinity has NaN in all outputs but the indices, which are -1, and a logp of no token.
 * Limits: rows < 2^31, classes 1 to 2^28, top 0 to 128.
 *
 * cr_log_probs_backward: from what the forward pass was given and left,
 *     dlogits_j = a ([j = t] - exp(l_j)) - b exp(l_j) (l_j + entropy),   a = dlogp (0 where there is no token), b = dentropy
 *   tokens, dlogp       or NULL (both): a = 0;   entropy, dentropy  `rows` floats each, or NULL (both): b = 0
 *   dlogits             like logits, may be logits itself
 * A class that cannot be has 0 (a where it is the token); a row of nothing else has 0, one with no such class as its token NaN. */
int cr_log_probs_workspace_bytes(int64_t rows, int64_t classes, int dtype, int top, size_t *bytes);
int cr_log_probs(int64_t rows, int64_t classes, int dtype, const void *logits, int64_t row_stride, const int64_t *tokens, float *logp,
                 float *entropy, int top, int64_t *top_index, float *top_logp, float *largest, float *log_sum, void *workspace,
                 size_t workspace_bytes, void *hip_stream);
int cr_log_probs_backward(int64_t rows, int64_t classes, int dtype, const void *logits, int64_t row_stride, const int64_t *tokens,
                          const float *largest, const float *log_sum, const float *entropy, const float *dlogp, const float *dentropy,
                          void *dlogits, int64_t dlogits_row_stride, void *hip_stream);

/* ---- distillation ------------------------------------------------------------------------------------------------------------------------
 * Row by row, with x the student's logits, j_i and z_i the classes and logits (or log probabilities: a constant for all of a row's changes
 * nothing) that a teacher gave, T the temperature and w the row's weight:
 *     q_i = exp(z_i / T) / sum_k exp(z_k / T),   p = softmax(x / T) over all classes
 *     loss = w T^2 sum_i q_i (log q_i - log p_(j_i)),   dlogits_j = w T (p_j - sum_(i: j_i = j) q_i)
 *   logits              rows x classes of `dtype` (enum cr_xdtype), contiguous classes, row_stride elements apart
 *   top                 entries of a row, 1 to 128
 *   top_index, top_logits   int64 and floats, `top` a row, rows top_row_stride elements apart (both).  An entry with a negative index or a logit
 *                       of -infinity is not there.  An index may come several times.  At least `classes`: no class; loss and gradient are NaN
 *   temperature         2^-40 to 2^40
 *   weights             `rows` floats or NULL: 1
 *   loss                `rows` floats
 *   dlogits             like logits, may be logits itself; NULL: not wanted
 * A row with no entry counts for nothing (loss and gradient 0, whatever its logits).  A logit of -infinity is a class that cannot be: its share
 * is 0, and if the teacher gives it a share the loss is infinite.  In a row of nothing else the loss is +infinity (times w) and the gradient 0.
 * A row with a NaN or +infinity among logits or entries has NaN in all outputs.
 * Limits: rows < 2^31, classes 1 to 2^28. */
int cr_distill_loss_workspace_bytes(int64_t rows, int64_t classes, int dtype, int top, size_t *bytes);
int cr_distill_loss(int64_t rows, int64_t classes, int dtype, const void *logits, int64_t row_stride, int top, const int64_t *top_index,
                    const float *top_logits, int64_t top_row_stride, float temperature, const float *weights, float *loss, void *dlogits,
                    int64_t dlogits_row_stride, void *workspace, size_t workspace_bytes, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* CODEDREDUCE_LAYERS_H */

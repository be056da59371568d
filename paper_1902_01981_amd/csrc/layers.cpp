// C-ABI boundary of the network layers: checks of arguments, and launches.
#include "codedreduce_layers.h"

#include <hip/hip_runtime_api.h>

#include <cmath>
#include <new>
#include <string>
#include <vector>

#include "layers.h"

namespace {

thread_local std::string g_last_error;

int fail(int code, const char *what, const char *why)
{
    try {
        g_last_error = std::string(what) + why;
    } catch (const std::bad_alloc &) {
        g_last_error.clear();
    }
    return code;
}

int launched(hipError_t e, const char *what) { return e == hipSuccess ? CR_OK : fail(CR_E_HIP, what, hipGetErrorString(e)); }

#define CR_TRY(call)                          \
    do {                                      \
        const int status_ = (call);           \
        if (status_ != CR_OK) return status_; \
    } while (0)

int read_shape(const cr_layer_shape_t *shape, cr::LayerShape *out)
{
    if (!shape) return fail(CR_E_INVAL, "shape", " is NULL");
    if (shape->points < 0 || shape->points >= int64_t(1) << 31) return fail(CR_E_INVAL, "points", " must be in 0 .. 2^31 - 1");
    if (shape->positions < 1 || shape->positions >= int64_t(1) << 31) return fail(CR_E_INVAL, "positions", " must be in 1 .. 2^31 - 1");
    if (shape->channels < 1 || shape->channels > int64_t(1) << 24) return fail(CR_E_INVAL, "channels", " must be in 1 .. 2^24");
    if (shape->dtype != CR_F32 && shape->dtype != CR_BF16) return fail(CR_E_INVAL, "dtype", " is unknown");
    *out = {shape->points, static_cast<int>(shape->positions), static_cast<int>(shape->channels), shape->dtype == CR_BF16};
    return CR_OK;
}

bool aligned(const void *p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }

int read_view(const cr_layer_view_t *view, const cr::LayerShape &shape, bool output, const char *name, cr::Rows *out)
{
    if (!view || !view->dev) return fail(CR_E_INVAL, name, " is required");
    if (!aligned(view->dev, shape.bf16 ? 2 : 4)) return fail(CR_E_INVAL, name, " is not aligned to its elements");
    // strides of dimensions of one entry mean nothing
    int64_t point = shape.points > 1 ? view->point_stride : 0, position = shape.positions > 1 ? view->position_stride : 0;
    constexpr int64_t kMost = int64_t(1) << 40;
    if (point < 0 || position < 0 || point > kMost || position > kMost) return fail(CR_E_INVAL, name, ": strides must be in 0 .. 2^40");
    // the kernels' offsets, and the sums below, have 64 bits; strides and counts can each be what they may and their products more
    if (static_cast<__int128>(shape.points) * point + static_cast<__int128>(shape.positions) * position + shape.channels > int64_t(1) << 60)
        return fail(CR_E_INVAL, name, " reaches past any address");
    if (output) {                                        // rows beside each other, the dimension of the smaller stride inside the other
        const bool points_outside = shape.points == 1 || (shape.positions == 1 ? true : point >= position);
        const int64_t inner = points_outside ? position : point, inner_count = points_outside ? shape.positions : shape.points;
        const int64_t outer = points_outside ? point : position, outer_count = points_outside ? shape.points : shape.positions;
        if (inner_count > 1 && inner < shape.channels) return fail(CR_E_INVAL, name, ": its rows overlap");
        const int64_t block = inner_count > 1 ? (inner_count - 1) * inner + shape.channels : shape.channels;
        if (outer_count > 1 && outer < block) return fail(CR_E_INVAL, name, ": its rows overlap");
    }
    *out = {view->dev, point, position};
    return CR_OK;
}

int check_floats(const void *p, bool required, const char *name)
{
    if (!p) return required ? fail(CR_E_INVAL, name, " is required") : CR_OK;
    return aligned(p, 4) ? CR_OK : fail(CR_E_INVAL, name, " is not 4-byte aligned");
}

int check_groups(const cr::LayerShape &shape, int groups)
{
    if (groups < 1 || shape.channels % groups != 0) return fail(CR_E_INVAL, "groups", " must divide the channels");
    return CR_OK;
}

int check_activation(int activation)
{
    return activation >= CR_ACT_NONE && activation <= CR_ACT_SILU ? CR_OK : fail(CR_E_INVAL, "activation", " is unknown");
}

int check_pieces(const cr::LayerShape &shape, int groups)
{
    return cr::norm_backward_numbered(shape, groups) ? CR_OK : fail(CR_E_INVAL, "points, positions", " are too many together for a gradient");
}

// The runs' bounds as they are, or one run of all points in `whole`.
int read_bounds(const cr::LayerShape &shape, const int64_t *bounds, int runs, int64_t (&whole)[2], const int64_t **out)
{
    if (!bounds) {
        if (runs != 1) return fail(CR_E_INVAL, "bounds", " are required for more runs than one");
        whole[0] = 0;
        whole[1] = shape.points;
        *out = whole;
        return CR_OK;
    }
    if (runs < 1) return fail(CR_E_INVAL, "runs", " must be positive");
    if (bounds[0] != 0 || bounds[runs] != shape.points) return fail(CR_E_INVAL, "bounds", " must go from 0 to the number of points");
    for (int r = 0; r < runs; ++r)
        if (bounds[r] > bounds[r + 1]) return fail(CR_E_INVAL, "bounds", " must ascend");
    *out = bounds;
    return CR_OK;
}

int check_workspace(const void *workspace, size_t have, size_t need)
{
    if (need == 0) return CR_OK;
    if (!workspace) return fail(CR_E_INVAL, "workspace", " is required");
    if (!aligned(workspace, 256)) return fail(CR_E_INVAL, "workspace", " is not 256-byte aligned");
    return have >= need ? CR_OK : fail(CR_E_INVAL, "workspace", " is too small");
}

int read_mask(const cr_dropout_t *d, cr::Mask *out)
{
    if (!d) return fail(CR_E_INVAL, "dropout", " is NULL");
    if (!(d->rate >= 0.0 && d->rate < 1.0)) return fail(CR_E_INVAL, "rate", " must be at least 0 and less than 1");
    const uint32_t least = static_cast<uint32_t>(std::floor(d->rate * 65536.0 + 0.5));
    if (least > 65535) return fail(CR_E_INVAL, "rate", " is nearer to 1 than draws of 16 bits can tell apart");
    if (!aligned(d->draw_dev, 8)) return fail(CR_E_INVAL, "draw_dev", " is not 8-byte aligned");
    if (!aligned(d->point_dev, 8)) return fail(CR_E_INVAL, "point_dev", " is not 8-byte aligned");
    if (d->point_dev && d->first_point != 0) return fail(CR_E_INVAL, "first_point", " must be 0 where point_dev lists the points");
    *out = {least, static_cast<float>(65536.0 / (65536.0 - least)), d->seed + (d->draw + 1) * 0x9E3779B97F4A7C15ull, d->draw_dev, d->first_point, d->point_dev};
    return CR_OK;
}

}  // namespace

extern "C" {

const char *cr_layers_last_error(void) { return g_last_error.c_str(); }

int cr_group_norm_workspace_bytes(const cr_layer_shape_t *shape, int groups, const int64_t *bounds, int runs, size_t *forward_bytes, size_t *backward_bytes)
{
    cr::LayerShape s;
    int64_t whole[2];
    const int64_t *b = nullptr;
    CR_TRY(read_shape(shape, &s));
    CR_TRY(check_groups(s, groups));
    CR_TRY(read_bounds(s, bounds, runs, whole, &b));
    CR_TRY(check_pieces(s, groups));
    if (!forward_bytes || !backward_bytes) return fail(CR_E_INVAL, "forward_bytes, backward_bytes", " are required");
    *forward_bytes = cr::norm_forward_bytes(s, groups);
    *backward_bytes = cr::norm_backward_bytes(s, groups, b, runs);
    return CR_OK;
}

int cr_group_norm_forward(const cr_layer_shape_t *shape, const cr_layer_view_t *x, const float *gamma, const float *beta, int groups, float eps,
                          int activation, const cr_layer_view_t *y, float *mean, float *rstd, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    cr::NormArgs a = {};
    CR_TRY(read_shape(shape, &a.shape));
    CR_TRY(check_groups(a.shape, groups));
    CR_TRY(check_activation(activation));
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(CR_E_INVAL, "eps", " must be a number of at least 0");
    CR_TRY(check_floats(gamma, false, "gamma"));
    CR_TRY(check_floats(beta, false, "beta"));
    CR_TRY(check_floats(mean, false, "mean"));
    CR_TRY(check_floats(rstd, false, "rstd"));
    if (!mean != !rstd) return fail(CR_E_INVAL, "mean, rstd", " come together or not at all");
    if (a.shape.points == 0) return CR_OK;
    CR_TRY(read_view(x, a.shape, false, "x", &a.x));
    CR_TRY(read_view(y, a.shape, true, "y", &a.y));
    CR_TRY(check_workspace(workspace, workspace_bytes, cr::norm_forward_bytes(a.shape, groups)));
    a.gamma = gamma; a.beta = beta; a.groups = groups; a.eps = eps; a.activation = activation; a.mean = mean; a.rstd = rstd;
    return launched(cr::launch_norm_forward(a, workspace, static_cast<hipStream_t>(hip_stream)), "cr_group_norm_forward: ");
}

int cr_group_norm_backward(const cr_layer_shape_t *shape, const cr_layer_view_t *dy, const cr_layer_view_t *x, const float *mean, const float *rstd,
                           const float *gamma, const float *beta, int groups, int activation, const int64_t *bounds, int runs,
                           const cr_layer_view_t *dx, float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    cr::NormGradArgs a = {};
    int64_t whole[2];
    CR_TRY(read_shape(shape, &a.shape));
    CR_TRY(check_groups(a.shape, groups));
    CR_TRY(check_activation(activation));
    CR_TRY(read_bounds(a.shape, bounds, runs, whole, &a.bounds));
    CR_TRY(check_pieces(a.shape, groups));
    CR_TRY(check_floats(gamma, false, "gamma"));
    CR_TRY(check_floats(beta, false, "beta"));
    CR_TRY(check_floats(dgamma, false, "dgamma"));
    CR_TRY(check_floats(dbeta, false, "dbeta"));
    if (a.shape.points > 0) {
        CR_TRY(check_floats(mean, true, "mean"));
        CR_TRY(check_floats(rstd, true, "rstd"));
        CR_TRY(read_view(dy, a.shape, false, "dy", &a.dy));
        CR_TRY(read_view(x, a.shape, false, "x", &a.x));
        if (dx && dx->dev) CR_TRY(read_view(dx, a.shape, true, "dx", &a.dx));
        CR_TRY(check_workspace(workspace, workspace_bytes, cr::norm_backward_bytes(a.shape, groups, a.bounds, runs)));
    }
    a.mean = mean; a.rstd = rstd; a.gamma = gamma; a.beta = beta; a.groups = groups; a.activation = activation; a.runs = runs;
    a.dgamma = dgamma; a.dbeta = dbeta;
    return launched(cr::launch_norm_backward(a, workspace, static_cast<hipStream_t>(hip_stream)), "cr_group_norm_backward: ");
}

int cr_dropout_workspace_bytes(const cr_layer_shape_t *shape, const int64_t *bounds, int runs, size_t *backward_bytes)
{
    cr::LayerShape s;
    int64_t whole[2];
    const int64_t *b = nullptr;
    CR_TRY(read_shape(shape, &s));
    CR_TRY(read_bounds(s, bounds, runs, whole, &b));
    if (!backward_bytes) return fail(CR_E_INVAL, "backward_bytes", " is required");
    *backward_bytes = cr::dropout_backward_bytes(s, b, runs);
    return CR_OK;
}

int cr_dropout_forward(const cr_layer_shape_t *shape, const cr_layer_view_t *x, const float *bias, const cr_layer_view_t *residual,
                       const cr_dropout_t *dropout, const cr_layer_view_t *y, void *hip_stream)
{
    cr::DropoutArgs a = {};
    CR_TRY(read_shape(shape, &a.shape));
    CR_TRY(read_mask(dropout, &a.mask));
    CR_TRY(check_floats(bias, false, "bias"));
    if (a.shape.points == 0) return CR_OK;
    CR_TRY(read_view(x, a.shape, false, "x", &a.x));
    if (residual && residual->dev) CR_TRY(read_view(residual, a.shape, false, "residual", &a.residual));
    CR_TRY(read_view(y, a.shape, true, "y", &a.y));
    a.bias = bias;
    return launched(cr::launch_dropout_forward(a, static_cast<hipStream_t>(hip_stream)), "cr_dropout_forward: ");
}

int cr_dropout_backward(const cr_layer_shape_t *shape, const cr_layer_view_t *dy, const cr_dropout_t *dropout, const cr_layer_view_t *dx,
                        const int64_t *bounds, int runs, float *dbias, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    cr::DropoutGradArgs a = {};
    int64_t whole[2];
    CR_TRY(read_shape(shape, &a.shape));
    CR_TRY(read_mask(dropout, &a.mask));
    CR_TRY(read_bounds(a.shape, bounds, runs, whole, &a.bounds));
    CR_TRY(check_floats(dbias, false, "dbias"));
    if (a.shape.points > 0) {
        CR_TRY(read_view(dy, a.shape, false, "dy", &a.dy));
        if (dx && dx->dev) CR_TRY(read_view(dx, a.shape, true, "dx", &a.dx));
        if (dbias) CR_TRY(check_workspace(workspace, workspace_bytes, cr::dropout_backward_bytes(a.shape, a.bounds, runs)));
    }
    a.runs = runs; a.dbias = dbias;
    return launched(cr::launch_dropout_backward(a, workspace, static_cast<hipStream_t>(hip_stream)), "cr_dropout_backward: ");
}

int cr_softmax_loss_workspace_bytes(int64_t rows, int64_t classes, int dtype, size_t *bytes)
{
    if (rows < 0 || rows >= int64_t(1) << 31) return fail(CR_E_INVAL, "rows", " must be in 0 .. 2^31 - 1");
    if (classes < 1 || classes > int64_t(1) << 28) return fail(CR_E_INVAL, "classes", " must be in 1 .. 2^28");
    if (dtype != CR_F32 && dtype != CR_BF16) return fail(CR_E_INVAL, "dtype", " is unknown");
    if (!bytes) return fail(CR_E_INVAL, "bytes", " is required");
    *bytes = cr::loss_bytes(rows, classes, dtype == CR_BF16);
    return CR_OK;
}

int cr_softmax_loss(int64_t rows, int64_t classes, int dtype, const void *logits, int64_t row_stride, const int64_t *targets, const float *weights,
                    float *loss, float *lse, void *dlogits, int64_t dlogits_row_stride, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    size_t need = 0;
    CR_TRY(cr_softmax_loss_workspace_bytes(rows, classes, dtype, &need));
    CR_TRY(check_floats(weights, false, "weights"));
    CR_TRY(check_floats(lse, false, "lse"));
    if (rows == 0) return CR_OK;
    const cr::LayerShape shape = {rows, 1, static_cast<int>(classes), dtype == CR_BF16};
    const cr_layer_view_t x = {const_cast<void *>(logits), row_stride, 0}, dx = {dlogits, dlogits_row_stride, 0};
    cr::Rows in, out = {};
    CR_TRY(read_view(&x, shape, false, "logits", &in));
    if (dlogits) CR_TRY(read_view(&dx, shape, true, "dlogits", &out));
    if (!targets || !aligned(targets, 8)) return fail(CR_E_INVAL, "targets", " are required, 8-byte aligned");
    CR_TRY(check_floats(loss, true, "loss"));
    CR_TRY(check_workspace(workspace, workspace_bytes, need));
    const cr::LossArgs a = {rows, static_cast<int>(classes), shape.bf16, logits, in.point_stride, targets, weights, loss, lse, dlogits, out.point_stride};
    return launched(cr::launch_loss(a, workspace, static_cast<hipStream_t>(hip_stream)), "cr_softmax_loss: ");
}

}  // extern "C"

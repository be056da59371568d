// Launchers of the network layers (include/codedreduce_layers.h) on gfx950.  Host code sees only plain launch functions.
#pragma once
#include <hip/hip_runtime_api.h>

#include <cstddef>
#include <cstdint>

namespace cr {

// Rows of `channels` contiguous elements, `positions` of them per data point.
struct Rows {
    void *p;
    int64_t point_stride, position_stride;               // elements
};
struct LayerShape {
    int64_t points;
    int positions, channels;
    bool bf16;
};

struct NormArgs {
    LayerShape shape;
    Rows x, y;
    const float *gamma, *beta;                           // or null: 1 and 0
    int groups;
    float eps;
    int activation;
    float *mean, *rstd;                                  // or null
};
struct NormGradArgs {
    LayerShape shape;
    Rows dy, x, dx;                                      // dx.p may be null
    const float *mean, *rstd, *gamma, *beta;
    int groups, activation;
    const int64_t *bounds;                               // host
    int runs;
    float *dgamma, *dbeta;                               // or null
};
size_t norm_forward_bytes(const LayerShape &shape, int groups);
bool norm_backward_numbered(const LayerShape &shape, int groups);       // whether 32 bits number the pieces that leave sums
size_t norm_backward_bytes(const LayerShape &shape, int groups, const int64_t *bounds, int runs);
hipError_t launch_norm_forward(const NormArgs &a, void *workspace, hipStream_t stream);
hipError_t launch_norm_backward(const NormGradArgs &a, void *workspace, hipStream_t stream);

struct Mask {
    uint32_t least;                                      // a draw of 16 bits is kept from here on
    float scale;
    uint64_t key_state;                                  // the key is the mixing function of this,
    const uint64_t *draw_dev;                            // with golden * *draw_dev added before, or null
    int64_t first_point;
    const int64_t *point_dev;                            // or null
};
struct DropoutArgs {
    LayerShape shape;
    Rows x, residual, y;                                 // residual.p may be null
    const float *bias;                                   // or null
    Mask mask;
};
struct DropoutGradArgs {
    LayerShape shape;
    Rows dy, dx;                                         // dx.p may be null
    Mask mask;
    const int64_t *bounds;                               // host
    int runs;
    float *dbias;                                        // or null
};
size_t dropout_backward_bytes(const LayerShape &shape, const int64_t *bounds, int runs);
hipError_t launch_dropout_forward(const DropoutArgs &a, hipStream_t stream);
hipError_t launch_dropout_backward(const DropoutGradArgs &a, void *workspace, hipStream_t stream);

struct LossArgs {
    int64_t rows;
    int classes;
    bool bf16;
    const void *logits;
    int64_t row_stride;
    const int64_t *targets;
    const float *weights;                                // or null
    float *loss, *lse;                                   // lse may be null
    void *dlogits;                                       // or null
    int64_t dlogits_row_stride;
};
size_t loss_bytes(int64_t rows, int64_t classes, bool bf16);
hipError_t launch_loss(const LossArgs &a, void *workspace, hipStream_t stream);

}  // namespace cr

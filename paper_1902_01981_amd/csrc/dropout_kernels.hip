// Bias, dropout and residual, the mask drawn from a counter, for gfx950.
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ uint64_t mask_key(const Mask &m) { return splitmix_mix(m.key_state + (m.draw_dev ? kGolden * *m.draw_dev : 0)); }
// the word with the draws of channels [4 word, 4 word + 4) of a row
__device__ __forceinline__ uint64_t mask_word(const Mask &m, uint64_t key, int64_t n, int positions, int p, int words, int word)
{
    const uint64_t point = m.point_dev ? m.point_dev[n] : m.first_point + n;
    return splitmix_mix(key + ((point * positions + p) * words + word + 1) * kGolden);
}
__device__ __forceinline__ bool kept(uint64_t word, int field, uint32_t least) { return (static_cast<uint32_t>(word >> (16 * field)) & 0xffffu) >= least; }

// a thread per word of the mask
template <bool BF16> __global__ void __launch_bounds__(kThreads) dropout_forward_kernel(DropoutArgs a)
{
    using E = Element<BF16>;
    using T = typename E::type;
    const int words = (a.shape.channels + 3) / 4;
    const uint64_t key = mask_key(a.mask);
    const int64_t total = a.shape.points * a.shape.positions * words;
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kThreads) {
        const int word = static_cast<int>(i % words), p = static_cast<int>(i / words % a.shape.positions);
        const int64_t n = i / words / a.shape.positions;
        const uint64_t z = mask_word(a.mask, key, n, a.shape.positions, p, words, word);
        for (int f = 0; f < 4 && 4 * word + f < a.shape.channels; ++f) {
            const int c = 4 * word + f;
            float v = 0.f;
            if (kept(z, f, a.mask.least))
                v = (E::get(static_cast<const T *>(a.x.p) + n * a.x.point_stride + p * a.x.position_stride + c) + (a.bias ? a.bias[c] : 0.f)) * a.mask.scale;
            if (a.residual.p) v += E::get(static_cast<const T *>(a.residual.p) + n * a.residual.point_stride + p * a.residual.position_stride + c);
            E::put(static_cast<T *>(a.y.p) + n * a.y.point_stride + p * a.y.position_stride + c, v);
        }
    }
}

template <bool BF16> __global__ void __launch_bounds__(kThreads) dropout_dx_kernel(DropoutGradArgs a)
{
    using E = Element<BF16>;
    using T = typename E::type;
    const int words = (a.shape.channels + 3) / 4;
    const uint64_t key = mask_key(a.mask);
    const int64_t total = a.shape.points * a.shape.positions * words;
    for (int64_t i = int64_t(blockIdx.x) * kThreads + threadIdx.x; i < total; i += int64_t(gridDim.x) * kThreads) {
        const int word = static_cast<int>(i % words), p = static_cast<int>(i / words % a.shape.positions);
        const int64_t n = i / words / a.shape.positions;
        const uint64_t z = mask_word(a.mask, key, n, a.shape.positions, p, words, word);
        for (int f = 0; f < 4 && 4 * word + f < a.shape.channels; ++f) {
            const int c = 4 * word + f;
            const float v = kept(z, f, a.mask.least) ? E::get(static_cast<const T *>(a.dy.p) + n * a.dy.point_stride + p * a.dy.position_stride + c) * a.mask.scale : 0.f;
            E::put(static_cast<T *>(a.dx.p) + n * a.dx.point_stride + p * a.dx.position_stride + c, v);
        }
    }
}

// a workgroup per channel and run; before dx, which may replace dy
template <bool BF16> __global__ void __launch_bounds__(kThreads) dropout_bias_kernel(DropoutGradArgs a, RunTable table, int64_t first_run)
{
    using E = Element<BF16>;
    using T = typename E::type;
    __shared__ float lds[kThreads / 64];
    const int r = blockIdx.y, words = (a.shape.channels + 3) / 4;
    for (int c = blockIdx.x; c < a.shape.channels; c += gridDim.x) {
    const uint64_t key = mask_key(a.mask);
    const int64_t begin = int64_t(table.first[r]) * a.shape.positions, end = int64_t(table.first[r + 1]) * a.shape.positions;
    float sum = 0.f;
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
        const int64_t n = i / a.shape.positions;
        const int p = static_cast<int>(i % a.shape.positions);
        if (kept(mask_word(a.mask, key, n, a.shape.positions, p, words, c / 4), c % 4, a.mask.least))
            sum += E::get(static_cast<const T *>(a.dy.p) + n * a.dy.point_stride + p * a.dy.position_stride + c) * a.mask.scale;
    }
    sum = block_total<kThreads>(sum, lds);
    if (threadIdx.x == 0) a.dbias[(first_run + r) * a.shape.channels + c] = sum;
    }
}

unsigned grid_for(const LayerShape &s)
{
    const int64_t words = s.points * s.positions * ((s.channels + 3) / 4);
    return static_cast<unsigned>(std::min<int64_t>((words + kThreads - 1) / kThreads, 256 * 32));
}

}  // namespace

size_t dropout_backward_bytes(const LayerShape &, const int64_t *, int) { return 0; }

hipError_t launch_dropout_forward(const DropoutArgs &a, hipStream_t stream)
{
    if (a.shape.points == 0) return hipSuccess;
    (a.shape.bf16 ? dropout_forward_kernel<true> : dropout_forward_kernel<false>)<<<grid_for(a.shape), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_dropout_backward(const DropoutGradArgs &a, void *, hipStream_t stream)
{
    if (a.dbias) {
        for (int r = 0; r < a.runs; r += RunTable::kRuns) {
            RunTable table;
            table.runs = std::min(RunTable::kRuns, a.runs - r);
            for (int i = 0; i <= table.runs; ++i) table.first[i] = static_cast<int>(a.bounds[r + i]);
            const dim3 grid(std::min(a.shape.channels, 1 << 15), table.runs);
            (a.shape.bf16 ? dropout_bias_kernel<true> : dropout_bias_kernel<false>)<<<grid, kThreads, 0, stream>>>(a, table, r);
        }
    }
    if (a.dx.p && a.shape.points > 0)
        (a.shape.bf16 ? dropout_dx_kernel<true> : dropout_dx_kernel<false>)<<<grid_for(a.shape), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace cr

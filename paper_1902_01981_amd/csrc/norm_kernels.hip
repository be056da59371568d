// Group norm with an activation, channels last, for gfx950.
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256;

// act(z) and act'(z)
__device__ __forceinline__ float act(int kind, float z)
{
    if (kind == 1) return z < 0.f ? 0.f : z;
    if (kind == 2) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
    return z;
}
__device__ __forceinline__ float act_slope(int kind, float z)
{
    if (kind == 1) return z > 0.f ? 1.f : 0.f;
    if (kind == 2) {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
        return s * (1.f + z * (1.f - s));
    }
    return 1.f;
}

// a workgroup per group of a point
template <bool BF16> __global__ void __launch_bounds__(kThreads) norm_forward_kernel(NormArgs a)
{
    using E = Element<BF16>;
    using T = typename E::type;
    __shared__ float lds[kThreads / 64];
    const int cg = a.shape.channels / a.groups;
    for (int64_t item = blockIdx.x; item < a.shape.points * a.groups; item += gridDim.x) {
    const int64_t n = item / a.groups;
    const int g = static_cast<int>(item % a.groups);
    const int64_t count = int64_t(a.shape.positions) * cg;
    const T *x = static_cast<const T *>(a.x.p) + n * a.x.point_stride + g * cg;
    T *y = static_cast<T *>(a.y.p) + n * a.y.point_stride + g * cg;
    float sum = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += kThreads) sum += E::get(x + i / cg * a.x.position_stride + i % cg);
    const float mean = block_total<kThreads>(sum, lds) / static_cast<float>(count);
    sum = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += kThreads) {
        const float t = E::get(x + i / cg * a.x.position_stride + i % cg) - mean;
        sum += t * t;
    }
    const float rstd = 1.f / sqrtf(block_total<kThreads>(sum, lds) / static_cast<float>(count) + a.eps);
    for (int64_t i = threadIdx.x; i < count; i += kThreads) {
        const int c = static_cast<int>(i % cg);
        const float h = (E::get(x + i / cg * a.x.position_stride + c) - mean) * rstd;
        const float z = (a.gamma ? a.gamma[g * cg + c] : 1.f) * h + (a.beta ? a.beta[g * cg + c] : 0.f);
        E::put(y + i / cg * a.y.position_stride + c, act(a.activation, z));
    }
    if (a.mean && threadIdx.x == 0) {
        a.mean[n * a.groups + g] = mean;
        a.rstd[n * a.groups + g] = rstd;
    }
    }
}

// dx: a workgroup per group of a point
template <bool BF16> __global__ void __launch_bounds__(kThreads) norm_dx_kernel(NormGradArgs a)
{
    using E = Element<BF16>;
    using T = typename E::type;
    __shared__ float lds[kThreads / 64];
    const int cg = a.shape.channels / a.groups;
    for (int64_t item = blockIdx.x; item < a.shape.points * a.groups; item += gridDim.x) {
    const int64_t n = item / a.groups;
    const int g = static_cast<int>(item % a.groups);
    const int64_t count = int64_t(a.shape.positions) * cg;
    const T *x = static_cast<const T *>(a.x.p) + n * a.x.point_stride + g * cg;
    const T *dy = static_cast<const T *>(a.dy.p) + n * a.dy.point_stride + g * cg;
    T *dx = static_cast<T *>(a.dx.p) + n * a.dx.point_stride + g * cg;
    const float mean = a.mean[n * a.groups + g], rstd = a.rstd[n * a.groups + g];
    auto terms = [&](int64_t i, float &h) {
        const int c = static_cast<int>(i % cg);
        const float gamma = a.gamma ? a.gamma[g * cg + c] : 1.f;
        h = (E::get(x + i / cg * a.x.position_stride + c) - mean) * rstd;
        return gamma * E::get(dy + i / cg * a.dy.position_stride + c) * act_slope(a.activation, gamma * h + (a.beta ? a.beta[g * cg + c] : 0.f));
    };
    float A = 0.f, B = 0.f;
    for (int64_t i = threadIdx.x; i < count; i += kThreads) {
        float h;
        const float t = terms(i, h);
        A += t;
        B += t * h;
    }
    A = block_total<kThreads>(A, lds) / static_cast<float>(count);
    B = block_total<kThreads>(B, lds) / static_cast<float>(count);
    for (int64_t i = threadIdx.x; i < count; i += kThreads) {
        float h;
        const float t = terms(i, h);
        E::put(dx + i / cg * a.dx.position_stride + i % cg, rstd * (t - A - h * B));
    }
    }
}

// dgamma and dbeta: a workgroup per channel and run; before dx, which may replace dy or x
template <bool BF16> __global__ void __launch_bounds__(kThreads) norm_parameters_kernel(NormGradArgs a, RunTable table, int64_t first_run)
{
    using E = Element<BF16>;
    using T = typename E::type;
    __shared__ float lds[kThreads / 64];
    const int r = blockIdx.y;
    for (int c = blockIdx.x; c < a.shape.channels; c += gridDim.x) {
    const int g = c / (a.shape.channels / a.groups);
    const float gamma = a.gamma ? a.gamma[c] : 1.f, beta = a.beta ? a.beta[c] : 0.f;
    const int64_t begin = int64_t(table.first[r]) * a.shape.positions, end = int64_t(table.first[r + 1]) * a.shape.positions;
    float s1 = 0.f, s2 = 0.f;
    for (int64_t i = begin + threadIdx.x; i < end; i += kThreads) {
        const int64_t n = i / a.shape.positions, p = i % a.shape.positions;
        const float h = (E::get(static_cast<const T *>(a.x.p) + n * a.x.point_stride + p * a.x.position_stride + c) - a.mean[n * a.groups + g]) * a.rstd[n * a.groups + g];
        const float dz = E::get(static_cast<const T *>(a.dy.p) + n * a.dy.point_stride + p * a.dy.position_stride + c) * act_slope(a.activation, gamma * h + beta);
        s1 += dz;
        s2 += dz * h;
    }
    s1 = block_total<kThreads>(s1, lds);
    s2 = block_total<kThreads>(s2, lds);
    if (threadIdx.x == 0) {
        if (a.dbeta) a.dbeta[(first_run + r) * a.shape.channels + c] = s1;
        if (a.dgamma) a.dgamma[(first_run + r) * a.shape.channels + c] = s2;
    }
    }
}

}  // namespace

size_t norm_forward_bytes(const LayerShape &, int) { return 0; }
size_t norm_backward_bytes(const LayerShape &, int, const int64_t *, int) { return 0; }

hipError_t launch_norm_forward(const NormArgs &a, void *, hipStream_t stream)
{
    if (a.shape.points == 0) return hipSuccess;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.shape.points * a.groups, 1 << 20)));
    (a.shape.bf16 ? norm_forward_kernel<true> : norm_forward_kernel<false>)<<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormGradArgs &a, void *, hipStream_t stream)
{
    if (a.dgamma || a.dbeta) {
        for (int r = 0; r < a.runs; r += RunTable::kRuns) {
            RunTable table;
            table.runs = std::min(RunTable::kRuns, a.runs - r);
            for (int i = 0; i <= table.runs; ++i) table.first[i] = static_cast<int>(a.bounds[r + i]);
            const dim3 grid(std::min(a.shape.channels, 1 << 15), table.runs);
            (a.shape.bf16 ? norm_parameters_kernel<true> : norm_parameters_kernel<false>)<<<grid, kThreads, 0, stream>>>(a, table, r);
        }
    }
    if (a.dx.p && a.shape.points > 0) {
        const dim3 grid(static_cast<unsigned>(std::min<int64_t>(a.shape.points * a.groups, 1 << 20)));
        (a.shape.bf16 ? norm_dx_kernel<true> : norm_dx_kernel<false>)<<<grid, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace cr

// Softmax loss and its gradient, for gfx950.
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256;

template <int T> __device__ __forceinline__ float block_most(float v, float *lds)
{
    for (int o = 1; o < 64; o *= 2) v = fmaxf(v, __shfl_xor(v, o, 64));
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    for (int w = 0; w < T / 64; ++w) v = fmaxf(v, lds[w]);
    __syncthreads();
    return v;
}

// a workgroup per row
template <bool BF16> __global__ void __launch_bounds__(kThreads) loss_kernel(LossArgs a)
{
    using E = Element<BF16>;
    using T = typename E::type;
    __shared__ float lds[kThreads / 64];
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
    float top = -__builtin_inff();
    for (int j = threadIdx.x; j < a.classes; j += kThreads) top = fmaxf(top, E::get(x + j));
    top = block_most<kThreads>(top, lds);
    const float from = top == -__builtin_inff() ? 0.f : top;         // a row of no class, or of NaN
    float sum = 0.f;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) sum += expf(E::get(x + j) - from);
    sum = block_total<kThreads>(sum, lds);
    const float lse = from + logf(sum);
    const int64_t t = a.targets[row];
    const float w = a.weights ? a.weights[row] : 1.f;
    const float xt = t >= 0 && t < a.classes ? E::get(x + t) : __builtin_nanf("");
    __syncthreads();
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = lse;
        a.loss[row] = t < 0 ? 0.f : w * (sum == 0.f && t < a.classes ? __builtin_inff() : lse - xt);
    }
    if (!a.dlogits) continue;
    T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
    const float share = w / sum;
    for (int j = threadIdx.x; j < a.classes; j += kThreads) {
        const float p = share * expf(E::get(x + j) - from);
        E::put(dx + j, t < 0 ? 0.f : t >= a.classes ? __builtin_nanf("") : sum == 0.f ? 0.f : j == t ? p - w : p);
    }
    }
}

}  // namespace

size_t loss_bytes(int64_t, int64_t, bool) { return 0; }

hipError_t launch_loss(const LossArgs &a, void *, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    (a.bf16 ? loss_kernel<true> : loss_kernel<false>)<<<static_cast<unsigned>(std::min<int64_t>(a.rows, 1 << 20)), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace cr

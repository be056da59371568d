// Softmax over the classes of a row, as sums about a reference: what the kernels of the losses and of the log probabilities share on the device.
#pragma once
#include "layers_device.h"

namespace cr {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float infinity() { return __builtin_inff(); }
// e^v for v <= 0, the distance from the largest logit: off by 1.25 |v| + 2 units of 2^-24 of itself (the product's rounding, 0.23 of one that the constant is off by, and the
// hardware's exponential), by less than 3 of them of the largest share, whose v is 0.  Results below 2^-126 are 0.
// unit: log2(e) / T, for e^(v / T); that is one rounding more, 2.25 |v| / T + 2 units.
__device__ __forceinline__ float exp_fast(float v, float unit = kLog2e) { return __builtin_amdgcn_exp2f(v * unit); }

// c = reference, S = sum; c is finite unless the part has nothing but -infinity (S = 0 then) or a +infinity (S is NaN then)
struct Softmax {
    float c = -__builtin_inff(), S = 0.f;
};
// a reference that can be subtracted: 0 stands in where nothing has been seen but -infinity (or NaN, which the sum then shows)
__device__ __forceinline__ float usable(float c) { return c == -infinity() ? 0.f : c; }

// element offset of chunk q of a row: the last one is moved back to end with the row
template <int VEC> __device__ __forceinline__ int chunk_at(int q, int nq, int classes) { return q < nq - 1 ? q * VEC : classes - VEC; }

// Adds VEC elements, if they count.
template <int VEC> __device__ __forceinline__ void take(Softmax &s, const float (&x)[VEC], bool count, float unit = kLog2e)
{
    float most = x[0];
#pragma unroll
    for (int v = 1; v < VEC; ++v) most = fmaxf(most, x[v]);
    const float c = count ? fmaxf(s.c, most) : s.c, from = usable(c);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum += exp_fast(x[v] - from, unit);
    s.S = s.S * exp_fast(s.c - from, unit) + (count ? sum : 0.f);
    s.c = c;
}
template <int LANES> __device__ __forceinline__ void join_lanes(Softmax &s, float unit = kLog2e)
{
    const float c = lanes_most<LANES>(s.c);
    s.S = lanes_total<LANES>(s.S * exp_fast(s.c - usable(c), unit));
    s.c = c;
}

}  // namespace

}  // namespace cr

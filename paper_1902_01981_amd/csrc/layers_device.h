// What the kernels of the network layers share on the device.
#pragma once
#include <hip/hip_runtime.h>

#include "layers.h"

namespace cr {

template <bool BF16> struct Element;
template <> struct Element<false> {
    using type = float;
    static __device__ __forceinline__ float get(const float *p) { return *p; }
    static __device__ __forceinline__ void put(float *p, float v) { *p = v; }
};
template <> struct Element<true> {
    using type = uint16_t;
    static __device__ __forceinline__ float get(const uint16_t *p) { return __uint_as_float(static_cast<uint32_t>(*p) << 16); }
    static __device__ __forceinline__ void put(uint16_t *p, float v)      // to nearest, ties to even; a NaN stays one
    {
        __bf16 b = static_cast<__bf16>(v);
        __builtin_memcpy(p, &b, 2);
    }
};

__device__ __forceinline__ float wave_total(float v)
{
#pragma unroll
    for (int o = 1; o < 64; o *= 2) v += __shfl_xor(v, o, 64);
    return v;
}
// The sum over a workgroup of T threads, for every thread; lds holds T / 64 floats and may be used again at once.
template <int T> __device__ __forceinline__ float block_total(float v, float *lds)
{
    v = wave_total(v);
    if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) v += lds[w];
    __syncthreads();
    return v;
}

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;      // the increment of the splitmix64 generator
__host__ __device__ __forceinline__ uint64_t splitmix_mix(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

}  // namespace cr

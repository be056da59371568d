// What the kernels of the network layers share on the device.
#pragma once
#include <hip/hip_runtime.h>

#include <type_traits>

#include "layers.h"

namespace cr {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));       // the same in memory, on any boundary that the elements have
typedef unsigned u4h __attribute__((ext_vector_type(4), aligned(2)));
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
typedef float f2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)        // to nearest, ties to even; a NaN stays one
{
    const f2 v = {lo, hi};
    const bf2 b = __builtin_convertvector(v, bf2);
    uint32_t u;
    __builtin_memcpy(&u, &b, 4);
    return u;
}

// One element of a row, and VEC of them on any boundary that the element has (gfx950 serves unaligned vector accesses).  load_once, store_once:
// with the non-temporal hint, for what nobody asks for again soon.
template <bool BF16, int VEC> struct Chunk;
template <> struct Chunk<false, 1> {
    using element = float;
    using raw = float;
    static __device__ __forceinline__ raw load(const element *p) { return *p; }
    static __device__ __forceinline__ raw load_once(const element *p) { return __builtin_nontemporal_load(p); }
    static __device__ __forceinline__ void store(element *p, raw r) { *p = r; }
    static __device__ __forceinline__ void store_once(element *p, raw r) { __builtin_nontemporal_store(r, p); }
    static __device__ __forceinline__ void widen(raw r, float (&v)[1]) { v[0] = r; }
    static __device__ __forceinline__ raw narrow(const float (&v)[1]) { return v[0]; }
};
template <> struct Chunk<true, 1> {
    using element = uint16_t;
    using raw = uint16_t;
    static __device__ __forceinline__ raw load(const element *p) { return *p; }
    static __device__ __forceinline__ raw load_once(const element *p) { return __builtin_nontemporal_load(p); }
    static __device__ __forceinline__ void store(element *p, raw r) { *p = r; }
    static __device__ __forceinline__ void store_once(element *p, raw r) { __builtin_nontemporal_store(r, p); }
    static __device__ __forceinline__ void widen(raw r, float (&v)[1]) { v[0] = __uint_as_float(static_cast<uint32_t>(r) << 16); }
    static __device__ __forceinline__ raw narrow(const float (&v)[1]) { return static_cast<raw>(pack_bf16(v[0], 0.f)); }
};
template <> struct Chunk<false, 4> {
    using element = float;
    using raw = f4;
    using memory = f4u;
    static __device__ __forceinline__ raw load(const element *p) { return *reinterpret_cast<const memory *>(p); }
    static __device__ __forceinline__ raw load_once(const element *p) { return __builtin_nontemporal_load(reinterpret_cast<const memory *>(p)); }
    static __device__ __forceinline__ void store(element *p, raw r) { *reinterpret_cast<memory *>(p) = r; }
    static __device__ __forceinline__ void store_once(element *p, raw r) { __builtin_nontemporal_store(r, reinterpret_cast<memory *>(p)); }
    static __device__ __forceinline__ void widen(const raw &r, float (&v)[4]) { v[0] = r.x; v[1] = r.y; v[2] = r.z; v[3] = r.w; }
    static __device__ __forceinline__ raw narrow(const float (&v)[4]) { return raw{v[0], v[1], v[2], v[3]}; }
};
template <> struct Chunk<true, 8> {
    using element = uint16_t;
    using raw = u4;
    using memory = u4h;
    static __device__ __forceinline__ raw load(const element *p) { return *reinterpret_cast<const memory *>(p); }
    static __device__ __forceinline__ raw load_once(const element *p) { return __builtin_nontemporal_load(reinterpret_cast<const memory *>(p)); }
    static __device__ __forceinline__ void store(element *p, raw r) { *reinterpret_cast<memory *>(p) = r; }
    static __device__ __forceinline__ void store_once(element *p, raw r) { __builtin_nontemporal_store(r, reinterpret_cast<memory *>(p)); }
    static __device__ __forceinline__ void widen(const raw &r, float (&v)[8])
    {
        v[0] = __uint_as_float(r.x << 16); v[1] = __uint_as_float(r.x & 0xffff0000u);
        v[2] = __uint_as_float(r.y << 16); v[3] = __uint_as_float(r.y & 0xffff0000u);
        v[4] = __uint_as_float(r.z << 16); v[5] = __uint_as_float(r.z & 0xffff0000u);
        v[6] = __uint_as_float(r.w << 16); v[7] = __uint_as_float(r.w & 0xffff0000u);
    }
    static __device__ __forceinline__ raw narrow(const float (&v)[8])
    {
        return raw{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
    }
};

template <bool BF16> struct Element {
    using type = typename Chunk<BF16, 1>::element;
    static __device__ __forceinline__ float get(const type *p)
    {
        float v[1];
        Chunk<BF16, 1>::widen(*p, v);
        return v[0];
    }
    static __device__ __forceinline__ void put(type *p, float f)
    {
        const float v[1] = {f};
        *p = Chunk<BF16, 1>::narrow(v);
    }
};

// v of the lane that the cross-lane pattern CTRL pairs this one with inside its row of 16 lanes
template <int CTRL> __device__ __forceinline__ float dpp(float v) { return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, false)); }
// v of the lane 16 or 32 lanes away: rows of 16 lanes exchanged between two copies of v
template <typename F> __device__ __forceinline__ float fold_16(float v, F f)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
template <typename F> __device__ __forceinline__ float fold_32(float v, F f)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return f(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
// Folds f over each LANES neighbouring lanes (a power of two), for every lane: quad swaps, the mirrored half-row and row (as good as an exchange once
// the lanes of a half agree), then exchanges between rows.
template <int LANES, typename F> __device__ __forceinline__ float fold_lanes(float v, F f)
{
    if constexpr (LANES >= 2) v = f(v, dpp<0xB1>(v));    // quad_perm [1,0,3,2]
    if constexpr (LANES >= 4) v = f(v, dpp<0x4E>(v));    // quad_perm [2,3,0,1]
    if constexpr (LANES >= 8) v = f(v, dpp<0x141>(v));   // row_half_mirror
    if constexpr (LANES >= 16) v = f(v, dpp<0x140>(v));  // row_mirror
    if constexpr (LANES >= 32) v = fold_16(v, f);
    if constexpr (LANES == 64) v = fold_32(v, f);
    return v;
}
// The sum over the lanes of a wavefront that are a multiple of `across` apart (a power of two up to 32), for every lane.
__device__ __forceinline__ float total_every(float v, int across)
{
    auto add = [](float a, float b) { return a + b; };
    if (across <= 8) v += dpp<0x128>(v);                 // row_ror:8
    if (across <= 4) v += dpp<0x124>(v);                 // row_ror:4
    if (across <= 2) v += dpp<0x122>(v);                 // row_ror:2
    if (across <= 1) v += dpp<0x121>(v);                 // row_ror:1
    if (across <= 16) v = fold_16(v, add);
    return fold_32(v, add);
}
template <int LANES> __device__ __forceinline__ float lanes_total(float v)
{
    return fold_lanes<LANES>(v, [](float a, float b) { return a + b; });
}
template <int LANES> __device__ __forceinline__ float lanes_most(float v)
{
    return fold_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); });
}
// A pointer that is the same for all lanes, kept from being taken apart: what is added to it afterwards is the lane's offset of one access, not part
// of an address per access that is held in registers throughout a loop.
template <typename P> __device__ __forceinline__ P *scalar(P *p)
{
    uintptr_t at = reinterpret_cast<uintptr_t>(p);
    asm("" : "+s"(at));
    return (P *)reinterpret_cast<__attribute__((address_space(1))) P *>(at);          // an address in global memory
}
// Says that a loaded value is needed from here on, so that its load is not moved behind a branch to where it is first used: several loads asked for together
// stay together.
template <typename R> __device__ __forceinline__ void hold(R &raw) { asm volatile("" : "+v"(raw)); }
// A value at an address that is the same for all lanes, through the scalar cache: waiting for it is not waiting for vector loads.  For memory that nobody
// writes while the kernel runs: the compiler takes it for constant.
template <typename P> __device__ __forceinline__ P scalar_load(const P *p)
{
    return *reinterpret_cast<const __attribute__((address_space(4))) P *>(reinterpret_cast<uintptr_t>(p));
}

// n / d for n < 2^31, by a product
struct Divisor {
    uint32_t d, magic, shift;
    explicit Divisor(uint32_t divisor) : d(divisor), shift(0)
    {
        while ((uint64_t(1) << shift) < d) ++shift;
        magic = static_cast<uint32_t>(((uint64_t(1) << 32) * ((uint64_t(1) << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, magic) + n) >> shift; }
};

constexpr uint64_t kGolden = 0x9E3779B97F4A7C15ull;      // the increment of the splitmix64 generator
__host__ __device__ __forceinline__ uint64_t splitmix_mix(uint64_t z)
{
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return z ^ (z >> 31);
}

}  // namespace cr

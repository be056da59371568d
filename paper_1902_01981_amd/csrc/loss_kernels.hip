// Softmax loss and its gradient, for gfx950.
//
// With c the largest x_j:  S = sum_j exp(x_j - c),  lse = c + log S,  loss = w (c - x_t + log S),  share of class j = exp(x_j - c) / S.  Sums about two
// references meet by S exp(c - c'), so one pass over a row does, with a running maximum.  (One multiply-add, x log2(e) - c log2(e), in place of a subtraction and a
// product would be lost on rows of the type's lowest value, whose product is infinite.)
//
//   loss_narrow_kernel   2 to 32 lanes per row
//   loss_rows_kernel     a row in the registers of a wavefront or a workgroup, read once
//   loss_slices_kernel, loss_join_kernel   rows wider than that: a row cut into slices, read twice
//
// With the gradient, bf16, the reads and writes bound it: 32 768 x 4 096 82 us, 6.5 TB/s; 4 099 x 50 008 165 us, 5.0 TB/s; 8 192 x 131 072 817 us, 5.3 TB/s,
// and 913 us, 4.7 TB/s, of 131 071 classes, whose rows begin anywhere.  fp32, 4 099 x 50 008: 330 us, 5.0 TB/s.  Without it 32 768 x 4 096 bf16 43 us, 6.2 TB/s.
// Narrow rows: 100 000 x 100 bf16 16 us, 2.5 TB/s.  3 x 131 072 fp32 13 us, the launches.  Rows wider than the registers: 8 192 x 152 064 bf16 1.55 ms, 4 096 x
// 128 000 fp32 1.26 ms, both 5.0 TB/s of what moves, 3.3 of what has to.
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
__device__ __forceinline__ float infinity() { return __builtin_inff(); }
// e^v for v <= 0, the distance from the largest logit: off by |v| + 2 units of 2^-24 of itself, by less than 3 of them of the largest share, whose v is 0.
// Results below 2^-126 are 0.
__device__ __forceinline__ float exp_fast(float v) { return __builtin_amdgcn_exp2f(v * kLog2e); }

// c = reference, S = sum; c is finite unless the part has nothing but -infinity (S = 0 then) or a +infinity (S is NaN then)
struct Softmax {
    float c = -__builtin_inff(), S = 0.f;
};
// a reference that can be subtracted: 0 stands in where nothing has been seen but -infinity (or NaN, which the sum then shows)
__device__ __forceinline__ float usable(float c) { return c == -infinity() ? 0.f : c; }

// element offset of chunk q of a row: the last one is moved back to end with the row
template <int VEC> __device__ __forceinline__ int chunk_at(int q, int nq, int classes) { return q < nq - 1 ? q * VEC : classes - VEC; }

// Adds VEC elements, if they count.
template <int VEC> __device__ __forceinline__ void take(Softmax &s, const float (&x)[VEC], bool count)
{
    float most = x[0];
#pragma unroll
    for (int v = 1; v < VEC; ++v) most = fmaxf(most, x[v]);
    const float c = count ? fmaxf(s.c, most) : s.c, from = usable(c);
    float sum = 0.f;
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum += exp_fast(x[v] - from);
    s.S = s.S * exp_fast(s.c - from) + (count ? sum : 0.f);
    s.c = c;
}
template <int LANES> __device__ __forceinline__ void join_lanes(Softmax &s)
{
    const float c = lanes_most<LANES>(s.c);
    s.S = lanes_total<LANES>(s.S * exp_fast(s.c - usable(c)));
    s.c = c;
}

// what the rows' outputs are made of
struct RowTarget {
    int64_t t;
    float w, xt;
};
// SCALAR: the row is the same for the whole wavefront
template <bool SCALAR> __device__ __forceinline__ void read_target(RowTarget &r, const LossArgs &a, int64_t row)
{
    r.t = SCALAR ? scalar_load(a.targets + row) : a.targets[row];
    r.w = !a.weights ? 1.f : SCALAR ? scalar_load(a.weights + row) : a.weights[row];
}
// SCALAR only where no gradient is written: it may be written over the logits, and what is read through the scalar cache has to stay as it is while the
// kernel runs, so that the compiler may read it late, or twice.
template <bool BF16, bool SCALAR> __device__ __forceinline__ void read_logit(RowTarget &r, const LossArgs &a, int64_t row)
{
    using E = Element<BF16>;
    const int64_t t = r.t >= 0 && r.t < a.classes ? r.t : 0;
    const auto *at = static_cast<const typename E::type *>(a.logits) + row * a.row_stride + t;
    float xt;
    if constexpr (SCALAR && BF16) {                      // scalar loads have four bytes: those on whose boundary the two lie
        const uintptr_t byte = reinterpret_cast<uintptr_t>(at);
        const uint32_t both = scalar_load(reinterpret_cast<const uint32_t *>(byte & ~uintptr_t(3)));
        xt = __uint_as_float(byte & 2 ? both & 0xffff0000u : both << 16);
    } else if constexpr (SCALAR) {
        xt = scalar_load(at);
    } else {
        xt = E::get(at);
    }
    r.xt = xt;
}
__device__ __forceinline__ void write_row(const LossArgs &a, int64_t row, const RowTarget &r, const Softmax &s)
{
    const float c = usable(s.c), log2_S = __builtin_amdgcn_logf(s.S);             // the hardware's logarithm is that to base 2
    if (a.lse) a.lse[row] = fmaf(kLn2, log2_S, c);
    // Not lse - x_t: lse is rounded at the logits' size, and a loss may be far smaller.  Losses of 8e-4 under logits of 3 000: that is off by 7 to 20 %, this by
    // at most 7e-4 of itself, S's own rounding beside 1.
    a.loss[row] = r.t < 0 ? 0.f : r.w * (r.t >= a.classes ? __builtin_nanf("") : s.S == 0.f ? infinity() : fmaf(kLn2, log2_S, c - r.xt));
}
// The gradient is one value for the whole row where there is no target, no such class, or no class at all.
__device__ __forceinline__ bool one_value(const LossArgs &a, const RowTarget &r, const Softmax &s, float &value)
{
    value = r.t >= a.classes ? __builtin_nanf("") : 0.f;
    return r.t < 0 || r.t >= a.classes || s.S == 0.f;
}
// the weighted shares of a chunk's classes
template <bool BF16, int VEC> __device__ __forceinline__ void shares(float (&x)[VEC], const typename Chunk<BF16, VEC>::raw &raw, float from, float factor)
{
    Chunk<BF16, VEC>::widen(raw, x);
#pragma unroll
    for (int v = 0; v < VEC; ++v) x[v] = exp_fast(x[v] - from) * factor;
}

// Rows narrower than 64 chunks: TS lanes of a wavefront per row, a whole chunk each, and the last lane also what is left of the row, as a chunk moved
// back to end with it (elements that it shares with its neighbour count there, and both store the same bits).
template <bool BF16, int VEC, int TS, bool GRAD> __global__ void __launch_bounds__(256) loss_narrow_kernel(LossArgs a)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int lane = threadIdx.x % TS, whole = a.classes / VEC, left = a.classes % VEC;
    const int q = std::min(lane, whole - 1);
    const bool has_left = VEC > 1 && left > 0 && lane == TS - 1;
    for (int64_t row = int64_t(blockIdx.x) * (256 / TS) + threadIdx.x / TS; row < a.rows; row += int64_t(gridDim.x) * (256 / TS)) {
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        typename C::raw raw = C::load(x + q * VEC), last = raw;
        if (has_left) last = C::load(x + (a.classes - VEC));
        RowTarget target;
        read_target<false>(target, a, row);
        read_logit<BF16, false>(target, a, row);
        float v[VEC], u[VEC];
        Softmax s;
        C::widen(raw, v);
        take<VEC>(s, v, lane < whole);
        if (has_left) {
            C::widen(last, u);
#pragma unroll
            for (int i = 0; i < VEC; ++i) u[i] = i < VEC - left ? -infinity() : u[i];
            take<VEC>(s, u, true);
        }
        join_lanes<TS>(s);
        if (lane == 0) write_row(a, row, target, s);
        if constexpr (GRAD) {
            T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
            float value;
            const bool flat = one_value(a, target, s, value);
            const float from = usable(s.c), factor = target.w / s.S, at_target = exp_fast(target.xt - from) * factor - target.w;
            auto form = [&](const typename C::raw &in, int at) {
                shares<BF16, VEC>(v, in, from, factor);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = flat ? value : at + i == target.t ? at_target : v[i];
                C::store(dx + at, C::narrow(v));
            };
            form(raw, q * VEC);
            if (has_left) form(last, a.classes - VEC);
        }
    }
}

// Wider rows: a wavefront per row (BLOCK = 256: four of them), or a workgroup.  A thread holds K chunks of the row in registers as they were read; they
// are added to the running sum as they arrive, and as soon as a chunk's gradient is stored its place takes the chunk of the team's next row, so that
// reads go on while gradients are formed and written.  For that to be so, a wait for one chunk must not be a wait for all: there is no branch around a
// load or a store of a chunk, and a step ends with the sum over the row that it has asked for, so that its waits are counted from its own loads and
// stores.  That took 8 192 x 131 072 bf16, a row per workgroup, from 1 006 us to 801 (817 with loads that suit rows of odd lengths, below).
// `lanes` threads have chunks, lanes = ceil(whole / K), so that all but the last of a thread lie in the row; whoever has no chunk there forms the last
// whole one again, with the same bits, and does not count it.  What is behind the chunks has a lane per element in the last wavefront.  (Chunks on
// 16-byte boundaries, whatever the row starts on, are faster where rows have odd lengths, 8 192 x 131 071 bf16 351 us against 430 without and 913
// against 917 with the gradient, but then a row's bits depend on where it lies, and two holders of a point would not form the same.)
template <bool BF16, int K, bool WAVE, bool GRAD> __global__ void __launch_bounds__(WAVE ? 256 : 1024) loss_rows_kernel(LossArgs a, int lanes)
{
    constexpr int VEC = BF16 ? 8 : 4;
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    constexpr unsigned kBytes = VEC * sizeof(T);
    __shared__ float lds[2][2][WAVE ? 1 : 16];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int lane = WAVE ? threadIdx.x % 64 : threadIdx.x, tl = std::min(lane, lanes - 1);
    const bool edges = WAVE || wave == static_cast<int>(blockDim.x / 64) - 1;
    const int64_t stride = int64_t(gridDim.x) * (WAVE ? 4 : 1);
    int64_t row = WAVE ? int64_t(blockIdx.x) * 4 + wave : blockIdx.x;
    if (row >= a.rows) return;                           // whole teams

    const int whole = a.classes / VEC, left = a.classes % VEC;
    auto row_at = [&](int64_t of) { return static_cast<const T *>(a.logits) + std::min(of, a.rows - 1) * a.row_stride; };
    // the element behind the chunks that is this lane's, if it has one
    const int edge_at = std::min<int>(whole * VEC + threadIdx.x % 64, a.classes - 1);
    const bool has_edge = edges && static_cast<int>(threadIdx.x % 64) < left;
    typename C::raw raw[K];
    typename Chunk<BF16, 1>::raw edge;
    const unsigned lane_byte = tl * kBytes;
    const unsigned last_byte = std::min(tl + (K - 1) * lanes, whole - 1) * kBytes;
    auto chunk = [&](auto *x, int k) {                   // a scalar address and the lane's offset
        using P = std::remove_pointer_t<decltype(x)>;
        auto *bytes = reinterpret_cast<std::conditional_t<std::is_const_v<P>, const char, char> *>(x);
        if (k < K - 1) return reinterpret_cast<P *>(scalar(bytes + static_cast<unsigned>(k * lanes) * kBytes) + lane_byte);
        return reinterpret_cast<P *>(scalar(bytes) + last_byte);
    };
    // What is read and replaced by its gradient soon may stay in the caches, where rows that do not start on a line share lines: 8 192 x 131 071 bf16
    // 917 us, past the caches 960.  What is only read passes them: 429 and 447.  (A wavefront per row: 32 768 x 4 096 81 us, read from the caches 105.)
    auto fetch = [&](int k, const T *x) { raw[k] = WAVE || !GRAD ? C::load_once(chunk(x, k)) : C::load(chunk(x, k)); };
    auto fetch_edge = [&](const T *x) { edge = Chunk<BF16, 1>::load(x + edge_at); };
    Softmax s;
    auto add = [&](int k) {
        float x[VEC];
        C::widen(raw[k], x);
        take<VEC>(s, x, k < K - 1 || lane + k * lanes < whole);
    };
    auto add_edge = [&] {
        if (lane >= lanes) s = Softmax();                // had the chunks of the last lane that has any
        if (!edges) return;
        float x[1];
        Chunk<BF16, 1>::widen(edge, x);
        take<1>(s, x, has_edge);
    };
    int turn = 0;
    auto join = [&] {
        join_lanes<64>(s);
        if constexpr (!WAVE) {
            auto &meet = lds[turn];                      // two in turn: one barrier a step
            turn ^= 1;
            if (threadIdx.x % 64 == 0) {
                meet[0][wave] = s.c;
                meet[1][wave] = s.S;
            }
            __syncthreads();
            s = Softmax();
            if (threadIdx.x % 16 < blockDim.x / 64) {
                s.c = meet[0][threadIdx.x % 16];
                s.S = meet[1][threadIdx.x % 16];
            }
            join_lanes<16>(s);
        }
        s.c = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(s.c)));       // scalars: branches on them are not divergent
        s.S = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(s.S)));
    };
    // the gradient of a row, each chunk making place for one of the row at x
    auto form = [&](int64_t of, const RowTarget &now, auto more, const T *x) {
        T *dx = static_cast<T *>(a.dlogits) + of * a.dlogits_row_stride;
        float value;
        const bool flat = one_value(a, now, s, value);
        const float from = usable(s.c), factor = now.w / s.S;
        const float at_target = exp_fast(now.xt - from) * factor - now.w;
        if (has_edge) {
            float v[1];
            shares<BF16, 1>(v, edge, from, factor);
            Element<BF16>::put(dx + edge_at, flat ? value : edge_at == now.t ? at_target : v[0]);
        }
        float v[VEC];
        if (flat) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = value;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                C::store(chunk(dx, k), C::narrow(v));
                if (more()) fetch(k, x);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                shares<BF16, VEC>(v, raw[k], from, factor);
                C::store(chunk(dx, k), C::narrow(v));
                if (more()) fetch(k, x);
            }
        }
        if (more()) fetch_edge(x);
        // the target's own entry follows the chunk it is in, from every thread that stored that chunk
        const int c_t = static_cast<int>(now.t / VEC);
        const bool mine = c_t == whole - 1 ? tl + (K - 1) * lanes >= c_t : tl == c_t % lanes;
        if (!flat && c_t < whole && mine) Element<BF16>::put(dx + now.t, at_target);
    };

    const T *x = row_at(row);
#pragma unroll
    for (int k = 0; k < K; ++k) fetch(k, x);
    fetch_edge(x);
    // the target of a row is read a step before its logit, and that a step before it is needed
    RowTarget now, next, after;
    read_target<true>(now, a, row);
    read_target<true>(next, a, std::min(row + stride, a.rows - 1));
    read_logit<BF16, !GRAD>(now, a, row);
    if constexpr (GRAD) {
#pragma unroll
        for (int k = 0; k < K; ++k) add(k);
        add_edge();
        for (; row + stride < a.rows; row += stride) {
            join();
            if (lane == 0) write_row(a, row, now, s);
            read_target<true>(after, a, std::min(row + 2 * stride, a.rows - 1));
            read_logit<BF16, !GRAD>(next, a, row + stride);
            form(row, now, std::true_type(), row_at(row + stride));
            now = next;
            next = after;
            s = Softmax();
#pragma unroll
            for (int k = 0; k < K; ++k) add(k);
            add_edge();
        }
        join();
        if (lane == 0) write_row(a, row, now, s);
        form(row, now, std::false_type(), x);
    } else {
        for (; row < a.rows; row += stride) {
            x = row_at(row + stride);                    // past the last row: that row once more, from the caches
            read_target<true>(after, a, std::min(row + 2 * stride, a.rows - 1));
            read_logit<BF16, !GRAD>(next, a, std::min(row + stride, a.rows - 1));
            s = Softmax();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                add(k);
                fetch(k, x);
            }
            add_edge();
            fetch_edge(x);
            join();
            if (lane == 0) write_row(a, row, now, s);
            now = next;
            next = after;
        }
    }
}

// ---- a row in slices ------------------------------------------------------------------------------------------------------------
constexpr int kSliceThreads = 256, kSliceChunks = 4;     // chunks that a thread has in flight

// Adds up a slice of a row: chunks [begin, end).
template <bool BF16, int VEC> __device__ __forceinline__ Softmax add_slice(const LossArgs &a, const typename Chunk<BF16, VEC>::element *x, int nq, int begin, int end)
{
    using C = Chunk<BF16, VEC>;
    const int doubled = nq * VEC - a.classes;
    Softmax s;
    for (int q0 = begin + threadIdx.x; q0 < end; q0 += kSliceThreads * kSliceChunks) {
        typename C::raw raw[kSliceChunks];
#pragma unroll
        for (int k = 0; k < kSliceChunks; ++k) raw[k] = C::load(x + chunk_at<VEC>(std::min(q0 + k * kSliceThreads, end - 1), nq, a.classes));
#pragma unroll
        for (int k = 0; k < kSliceChunks; ++k) {
            const int q = q0 + k * kSliceThreads;
            float v[VEC];
            C::widen(raw[k], v);
            if (q == nq - 1) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = i < doubled ? -infinity() : v[i];
            }
            take<VEC>(s, v, q < end);
        }
    }
    return s;
}
__device__ __forceinline__ void join_block(Softmax &s, float (&lds)[2][kSliceThreads / 64])
{
    join_lanes<64>(s);
    if (threadIdx.x % 64 == 0) {
        lds[0][threadIdx.x / 64] = s.c;
        lds[1][threadIdx.x / 64] = s.S;
    }
    __syncthreads();
    s.c = lds[0][threadIdx.x % (kSliceThreads / 64)];
    s.S = lds[1][threadIdx.x % (kSliceThreads / 64)];
    join_lanes<kSliceThreads / 64>(s);
}

// parts[row of the batch][slice] = (c, S).  The targets' logits go to at_targets[row]: in the next kernel the gradient may have replaced them.
template <bool BF16, int VEC> __global__ void __launch_bounds__(kSliceThreads) loss_slices_kernel(LossArgs a, int slice, f2 *parts, float *at_targets)
{
    using T = typename Chunk<BF16, VEC>::element;
    __shared__ float lds[2][kSliceThreads / 64];
    const int nq = (a.classes + VEC - 1) / VEC, begin = blockIdx.x * slice;
    Softmax s = add_slice<BF16, VEC>(a, static_cast<const T *>(a.logits) + blockIdx.y * a.row_stride, nq, begin, std::min(begin + slice, nq));
    join_block(s, lds);
    if (threadIdx.x == 0) parts[int64_t(blockIdx.y) * gridDim.x + blockIdx.x] = f2{s.c, s.S};
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        RowTarget target;
        read_target<false>(target, a, blockIdx.y);
        read_logit<BF16, false>(target, a, blockIdx.y);
        at_targets[blockIdx.y] = target.xt;
    }
}
// Joins a row's slices, every workgroup for itself, and forms the gradient of its own slice.
template <bool BF16, int VEC, bool GRAD> __global__ void __launch_bounds__(kSliceThreads) loss_join_kernel(LossArgs a, int slice, int slices, const f2 *parts, const float *at_targets)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float lds[2][kSliceThreads / 64];
    const int64_t row = blockIdx.y;
    RowTarget target;
    read_target<true>(target, a, row);
    target.xt = scalar_load(at_targets + row);
    Softmax s;
    for (int i = threadIdx.x; i < slices; i += kSliceThreads) {
        const f2 p = parts[row * slices + i];
        const float c = fmaxf(s.c, p.x), from = usable(c);
        s.S = s.S * exp_fast(s.c - from) + p.y * exp_fast(p.x - from);
        s.c = c;
    }
    join_block(s, lds);
    if (blockIdx.x == 0 && threadIdx.x == 0) write_row(a, row, target, s);
    if constexpr (GRAD) {
        const int nq = (a.classes + VEC - 1) / VEC, begin = blockIdx.x * slice, end = std::min(begin + slice, nq);
        const int doubled = nq * VEC - a.classes;
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
        float value;
        const bool flat = one_value(a, target, s, value);
        const float from = usable(s.c), factor = target.w / s.S;
        const float at_target = exp_fast(target.xt - from) * factor - target.w;
        for (int q0 = begin + threadIdx.x; q0 < end; q0 += kSliceThreads * kSliceChunks) {
            typename C::raw raw[kSliceChunks];
#pragma unroll
            for (int k = 0; k < kSliceChunks; ++k) raw[k] = C::load(x + chunk_at<VEC>(std::min(q0 + k * kSliceThreads, end - 1), nq, a.classes));
#pragma unroll
            for (int k = 0; k < kSliceChunks; ++k) {
                const int q = q0 + k * kSliceThreads, at = chunk_at<VEC>(q, nq, a.classes);
                if (q >= end) break;
                float v[VEC];
                shares<BF16, VEC>(v, raw[k], from, factor);
                if (flat) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) v[i] = value;
                }
                if (q < nq - 1 || doubled == 0) {
                    C::store(dx + at, C::narrow(v));
                } else {                                 // what the neighbour has too may have been read after it was replaced: it is the neighbour's
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (i >= doubled) Element<BF16>::put(dx + at + i, v[i]);
                }
                if (!flat && target.t >= at + (q < nq - 1 ? 0 : doubled) && target.t < at + VEC) Element<BF16>::put(dx + target.t, at_target);
            }
        }
    }
}

struct LossPlan {
    bool slices;
    int team, k;                 // threads that share a row, chunks per thread
    int slice, per_row;          // chunks of a slice, slices of a row
    int64_t batch;               // rows per pair of launches
};

constexpr int kMostTeam = 1024, kMostChunks = 16;

LossPlan plan_loss(int64_t rows, int64_t classes, bool bf16)
{
    LossPlan p = {};
    const int vec = classes < (bf16 ? 8 : 4) ? 1 : bf16 ? 8 : 4;
    const int64_t whole = classes / vec;
    p.slices = whole > kMostTeam * kMostChunks;
    if (!p.slices) {
        p.k = 1;
        p.team = 2;
        while (p.team < 64 && p.team < whole) p.team *= 2;
        if (whole <= 64 * 8) {
            while (int64_t(p.team) * p.k < whole) ++p.k;
            return p;
        }
        p.k = whole <= kMostTeam * 8 ? 8 : 16;
        p.team = static_cast<int>((whole + p.k * 64 - 1) / (p.k * 64)) * 64;
        return p;
    }
    constexpr int kStep = kSliceThreads * kSliceChunks;
    int64_t slice = kStep;
    while (whole > slice * 512) slice *= 2;
    p.slice = static_cast<int>(slice);
    p.per_row = static_cast<int>(((classes + vec - 1) / vec + slice - 1) / slice);
    p.batch = std::max<int64_t>(1, std::min<int64_t>(rows, (int64_t(64) << 20) / (classes * (bf16 ? 2 : 4))));
    return p;
}

constexpr int kUnits = 256;      // compute units, for the number of workgroups that stay

template <bool BF16, int VEC, int TS> void launch_narrow(const LossArgs &a, hipStream_t stream)
{
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>((a.rows * TS + 255) / 256, 1 << 20));
    (a.dlogits ? loss_narrow_kernel<BF16, VEC, TS, true> : loss_narrow_kernel<BF16, VEC, TS, false>)<<<groups, 256, 0, stream>>>(a);
}
template <bool BF16, int K, bool WAVE> void launch_rows(const LossArgs &a, int threads, hipStream_t stream)
{
    // as many workgroups as the registers of the compute units take at once
    constexpr int kWaves = K >= 16 ? 20 : K >= 8 ? 24 : 28;
    const int lanes = (a.classes / (BF16 ? 8 : 4) + K - 1) / K, teams = WAVE ? 4 : 1;
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>((a.rows + teams - 1) / teams, kUnits * (kWaves / (threads / 64))));
    (a.dlogits ? loss_rows_kernel<BF16, K, WAVE, true> : loss_rows_kernel<BF16, K, WAVE, false>)<<<groups, threads, 0, stream>>>(a, lanes);
}

template <bool BF16> hipError_t launch(const LossArgs &a, const LossPlan &p, void *workspace, hipStream_t stream)
{
    constexpr int VEC = BF16 ? 8 : 4;
    if (p.slices) {
        f2 *parts = static_cast<f2 *>(workspace);
        float *at_targets = reinterpret_cast<float *>(parts + p.batch * p.per_row);
        constexpr int64_t e = BF16 ? 2 : 4;
        for (int64_t row = 0; row < a.rows; row += p.batch) {
            LossArgs b = a;
            b.rows = std::min(p.batch, a.rows - row);
            b.logits = static_cast<const char *>(a.logits) + row * a.row_stride * e;
            b.targets += row;
            if (b.weights) b.weights += row;
            b.loss += row;
            if (b.lse) b.lse += row;
            if (b.dlogits) b.dlogits = static_cast<char *>(a.dlogits) + row * a.dlogits_row_stride * e;
            const dim3 grid(p.per_row, static_cast<unsigned>(b.rows));
            loss_slices_kernel<BF16, VEC><<<grid, kSliceThreads, 0, stream>>>(b, p.slice, parts, at_targets);
            if (b.dlogits) loss_join_kernel<BF16, VEC, true><<<grid, kSliceThreads, 0, stream>>>(b, p.slice, p.per_row, parts, at_targets);
            else loss_join_kernel<BF16, VEC, false><<<dim3(1, grid.y), kSliceThreads, 0, stream>>>(b, p.slice, p.per_row, parts, at_targets);
        }
        return hipGetLastError();
    }
    if (a.classes < VEC) {
        if (p.team == 2) launch_narrow<BF16, 1, 2>(a, stream);
        else if (p.team == 4) launch_narrow<BF16, 1, 4>(a, stream);
        else launch_narrow<BF16, 1, 8>(a, stream);
        return hipGetLastError();
    }
    switch (p.team) {
    case 2: launch_narrow<BF16, VEC, 2>(a, stream); break;
    case 4: launch_narrow<BF16, VEC, 4>(a, stream); break;
    case 8: launch_narrow<BF16, VEC, 8>(a, stream); break;
    case 16: launch_narrow<BF16, VEC, 16>(a, stream); break;
    case 32: launch_narrow<BF16, VEC, 32>(a, stream); break;
    case 64:
        switch (p.k) {
        case 1: launch_rows<BF16, 1, true>(a, 256, stream); break;
        case 2: launch_rows<BF16, 2, true>(a, 256, stream); break;
        case 3: launch_rows<BF16, 3, true>(a, 256, stream); break;
        case 4: launch_rows<BF16, 4, true>(a, 256, stream); break;
        case 5: launch_rows<BF16, 5, true>(a, 256, stream); break;
        case 6: launch_rows<BF16, 6, true>(a, 256, stream); break;
        case 7: launch_rows<BF16, 7, true>(a, 256, stream); break;
        default: launch_rows<BF16, 8, true>(a, 256, stream); break;
        }
        break;
    default:
        if (p.k == 8) launch_rows<BF16, 8, false>(a, p.team, stream);
        else launch_rows<BF16, 16, false>(a, p.team, stream);
    }
    return hipGetLastError();
}

}  // namespace

size_t loss_bytes(int64_t rows, int64_t classes, bool bf16)
{
    if (rows == 0) return 0;
    const LossPlan p = plan_loss(rows, classes, bf16);
    return p.slices ? static_cast<size_t>(p.batch) * (p.per_row * sizeof(f2) + sizeof(float)) : 0;
}

hipError_t launch_loss(const LossArgs &a, void *workspace, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const LossPlan p = plan_loss(a.rows, a.classes, a.bf16);
    return a.bf16 ? launch<true>(a, p, workspace, stream) : launch<false>(a, p, workspace, stream);
}

}  // namespace cr

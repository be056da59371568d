// What the kernels of the group norm share: tiles and pieces of points, and sums over groups.
#pragma once
#include "norm_plan.h"
#include "runs_device.h"

namespace cr {

// norm_rows.hip
void launch_norm_rows_forward(const NormArgs &a, const RowsPlan &p, hipStream_t stream);
void launch_norm_rows_backward(const NormGradArgs &a, const RowsPlan &p, const Pieces &pieces, int count, float *parts_gamma, float *parts_beta, hipStream_t stream);

namespace {

// act(z), and d act'(z) from d and z.  SiLU by the hardware's exponential and reciprocal: e^-z is off by |z| + 2 units of 2^-24 of itself (z log2(e)
// is rounded), but where that is much the sigmoid is small, so that z sigmoid(z) and its slope stay within a few units of |z| and of 1.  Below z of about -87
// both are 0.
template <int ACT> __device__ __forceinline__ float activated(float z)
{
    if constexpr (ACT == 1) return z < 0.f ? 0.f : z;
    if constexpr (ACT == 2) return z * __builtin_amdgcn_rcpf(1.f + __expf(-z));
    return z;
}
template <int ACT> __device__ __forceinline__ float through_slope(float z, float d)
{
    if constexpr (ACT == 1) return z > 0.f ? d : z <= 0.f ? 0.f : z;     // not 0 where z is not a number
    if constexpr (ACT == 2) {
        const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z));
        return d * (s * fmaf(z, 1.f - s, 1.f));
    }
    return d;
}
// sum / count with share = 1 / count rounded: the product, and what it leaves of the sum.  An exact sum's mean is exact if 32 bits hold it, so that equal values
// have no distance from it that a large rstd would show; an infinite sum's is NaN.
__device__ __forceinline__ float quotient(float sum, float count, float share)
{
    const float q = sum * share;
    return fmaf(fmaf(-q, count, sum), share, q);
}
template <int VEC> __device__ __forceinline__ void read_floats(float (&out)[VEC], const float *p, int at, float otherwise)
{
#pragma unroll
    for (int v = 0; v < VEC; ++v) out[v] = p ? p[at + v] : otherwise;
}

// Adds up the columns of `rows` rows of `width` floats in LDS, which the workgroup has just put there: thread t < width has the total of column t, t + T, ...
// through give(column, total).  LDS is free again afterwards.
template <typename F> __device__ __forceinline__ void add_columns_in_lds(int rows, int width, float *lds, F give)
{
    __syncthreads();
    // side by side by as many threads as there are, then by one each
    const int threads = blockDim.x, shares = threads / width;
    if (shares > 1) {
        const int col = threadIdx.x % width, share = threadIdx.x / width;
        float s = 0.f;
        if (share < shares)
            for (int r = share; r < rows; r += shares) s += lds[r * width + col];
        __syncthreads();
        if (share < shares) lds[share * width + col] = s;
        __syncthreads();
        rows = min(rows, shares);
    }
    for (int col = threadIdx.x; col < width; col += threads) {
        float s = 0.f;
        for (int r = 0; r < rows; ++r) s += lds[r * width + col];
        give(col, s);
    }
    __syncthreads();
}
// The same of what every thread brings: its sums of VEC columns from `at` on, of its row.
template <int VEC, typename F> __device__ __forceinline__ void add_columns(const float (&sum)[VEC], bool has, int at, int row, int rows, int width, float *lds, F give)
{
    if (has) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) lds[row * width + at + v] = sum[v];
    }
    add_columns_in_lds(rows, width, lds, give);
}

// ---- tiles ------------------------------------------------------------------------------------------------------------------------------------
struct Columns {
    int group, groups, first, width;                     // of a tile
};
__device__ __forceinline__ int slice_begin(const Tiling &t, int cg, int slice) { return static_cast<int>(int64_t(slice) * (cg / t.unit) / t.slices) * t.unit; }
__device__ __forceinline__ Columns columns_of(const LayerShape &shape, int groups, const Tiling &t, int tile)
{
    const int cg = shape.channels / groups;
    Columns c;
    if (t.slices == 1) {
        c.group = static_cast<int>(int64_t(tile) * groups / t.tiles);
        c.groups = static_cast<int>(int64_t(tile + 1) * groups / t.tiles) - c.group;
        c.first = c.group * cg;
        c.width = c.groups * cg;
    } else {
        c.group = tile / t.slices;
        c.groups = 1;
        const int s = tile % t.slices, begin = slice_begin(t, cg, s);
        c.first = c.group * cg + begin;
        c.width = slice_begin(t, cg, s + 1) - begin;
    }
    return c;
}

// What a thread of a tile has: a chunk of the tile's columns (the last one moved back to end with them: the columns it shares with its neighbour come
// out the same in both), positions ty, ty + down, ... of point `side` of those side by side.
struct Seat {
    int at, ty, side;            // at: channel in the tile
    bool has;                    // a seat at all; the others only come along to the barriers
};
template <int VEC> __device__ __forceinline__ Seat take_seat(const Tiling &t, const Columns &c)
{
    Seat s;
    const int tx = threadIdx.x % t.across, row = threadIdx.x / t.across, chunks = (c.width + VEC - 1) / VEC;
    s.ty = row % t.down;
    s.side = row / t.down;
    s.has = s.side < t.side && tx < chunks;
    s.side = min(s.side, t.side - 1);
    s.at = min(tx * VEC, c.width - VEC);
    return s;
}

// Sums over the groups of a tile.  A thread brings a value for each UNIT of its channels, which lie in one group; the sum over the rows and the channels of
// a group goes to out[side * groups + group], where every thread finds it after the call.
template <int VEC, int UNIT> struct GroupSum {
    static constexpr int NV = VEC / UNIT;
    float *lds;                  // threads * NV floats
    const Tiling &t;
    const Columns &c;
    int cg;
    __device__ __forceinline__ void put(const Seat &s, const float (&value)[NV], float *to)
    {
        const int width = c.width / UNIT;
        if (t.fold) {
            float v[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) v[i] = total_every(value[i], t.across);
            if (s.has && static_cast<int>(threadIdx.x % 64) < t.across) {
#pragma unroll
                for (int i = 0; i < NV; ++i) to[threadIdx.x / 64 * width + s.at / UNIT + i] = v[i];
            }
        } else if (s.has) {
#pragma unroll
            for (int i = 0; i < NV; ++i) to[(s.side * t.down + s.ty) * width + s.at / UNIT + i] = value[i];
        }
    }
    // `deep` tables of values, so many floats apart; the sums follow each other as the tables do
    __device__ __forceinline__ void add(const float *from, float *out, int deep = 1, int apart = 0)
    {
        const int per = cg / UNIT, width = c.width / UNIT, at_once = t.side * c.groups, sums = deep * at_once, rows = t.fold ? t.down * t.across / 64 : t.down;
        int lanes = 64;          // per sum: a power of two, so that the sums share out the workgroup's threads
        while (lanes > 1 && lanes * sums > static_cast<int>(blockDim.x)) lanes /= 2;
        const int lane = threadIdx.x % lanes, step_row = lanes / per, step_col = lanes % per;
        for (int q = threadIdx.x / lanes; q < sums; q += blockDim.x / lanes) {
            const int level = q / at_once, side = q % at_once / c.groups, g = q % c.groups;
            const float *base = from + level * apart + side * rows * width + g * per;
            int row = lane / per, col = lane % per;
            float sum = 0.f;
            while (row < rows) {
                sum += base[row * width + col];
                row += step_row;
                col += step_col;
                if (col >= per) {
                    col -= per;
                    ++row;
                }
            }
            for (int o = 1; o < lanes; o *= 2) sum += __shfl_xor(sum, o, 64);
            if (lane == 0) out[q] = sum;
        }
    }
    __device__ __forceinline__ void operator()(const Seat &s, const float (&value)[NV], float *out)
    {
        put(s, value, lds);
        __syncthreads();
        add(lds, out);
        __syncthreads();
    }
};
// what the groups' table has for the channels of a seat; WAIT: it has arrived afterwards, where every use is behind a branch, each of which would wait again, for
// stores too (2 000 x 49 x 512 bf16, gradient: 94 us, 98 without)
template <int VEC, int UNIT, bool WAIT = false> __device__ __forceinline__ void spread(float (&out)[VEC], const float *table, const Seat &s, const Columns &c, int cg)
{
    const int first = s.side * c.groups, per = cg / UNIT;
    int g = s.at / cg, r = s.at % cg / UNIT;
    float v[VEC / UNIT];
#pragma unroll
    for (int i = 0; i < VEC / UNIT; ++i) {
        v[i] = table[first + g];
        if (i + 1 < VEC / UNIT && ++r == per) {
            r = 0;
            ++g;
        }
    }
    if constexpr (WAIT) {
#pragma unroll
        for (int i = 0; i < VEC / UNIT; ++i) hold(v[i]);
    }
#pragma unroll
    for (int i = 0; i < VEC; ++i) out[i] = v[i / UNIT];
}
// the sums over UNIT neighbours
template <int VEC, int UNIT> __device__ __forceinline__ void gather(float (&out)[VEC / UNIT], const float (&v)[VEC])
{
#pragma unroll
    for (int i = 0; i < VEC / UNIT; ++i) {
        out[i] = v[i * UNIT];
#pragma unroll
        for (int j = 1; j < UNIT; ++j) out[i] += v[i * UNIT + j];
    }
}

// A thread's chunks of a tensor: positions first, first + down, ... of a point, from one channel on.  Their addresses are a scalar that moves on from one to
// the next and the thread's own offset.
template <bool BF16, int VEC> struct Walk {
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    T *base;
    int64_t offset, step;
    __device__ __forceinline__ Walk(const Rows &v, int64_t point, int64_t first, int channel, int down)
        : base(static_cast<T *>(v.p)), offset(point * v.point_stride + first * v.position_stride + channel), step(down * v.position_stride)
    {
    }
    __device__ __forceinline__ T *at(int k) const { return scalar(base + k * step) + offset; }
    // for a load that nobody branches around, where a branch would make every wait one for all loads: what is not there is the first once more
    __device__ __forceinline__ const T *at_or_first(int k, bool there) const { return base + (offset + (there ? k * step : 0)); }
    __device__ __forceinline__ void advance(int k) { base += k * step; }
};
// positions of a thread that exist: of K from `first` on, `down` apart
__device__ __forceinline__ bool exists(int first, int k, int down, int positions) { return static_cast<unsigned>(first + k * down) < static_cast<unsigned>(positions); }

// ---- pieces of a point's groups ------------------------------------------------------------------------------------------------------------
// parts[((point * tiles + tile) * pieces + piece) * (most groups of a tile) + group] = a pair of sums; forward: mean and M2, backward: A and B before
// they are divided.
struct Parts {
    f2 *pair;
    int stride;                  // most groups of a tile
    __device__ __forceinline__ int64_t at(const Tiling &t, int64_t point, int tile, int piece) const { return ((point * t.tiles + tile) * t.pieces + piece) * stride; }
};
// f(group, lane, lanes, first tile of the group) for every group of the tile, by lanes that share it and its pieces (and slices) between them.
template <typename F> __device__ __forceinline__ void join_parts(const Parts &parts, const Tiling &t, const Columns &c, int64_t point, int tile, F f)
{
    int lanes = 64;
    while (lanes > 1 && lanes * c.groups > static_cast<int>(blockDim.x)) lanes /= 2;
    const int lane = threadIdx.x % lanes, first = t.slices == 1 ? tile : tile / t.slices * t.slices;
    for (int g = threadIdx.x / lanes; g < c.groups; g += blockDim.x / lanes) f(g, lane, lanes, first);
}

// A thread's positions of a piece: from `first` on, `down` apart, `left` of them; they are taken U at a time.
struct Stretch {
    int64_t first;
    int left;
};
__device__ __forceinline__ Stretch stretch_of(const Tiling &t, int piece, int ty, int positions)
{
    const int64_t begin = int64_t(piece) * t.down * t.k, end = min(begin + int64_t(t.down) * t.k, int64_t(positions));
    const int rows = static_cast<int>(end - begin);
    return {begin + min(ty, rows - 1), (rows - ty + t.down - 1) / t.down};               // none where ty is past the end
}
template <bool ONCE, bool BF16, int VEC, int U> __device__ __forceinline__ void load_step(typename Chunk<BF16, VEC>::raw (&raw)[U], const Walk<BF16, VEC> &from, int left)
{
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const auto *p = from.at_or_first(u, u < left);
        raw[u] = ONCE ? Chunk<BF16, VEC>::load_once(p) : Chunk<BF16, VEC>::load(p);
    }
}
template <int U, typename R> __device__ __forceinline__ void hold_step(R (&raw)[U])
{
#pragma unroll
    for (int u = 0; u < U; ++u) hold(raw[u]);
}
// A chunk of an output that may be an input itself: the columns that the last chunk shares with its neighbour are the neighbour's, which may have replaced
// them before this thread read them.
template <bool BF16, int VEC> __device__ __forceinline__ void put_chunk(typename Chunk<BF16, 1>::element *to, const float (&v)[VEC], const Columns &c, const Seat &s)
{
    const int own = (c.width + VEC - 1) / VEC * VEC - c.width;           // the first element that is the last chunk's alone
    if (own == 0 || s.at < c.width - VEC) {
        Chunk<BF16, VEC>::store(to, Chunk<BF16, VEC>::narrow(v));
    } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (i >= own) Element<BF16>::put(to + i, v[i]);
    }
}
// ---- launches by type -------------------------------------------------------------------------------------------------------------------------
template <typename F> void with_k(int k, F f)
{
    switch (k) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    default: f(std::integral_constant<int, 8>()); break;
    }
}
// f(bf16, vec, unit): channels of a load, and of those the neighbours that always lie in one group
template <typename F> void with_types(const LayerShape &s, int groups, F f)
{
    using Yes = std::true_type;
    using No = std::false_type;
    const int vec = vec_of(s), cg = s.channels / groups;
    auto with = [&](auto bf16, auto v) {
        constexpr int V = v(), HALF = V > 1 ? V / 2 : 1, QUARTER = V > 3 ? V / 4 : 1;
        if (cg % V == 0) f(bf16, v, v);
        else if (cg % HALF == 0) f(bf16, v, std::integral_constant<int, HALF>());
        else if (cg % QUARTER == 0) f(bf16, v, std::integral_constant<int, QUARTER>());
        else f(bf16, v, std::integral_constant<int, 1>());
    };
    if (vec == 1) s.bf16 ? with(Yes(), std::integral_constant<int, 1>()) : with(No(), std::integral_constant<int, 1>());
    else if (s.bf16) with(Yes(), std::integral_constant<int, 8>());
    else with(No(), std::integral_constant<int, 4>());
}
template <typename F> void with_activation(int kind, F f)
{
    switch (kind) {
    case 0: f(std::integral_constant<int, 0>()); break;
    case 1: f(std::integral_constant<int, 1>()); break;
    default: f(std::integral_constant<int, 2>()); break;
    }
}
}  // namespace

}  // namespace cr

// What the kernels of the group norm share: tiles and pieces of points, sums over groups, and which kernels a call takes.
#pragma once
#include "runs_device.h"

#include <algorithm>

namespace cr {

// norm_rows.hip
struct RowsPlan {
    int lanes, chunks;           // lanes of a group, chunks of a lane; no lanes: not these kernels
    int wide, down;              // groups side by side in a workgroup, points
};
RowsPlan rows_plan(const LayerShape &shape, int groups, bool backward);
int64_t rows_piece(const LayerShape &shape, int groups, const RowsPlan &p);             // points of a piece of a run
void launch_norm_rows_forward(const NormArgs &a, const RowsPlan &p, hipStream_t stream);
void launch_norm_rows_backward(const NormGradArgs &a, const RowsPlan &p, const Pieces &pieces, int count, float *parts_gamma, float *parts_beta, hipStream_t stream);

namespace {

constexpr int kUnits = 256;

// act(z), and d act'(z) from d and z
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
// How a launch cuts points into tiles.  Columns: `tiles` of them, each some whole groups, or (slices > 1) a part of one group.  Rows: `down` positions side
// by side, K below each other in a thread; `side` points side by side.
struct Tiling {
    int tiles, slices, unit, across, down, side, threads, k;             // slices begin at multiples of `unit` channels of the group
    int pieces;                  // of a point's positions, down * k each
    int deep;                    // points of a thread, or 0: it has one point's positions (k of them)
    int fold;                    // the seats of a column in a wavefront are `across` lanes apart, and the wavefront has one point's: they are added up before LDS
};
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
// ---- which of them ----------------------------------------------------------------------------------------------------------------------------
inline int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

constexpr int kMostGroups = 4096;                        // sums of a workgroup: with what they are made from they fit 64 KB of LDS
constexpr int kPartThreads = 256;                        // of norm_part_* and norm_join_*
constexpr int kForwardThreads = 1024, kBackwardThreads = 256;           // of norm_tile_*, at most

inline int vec_of(const LayerShape &s) { return s.channels < (s.bf16 ? 8 : 4) ? 1 : s.bf16 ? 8 : 4; }
// of a load of vec channels, the neighbours that always lie in one group: the largest power of two that divides both
inline int unit_of(int cg, int vec)
{
    while (cg % vec != 0) vec /= 2;
    return vec;
}
inline int across_for(const LayerShape &s, int groups, int tiles) { return ceil_div(int64_t(ceil_div(groups, tiles)) * (s.channels / groups), vec_of(s)); }
// Whether the seats of a column can be added up inside a wavefront; rounds `down` for it where there is room.
inline void fold_columns(Tiling *t)
{
    t->fold = 0;
    if (t->across > 32 || (t->across & (t->across - 1)) != 0) return;
    const int step = 64 / t->across, down = (t->down + step - 1) / step * step;
    if (t->side > 1 ? t->down % step != 0 : down * t->across > t->threads) return;
    t->down = t->side > 1 ? t->down : down;
    t->fold = 1;
}

// Tiles in registers: at most so many threads and chunks of each; k == 0: the point is too large, and is cut into pieces.  Small workgroups, of which
// several share a compute unit and one loads while others add up; so tiles get more chunks of a thread, then narrower (down to a cache line of columns), and only
// then more threads.  320 x 1 024 x 16 bf16 forward, 256 threads with 8 chunks each 11.5 us, 1 024 with two 17.0; 1 000 x 196 x 256 47 with 8 chunks, 70 with 4;
// its gradient 96 with 8 chunks and 256 threads, 145 with 4 and 512, 112 in pieces.  Columns of half a line
// rather than pieces: 500 x 400 x 96 fp32 gradient 110 us against 77 in pieces, 64 x 1 800 x 160 forward 74 against 43.
inline Tiling tile(const LayerShape &s, int groups, bool backward)
{
    // (the gradient of one position each leaves room for a group of 512 chunks)
    const int most_threads = !backward ? kForwardThreads : s.positions == 1 ? 2 * kBackwardThreads : kBackwardThreads, most_chunks = 8, vec = vec_of(s);
    const int cg = s.channels / groups, line = std::max(1, 128 / (cg * (s.bf16 ? 2 : 4)));
    Tiling t = {};
    t.slices = t.unit = t.side = t.pieces = 1;
    const int most_tiles = std::max(1, std::min(groups / line, 65535));      // of a grid's second dimension
    auto fits = [&](int threads, int chunks, int tiles) {
        const int across = across_for(s, groups, tiles);
        return across <= threads && ceil_div(groups, tiles) <= kMostGroups && int64_t(s.positions) <= int64_t(threads / across) * chunks;
    };
    auto more = [&](int tiles) { return std::min(most_tiles, tiles * 2); };
    for (t.threads = 256; t.threads <= most_threads; t.threads *= 2) {
        int tiles = 1;
        while (tiles < most_tiles && !fits(t.threads, most_chunks, tiles)) tiles = more(tiles);
        if (!fits(t.threads, most_chunks, tiles)) continue;
        while (tiles < most_tiles && s.points * tiles < kUnits) tiles = more(tiles);
        t.tiles = tiles;
        t.across = across_for(s, groups, tiles);
        t.k = 1;
        while (int64_t(t.threads / t.across) * t.k < s.positions) t.k *= 2;
        // Where there are points enough, more chunks of a thread and more points side by side: a thread adds up its own rows of a group before it meets others,
        // and a step of a workgroup is that much more.  (Not where over two fifths of what a thread could have would be empty.)  Forward and gradient, us,
        // with the fewest chunks and so: 20 000 x 4 x 320 bf16 53 and 121, 29 and 69; 45 575 x 17 x 90 241 and 333, 77 and 190; 4 096 x 16 x 33 fp32 12 and
        // 33, 9 and 20.  Sums per channel of eight channels: the gradient's registers are full at four chunks (45 575 x 17 x 90 with eight: 247).
        const int values = vec / unit_of(cg, vec), side = t.threads / (t.across * ceil_div(s.positions, t.k)), fewest = t.k;
        for (int k = 2 * fewest; k <= (backward && values == 8 ? 4 : most_chunks) && k / 2 < s.positions; k *= 2) {
            const int more_side = t.threads / (t.across * ceil_div(s.positions, k));
            if (5 * more_side * fewest >= 3 * side * k && s.points * tiles >= int64_t(kUnits) * more_side) t.k = k;
        }
        t.down = ceil_div(s.positions, t.k);             // as even as can be
        t.side = std::max(1, std::min(t.threads / (t.across * t.down), kMostGroups / ceil_div(groups, tiles)));
        t.side = static_cast<int>(std::min<int64_t>(t.side, std::max<int64_t>(1, s.points)));
        fold_columns(&t);
        // one position each: several points each, so long as there are enough for all workgroups and LDS for their sums
        if (t.k == 1 && t.threads <= 512) {
            auto room = [&](int deep) { return (size_t(deep) * t.threads * values + size_t(2) * deep * t.side * ceil_div(groups, tiles)) * (backward ? 2 : 1) * sizeof(float); };
            // (the gradient of four, with a sum per channel, is more than the registers hold)
            for (int deep = backward && values > 1 ? 2 : 4; deep > 1 && !t.deep; deep /= 2)
                if (room(deep) <= size_t(48) << 10 && s.points * tiles >= int64_t(4) * kUnits * t.side * deep) t.deep = deep;
        }
        return t;
    }
    return t;
}
inline Tiling cut(const LayerShape &s, int groups)
{
    const int vec = vec_of(s), cg = s.channels / groups;
    Tiling t = {};
    t.side = t.slices = 1;
    t.threads = kPartThreads;
    t.unit = unit_of(cg, vec);
    if (ceil_div(cg, vec) > t.threads) {                 // a group is wider than a workgroup
        t.slices = ceil_div(cg, int64_t(t.threads) * vec);
        t.tiles = groups * t.slices;
        t.across = ceil_div(int64_t(ceil_div(cg / t.unit, t.slices)) * t.unit, vec);
    } else {
        t.tiles = ceil_div(ceil_div(s.channels, vec), t.threads);
        while (across_for(s, groups, t.tiles) > t.threads) ++t.tiles;
        t.across = across_for(s, groups, t.tiles);
    }
    // Positions of a thread: many where the chip has enough workgroups anyway.  Forward, us, for 8 / 16 / 32 / 64: 64 x 4 096 x 512 bf16 237 / 177 / 176 / 172,
    // 64 x 1 024 x 320 41 / 34 / 39 / 53, 16 x 16 384 x 64 27 / 28 / 32 / 50; backward 316 / 279 / 278 / 274, 64 / 57 / 64 / 79, 45 / 46 / 52 / 78.
    t.down = t.threads / t.across;
    t.k = 8;
    auto workgroups = [&](int k) { return s.points * t.tiles * (int64_t(s.positions) / (int64_t(t.down) * k)); };
    if (workgroups(16) >= 2 * kUnits) t.k = 16;
    while (t.k >= 16 && t.k < 64 && workgroups(2 * t.k) >= 4 * kUnits) t.k *= 2;
    t.pieces = ceil_div(s.positions, int64_t(t.down) * t.k);
    t.down = std::min(t.down, s.positions);
    fold_columns(&t);
    return t;
}
inline int most_groups(const Tiling &t, int groups) { return t.slices > 1 ? 1 : ceil_div(groups, t.tiles); }

// Points of a pair of launches: as many as a grid takes.  (Fewer, so that what is read twice comes from the last-level cache, cost more at the launches' ends
// than they gain: 64 x 4 096 x 512 bf16, points of 96 MB at a time / of 192 / all: forward 213 / 196 / 176 us, backward 365 / 320 / 279.)
inline int64_t batch_points(const LayerShape &s, const Tiling &t) { return std::max<int64_t>(1, std::min<int64_t>(s.points, (int64_t(1) << 22) / t.pieces)); }

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

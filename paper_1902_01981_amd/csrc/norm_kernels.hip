// Group norm with an activation, channels last, for gfx950.
//
// A thread has a chunk of 16 bytes of channels and goes down a point's positions, so that its gamma, beta and statistics stay in registers.  Sums over a
// group meet in LDS.  The variance is the mean of squared distances from the mean, taken from registers in a second step, never a difference of large
// sums; tiles of a group that several workgroups have meet by  M2 = sum M2_i + n_i (mean_i - mean)^2.
//
//   norm_rows_*    points of one position, groups of 1 to 64 chunks, a power of two: a group is a few lanes, no workgroup meets
//   norm_tile_*    a point's group (or some of them, or several points) in the registers of a workgroup, read once
//   norm_deep_*    the same for several points of few positions at a time
//   norm_part_*, norm_join_*   larger groups: pieces of a group leave their sums, then every piece is read again
#include "runs_device.h"

namespace cr {

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
// (x - mean) rstd.  From bf16 by one multiply-add: mean rstd is then rounded by itself, which is what the mean's own rounding does to all values of a
// group anyway, and x has no bits that it would cost.
template <bool BF16> struct Normal {
    float scale, shift;
    __device__ __forceinline__ Normal(float mean, float rstd) : scale(rstd), shift(BF16 ? -mean * rstd : mean) {}
    __device__ __forceinline__ float operator()(float x) const { return BF16 ? fmaf(x, scale, shift) : (x - shift) * scale; }
};
template <int VEC> __device__ __forceinline__ void read_floats(float (&out)[VEC], const float *p, int at, float otherwise)
{
#pragma unroll
    for (int v = 0; v < VEC; ++v) out[v] = p ? p[at + v] : otherwise;
}

// ---- points of one position, groups of a few lanes ---------------------------------------------------------------------------------------
// A thread stays with its chunk and goes through the points, U at a time.  Its group is the LANES lanes around it.
template <bool BF16, int LANES, int ACT> __global__ void __launch_bounds__(256) norm_rows_forward_kernel(NormArgs a, int across, int64_t length)
{
    constexpr int VEC = BF16 ? 8 : 4, U = 4;
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int chunks = a.shape.channels / VEC, tx = threadIdx.x % across, ty = threadIdx.x / across, down = 256 / across;
    const int q = blockIdx.x * across + tx;
    if (q >= chunks || ty >= down) return;               // whole groups of lanes
    float gamma[VEC], beta[VEC];
    read_floats(gamma, a.gamma, q * VEC, 1.f);
    read_floats(beta, a.beta, q * VEC, 0.f);
    const float share = 1.f / (LANES * VEC);
    const int64_t begin = blockIdx.y * length, end = min(begin + length, a.shape.points);
    const T *x = static_cast<const T *>(a.x.p) + q * VEC;
    T *y = static_cast<T *>(a.y.p) + q * VEC;
    for (int64_t n0 = begin + ty; n0 < end; n0 += U * down) {
        typename C::raw raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = C::load_once(x + min(n0 + u * down, end - 1) * a.x.point_stride);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t n = n0 + u * down;
            float v[VEC];
            C::widen(raw[u], v);
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) sum += v[i];
            const float mean = lanes_total<LANES>(sum) * share;
            sum = 0.f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[i] -= mean;
                sum = fmaf(v[i], v[i], sum);
            }
            const float rstd = 1.f / sqrtf(fmaf(lanes_total<LANES>(sum), share, a.eps));
            if (n >= end) continue;
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = activated<ACT>(fmaf(v[i] * rstd, gamma[i], beta[i]));
            C::store(y + n * a.y.point_stride, C::narrow(v));
            if (a.mean && q % LANES == 0) {
                a.mean[n * a.groups + q / LANES] = mean;
                a.rstd[n * a.groups + q / LANES] = rstd;
            }
        }
    }
}

// Adds up columns over the rows side by side of a workgroup: sum[VEC] of thread (tx, ty) with `across` chunks side by side.  Thread t < width has the total
// of column t, t + T, ... through `give(column, total)`.  lds holds down * width floats, which are free before and after.
template <int VEC, typename F> __device__ __forceinline__ void add_columns(const float (&sum)[VEC], bool has, int at, int row, int rows, int width, float *lds, F give)
{
    if (has) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) lds[row * width + at + v] = sum[v];
    }
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

template <bool BF16, int LANES, int ACT>
__global__ void __launch_bounds__(256) norm_rows_backward_kernel(NormGradArgs a, int across, Pieces pieces, float *parts_gamma, float *parts_beta)
{
    constexpr int VEC = BF16 ? 8 : 4, U = 4;
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float lds[256 * VEC];
    const int chunks = a.shape.channels / VEC, tx = threadIdx.x % across, ty = threadIdx.x / across, down = 256 / across;
    const int q = min(static_cast<int>(blockIdx.x * across) + tx, chunks - 1);           // lanes past the row go along with the last chunk
    const bool mine = ty < down && static_cast<int>(blockIdx.x * across) + tx < chunks;
    float gamma[VEC], beta[VEC], sum_gamma[VEC], sum_beta[VEC];
    read_floats(gamma, a.gamma, q * VEC, 1.f);
    read_floats(beta, a.beta, q * VEC, 0.f);
#pragma unroll
    for (int i = 0; i < VEC; ++i) sum_gamma[i] = sum_beta[i] = 0.f;
    const float share = 1.f / (LANES * VEC);
    const Piece piece = find_piece(pieces, blockIdx.y);
    const T *x = static_cast<const T *>(a.x.p) + q * VEC, *dy = static_cast<const T *>(a.dy.p) + q * VEC;
    T *dx = static_cast<T *>(a.dx.p) + q * VEC;
    if (mine) {
        for (int64_t n0 = piece.begin + ty; n0 < piece.end; n0 += U * down) {
            typename C::raw raw[U], raw_d[U];
            float mean[U], rstd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t n = min(n0 + u * down, piece.end - 1);
                raw[u] = C::load_once(x + n * a.x.point_stride);
                raw_d[u] = C::load_once(dy + n * a.dy.point_stride);
                mean[u] = a.mean[n * a.groups + q / LANES];
                rstd[u] = a.rstd[n * a.groups + q / LANES];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t n = n0 + u * down;
                const Normal<BF16> normal(mean[u], rstd[u]);
                float h[VEC], d[VEC], A = 0.f, B = 0.f;
                C::widen(raw[u], h);
                C::widen(raw_d[u], d);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[i] = normal(h[i]);
                    d[i] = through_slope<ACT>(fmaf(h[i], gamma[i], beta[i]), d[i]);
                    const float t = gamma[i] * d[i];
                    A += t;
                    B = fmaf(t, h[i], B);
                }
                A = lanes_total<LANES>(A) * share;
                B = lanes_total<LANES>(B) * share;
                if (n >= piece.end) continue;
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    sum_beta[i] += d[i];
                    sum_gamma[i] = fmaf(d[i], h[i], sum_gamma[i]);
                    d[i] = rstd[u] * fmaf(-h[i], B, fmaf(gamma[i], d[i], -A));
                }
                if (a.dx.p) C::store(dx + n * a.dx.point_stride, C::narrow(d));
            }
        }
    }
    if (!parts_gamma) return;
    const int width = across * VEC, first = blockIdx.x * width;
    auto give = [&](float *parts) {
        return [=](int col, float total) {
            if (first + col < a.shape.channels) parts[int64_t(blockIdx.y) * a.shape.channels + first + col] = total;
        };
    };
    add_columns(sum_gamma, ty < down, tx * VEC, ty, down, width, lds, give(parts_gamma));
    add_columns(sum_beta, ty < down, tx * VEC, ty, down, width, lds, give(parts_beta));
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

// What a thread of a tile has: chunk `chunk` of the tile's columns (the last one moved back to end with them: the columns it shares with its neighbour come
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
// what the groups' table has for the channels of a seat
template <int VEC, int UNIT> __device__ __forceinline__ void spread(float (&out)[VEC], const float *table, const Seat &s, const Columns &c, int cg)
{
    const int first = s.side * c.groups, per = cg / UNIT;
    int g = s.at / cg, r = s.at % cg / UNIT;
#pragma unroll
    for (int i = 0; i < VEC; i += UNIT) {
        const float v = table[first + g];
#pragma unroll
        for (int j = 0; j < UNIT; ++j) out[i + j] = v;
        if (i + UNIT < VEC && ++r == per) {
            r = 0;
            ++g;
        }
    }
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

// The mean and the sum of squared distances from it, for the groups of a tile: mean[side * groups + group], M2 likewise.
template <bool BF16, int VEC, int K, int UNIT>
__device__ __forceinline__ void tile_moments(const typename Chunk<BF16, VEC>::raw (&raw)[K], const Seat &s, int positions, const Tiling &t, const Columns &c, int cg,
                                             float count, GroupSum<VEC, UNIT> &sums, float *mean, float *m2)
{
    using C = Chunk<BF16, VEC>;
    constexpr int NV = VEC / UNIT;
    float sum[NV], m[VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) sum[i] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (exists(s.ty, k, t.down, positions)) {
            float x[VEC];
            C::widen(raw[k], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) sum[v / UNIT] += x[v];
        }
    }
    sums(s, sum, mean);
    for (int q = threadIdx.x; q < t.side * c.groups; q += blockDim.x) mean[q] /= count;
    __syncthreads();
    spread<VEC, UNIT>(m, mean, s, c, cg);
#pragma unroll
    for (int i = 0; i < NV; ++i) sum[i] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (exists(s.ty, k, t.down, positions)) {
            float x[VEC];
            C::widen(raw[k], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                x[v] -= m[v];
                sum[v / UNIT] = fmaf(x[v], x[v], sum[v / UNIT]);
            }
        }
    }
    sums(s, sum, m2);
}

// y from x: gamma h + beta and the activation; by one multiply-add from bf16, as Normal
template <bool BF16, int VEC, int ACT> struct Finish {
    float shift[VEC], scale[VEC], beta[VEC];
    __device__ __forceinline__ Finish(const NormArgs &a, int channel, const float (&mean)[VEC], const float (&rstd)[VEC])
    {
        read_floats(scale, a.gamma, channel, 1.f);
        read_floats(beta, a.beta, channel, 0.f);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            scale[v] *= rstd[v];
            shift[v] = mean[v];
            if (BF16) beta[v] = fmaf(-mean[v], scale[v], beta[v]);
        }
    }
    __device__ __forceinline__ void operator()(float (&x)[VEC]) const
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) x[v] = activated<ACT>(fmaf(BF16 ? x[v] : x[v] - shift[v], scale[v], beta[v]));
    }
};

template <bool BF16, int VEC, int K, int UNIT, int ACT, int MOST> __global__ void __launch_bounds__(MOST) norm_tile_forward_kernel(NormArgs a, Tiling t)
{
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, positions = a.shape.positions;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg};
    float *mean = lds + t.threads * (VEC / UNIT), *rstd = mean + t.side * c.groups;
    const float count = static_cast<float>(positions) * cg;
    for (int64_t n0 = int64_t(blockIdx.x) * t.side; n0 < a.shape.points; n0 += int64_t(gridDim.x) * t.side) {
        const int64_t n = n0 + s.side;
        typename C::raw raw[K];
        const Walk<BF16, VEC> x(a.x, min(n, a.shape.points - 1), min(s.ty, positions - 1), c.first + s.at, t.down);
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k] = C::load_once(x.at_or_first(k, exists(s.ty, k, t.down, positions)));
#pragma unroll
        for (int k = 0; k < K; ++k) hold(raw[k]);
        tile_moments<BF16, VEC, K, UNIT>(raw, s, positions, t, c, cg, count, sums, mean, rstd);
        for (int q = threadIdx.x; q < t.side * c.groups; q += blockDim.x) {
            rstd[q] = 1.f / sqrtf(rstd[q] / count + a.eps);
            const int64_t point = n0 + q / c.groups;
            if (a.mean && point < a.shape.points) {
                a.mean[point * a.groups + c.group + q % c.groups] = mean[q];
                a.rstd[point * a.groups + c.group + q % c.groups] = rstd[q];
            }
        }
        __syncthreads();
        if (s.has && n < a.shape.points) {
            float m[VEC], r[VEC];
            spread<VEC, UNIT>(m, mean, s, c, cg);
            spread<VEC, UNIT>(r, rstd, s, c, cg);
            const Finish<BF16, VEC, ACT> finish(a, c.first + s.at, m, r);
            const Walk<BF16, VEC> y(a.y, n, s.ty, c.first + s.at, t.down);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (exists(s.ty, k, t.down, positions)) {
                    float v[VEC];
                    C::widen(raw[k], v);
                    finish(v);
                    C::store(y.at(k), C::narrow(v));
                }
            }
        }
        __syncthreads();                                 // before the tables are another point's
    }
}

// Points of few positions: a thread has one position (if that many) of K points, which share the barriers.
template <bool BF16, int VEC, int K, int UNIT, int ACT> __global__ void __launch_bounds__(512) norm_deep_forward_kernel(NormArgs a, Tiling t)
{
    using C = Chunk<BF16, VEC>;
    constexpr int NV = VEC / UNIT;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, positions = a.shape.positions;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg};
    const int room = t.threads * NV, tables = t.side * c.groups;
    float *mean = lds + K * room, *rstd = mean + K * tables;
    const float count = static_cast<float>(positions) * cg, share = 1.f / count;
    const bool there = s.ty < positions;
    for (int64_t n0 = int64_t(blockIdx.x) * t.side * K; n0 < a.shape.points; n0 += int64_t(gridDim.x) * t.side * K) {
        const int64_t n = n0 + s.side;                   // and n + side, ...
        typename C::raw raw[K];
        const Walk<BF16, VEC> x(a.x, 0, min(s.ty, positions - 1), c.first + s.at, t.down);
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k] = C::load_once(x.base + (x.offset + min(n + k * t.side, a.shape.points - 1) * a.x.point_stride));
#pragma unroll
        for (int k = 0; k < K; ++k) {
            hold(raw[k]);
            float v[VEC], brought[NV];
            C::widen(raw[k], v);
            gather<VEC, UNIT>(brought, v);
#pragma unroll
            for (int i = 0; i < NV; ++i) brought[i] = there ? brought[i] : 0.f;
            sums.put(s, brought, lds + k * room);
        }
        __syncthreads();
        sums.add(lds, mean, K, room);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float v[VEC], m[VEC], brought[NV];
            C::widen(raw[k], v);
            spread<VEC, UNIT>(m, mean + k * tables, s, c, cg);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                v[i] = fmaf(-m[i], share, v[i]);
                v[i] *= v[i];
            }
            gather<VEC, UNIT>(brought, v);
#pragma unroll
            for (int i = 0; i < NV; ++i) brought[i] = there ? brought[i] : 0.f;
            sums.put(s, brought, lds + k * room);
        }
        __syncthreads();
        sums.add(lds, rstd, K, room);
        __syncthreads();
        for (int q = threadIdx.x; q < K * tables; q += blockDim.x) {
            mean[q] *= share;
            rstd[q] = 1.f / sqrtf(fmaf(rstd[q], share, a.eps));
            const int64_t point = n0 + q / c.groups;     // tables of points n0, n0 + 1, ...
            if (a.mean && point < a.shape.points) {
                a.mean[point * a.groups + c.group + q % c.groups] = mean[q];
                a.rstd[point * a.groups + c.group + q % c.groups] = rstd[q];
            }
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (s.has && there && n + k * t.side < a.shape.points) {
                float v[VEC], m[VEC], r[VEC];
                spread<VEC, UNIT>(m, mean + k * tables, s, c, cg);
                spread<VEC, UNIT>(r, rstd + k * tables, s, c, cg);
                const Finish<BF16, VEC, ACT> finish(a, c.first + s.at, m, r);
                C::widen(raw[k], v);
                finish(v);
                const Walk<BF16, VEC> y(a.y, n + k * t.side, s.ty, c.first + s.at, t.down);
                C::store(y.base + y.offset, C::narrow(v));
            }
        }
        __syncthreads();                                 // before the tables are other points'
    }
}

// What a thread needs of its channels for the gradient.
template <bool BF16, int VEC, int ACT> struct Gradient {
    float mean[VEC], rstd[VEC], gamma[VEC], beta[VEC];
    __device__ __forceinline__ float h(float x, int v) const { return Normal<BF16>(mean[v], rstd[v])(x); }
    // dz from dy; h is left in x
    __device__ __forceinline__ void slopes(float (&x)[VEC], float (&d)[VEC]) const
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            x[v] = h(x[v], v);
            d[v] = through_slope<ACT>(fmaf(x[v], gamma[v], beta[v]), d[v]);
        }
    }
};
// dx = rstd (gamma dz - A - h B); where a group is one value gamma dz and A are the same, and nothing is left of them
template <int VEC> struct Correction {
    float A[VEC], B[VEC];
    __device__ __forceinline__ Correction(const float (&sum_A)[VEC], const float (&sum_B)[VEC], float share)
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            A[v] = sum_A[v] * share;
            B[v] = sum_B[v] * share;
        }
    }
    template <typename G> __device__ __forceinline__ float operator()(const G &g, float h, float dz, int v) const
    {
        return g.rstd[v] * fmaf(-h, B[v], fmaf(g.gamma[v], dz, -A[v]));
    }
};
// mean and 1 / deviation of a seat's channels, from the tensors
template <int VEC, int UNIT> __device__ __forceinline__ void read_stats(float (&m)[VEC], float (&r)[VEC], const NormGradArgs &a, const Seat &s, const Columns &c, int64_t point, int cg)
{
    const float *mean = a.mean + point * a.groups + c.group, *rstd = a.rstd + point * a.groups + c.group;
    Columns one = c;
    Seat seat = s;
    one.groups = 0;                                      // the tables are this point's
    seat.side = 0;
    const int within = c.first - c.group * cg;           // a slice of a group begins inside it
    seat.at += within;
    spread<VEC, UNIT>(m, mean, seat, one, cg);
    spread<VEC, UNIT>(r, rstd, seat, one, cg);
}

// The groups' sums of gamma s1 and gamma s2, for every thread.
template <int VEC, int UNIT>
__device__ __forceinline__ void bring(GroupSum<VEC, UNIT> &sums, const Seat &s, const float (&gamma)[VEC], float (&s1)[VEC], float (&s2)[VEC], int room, float *A_of, float *B_of)
{
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        s1[v] *= gamma[v];
        s2[v] *= gamma[v];
    }
    float brought[VEC / UNIT];
    gather<VEC, UNIT>(brought, s1);
    sums.put(s, brought, sums.lds);
    gather<VEC, UNIT>(brought, s2);
    sums.put(s, brought, sums.lds + room);
    __syncthreads();
    sums.add(sums.lds, A_of);
    sums.add(sums.lds + room, B_of);
    __syncthreads();
}
// A workgroup goes through the points of a piece of a run, `side` at a time.
template <bool BF16, int VEC, int K, int UNIT, int ACT>
__global__ void __launch_bounds__(256) norm_tile_backward_kernel(NormGradArgs a, Tiling t, Pieces pieces, float *parts_gamma, float *parts_beta)
{
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, positions = a.shape.positions;
    const Columns c = columns_of(a.shape, a.groups, t, blockIdx.y);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg};
    const int room = t.threads * (VEC / UNIT);
    float *A_of = lds + 2 * room, *B_of = A_of + t.side * c.groups;
    const float share = 1.f / (static_cast<float>(positions) * cg);
    Gradient<BF16, VEC, ACT> g;
    float sum_gamma[VEC], sum_beta[VEC];
    read_floats(g.gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(g.beta, a.beta, c.first + s.at, 0.f);
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum_gamma[v] = sum_beta[v] = 0.f;
    const Piece piece = find_piece(pieces, blockIdx.x);
    for (int64_t n0 = piece.begin; n0 < piece.end; n0 += t.side) {
        const int64_t n = min(n0 + s.side, piece.end - 1);
        const bool live = s.has && n0 + s.side < piece.end;
        typename C::raw raw[K], raw_d[K];
        const int first = min(s.ty, positions - 1);
        const Walk<BF16, VEC> x(a.x, n, first, c.first + s.at, t.down), dy(a.dy, n, first, c.first + s.at, t.down);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = C::load_once(x.at_or_first(k, exists(s.ty, k, t.down, positions)));
            raw_d[k] = C::load_once(dy.at_or_first(k, exists(s.ty, k, t.down, positions)));
        }
        read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, n, cg);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            hold(raw[k]);
            hold(raw_d[k]);
        }
        float dz[K][VEC], s1[VEC], s2[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) s1[v] = s2[v] = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (exists(s.ty, k, t.down, positions)) {
                float h[VEC];
                C::widen(raw[k], h);
                C::widen(raw_d[k], dz[k]);
                g.slopes(h, dz[k]);
#pragma unroll
                for (int v = 0; v < VEC; ++v) {
                    s1[v] += dz[k][v];
                    s2[v] = fmaf(dz[k][v], h[v], s2[v]);
                }
            }
        }
        if (live) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                sum_beta[v] += s1[v];
                sum_gamma[v] += s2[v];
            }
        }
        if (!a.dx.p) continue;
        bring<VEC, UNIT>(sums, s, g.gamma, s1, s2, room, A_of, B_of);
        if (live) {
            float A[VEC], B[VEC];
            spread<VEC, UNIT>(A, A_of, s, c, cg);
            spread<VEC, UNIT>(B, B_of, s, c, cg);
            const Correction<VEC> dx_of(A, B, share);
            const Walk<BF16, VEC> dx(a.dx, n, s.ty, c.first + s.at, t.down);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (exists(s.ty, k, t.down, positions)) {
                    float h[VEC];
                    C::widen(raw[k], h);
#pragma unroll
                    for (int v = 0; v < VEC; ++v) h[v] = dx_of(g, g.h(h[v], v), dz[k][v], v);
                    C::store(dx.at(k), C::narrow(h));
                }
            }
        }
        // the next step's sums are put where this one's were read before the last barrier, and its results written after another one
    }
    if (!parts_gamma) return;
    __syncthreads();
    auto give = [&](float *parts) { return [=](int col, float total) { parts[int64_t(blockIdx.x) * a.shape.channels + c.first + col] = total; }; };
    const int row = s.side * t.down + s.ty, rows = t.side * t.down;
    add_columns(sum_gamma, s.has, s.at, row, rows, c.width, lds, give(parts_gamma));
    add_columns(sum_beta, s.has, s.at, row, rows, c.width, lds, give(parts_beta));
}

template <bool BF16, int VEC, int K, int UNIT, int ACT>
__global__ void __launch_bounds__(256) norm_deep_backward_kernel(NormGradArgs a, Tiling t, Pieces pieces, float *parts_gamma, float *parts_beta)
{
    using C = Chunk<BF16, VEC>;
    constexpr int NV = VEC / UNIT;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, positions = a.shape.positions;
    const Columns c = columns_of(a.shape, a.groups, t, blockIdx.y);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg};
    const int room = t.threads * NV, tables = t.side * c.groups;
    float *A_of = lds + 2 * K * room, *B_of = A_of + K * tables;
    const float share = 1.f / (static_cast<float>(positions) * cg);
    const bool there = s.ty < positions;
    Gradient<BF16, VEC, ACT> g;
    float sum_gamma[VEC], sum_beta[VEC];
    read_floats(g.gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(g.beta, a.beta, c.first + s.at, 0.f);
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum_gamma[v] = sum_beta[v] = 0.f;
    const Piece piece = find_piece(pieces, blockIdx.x);
    const Walk<BF16, VEC> x(a.x, 0, min(s.ty, positions - 1), c.first + s.at, t.down), dy(a.dy, 0, min(s.ty, positions - 1), c.first + s.at, t.down);
    for (int64_t n0 = piece.begin; n0 < piece.end; n0 += t.side * K) {
        typename C::raw raw[K], raw_d[K];
        auto point = [&](int k) { return min(n0 + s.side + k * t.side, piece.end - 1); };
        auto live = [&](int k) { return s.has && there && n0 + s.side + k * t.side < piece.end; };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            raw[k] = C::load_once(x.base + (x.offset + point(k) * a.x.point_stride));
            raw_d[k] = C::load_once(dy.base + (dy.offset + point(k) * a.dy.point_stride));
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            hold(raw[k]);
            hold(raw_d[k]);
        }
        float dz[K][VEC];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float h[VEC], s1[VEC], s2[VEC], brought[NV];
            C::widen(raw[k], h);
            C::widen(raw_d[k], dz[k]);
            read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, point(k), cg);
            g.slopes(h, dz[k]);
            const bool counts = live(k);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                s1[v] = counts ? dz[k][v] : 0.f;
                s2[v] = s1[v] * h[v];
                sum_beta[v] += s1[v];
                sum_gamma[v] = fmaf(s1[v], h[v], sum_gamma[v]);
                s1[v] *= g.gamma[v];
                s2[v] *= g.gamma[v];
            }
            if (!a.dx.p) continue;
            gather<VEC, UNIT>(brought, s1);
            sums.put(s, brought, lds + k * room);
            gather<VEC, UNIT>(brought, s2);
            sums.put(s, brought, lds + (K + k) * room);
        }
        if (!a.dx.p) continue;
        __syncthreads();
        sums.add(lds, A_of, K, room);
        sums.add(lds + K * room, B_of, K, room);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (live(k)) {
                float h[VEC], A[VEC], B[VEC];
                C::widen(raw[k], h);
                spread<VEC, UNIT>(A, A_of + k * tables, s, c, cg);
                spread<VEC, UNIT>(B, B_of + k * tables, s, c, cg);
                read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, point(k), cg);
                const Correction<VEC> dx_of(A, B, share);
#pragma unroll
                for (int v = 0; v < VEC; ++v) h[v] = dx_of(g, g.h(h[v], v), dz[k][v], v);
                const Walk<BF16, VEC> dx(a.dx, point(k), s.ty, c.first + s.at, t.down);
                C::store(dx.base + dx.offset, C::narrow(h));
            }
        }
        // the next step's sums are put where this one's were read before the last barrier, and its results written after another one
    }
    if (!parts_gamma) return;
    __syncthreads();
    auto give = [&](float *parts) { return [=](int col, float total) { parts[int64_t(blockIdx.x) * a.shape.channels + c.first + col] = total; }; };
    const int row = s.side * t.down + s.ty, rows = t.side * t.down;
    add_columns(sum_gamma, s.has, s.at, row, rows, c.width, lds, give(parts_gamma));
    add_columns(sum_beta, s.has, s.at, row, rows, c.width, lds, give(parts_beta));
}

// ---- pieces of a point's groups ------------------------------------------------------------------------------------------------------------
// parts[((point * tiles + tile) * pieces + piece) * (most groups of a tile) + group] = a pair of sums; forward: mean and M2, backward: A and B before
// they are divided.
struct Parts {
    f2 *pair;
    int stride;                  // most groups of a tile
    __device__ __forceinline__ int64_t at(const Tiling &t, int64_t point, int tile, int piece) const { return ((point * t.tiles + tile) * t.pieces + piece) * stride; }
};
// Folds f over the pieces (and slices) of every group of the tile; f(pair, values of the piece) per piece, by lanes that share a group.  Leaves F's
// results in the tables `one` and `two`.
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
// A thread's own mean and squared distances first, step by step, then the workgroup's about its mean: sum of (M2 + n (mean - all)^2).
template <bool BF16, int VEC, int UNIT> __global__ void __launch_bounds__(256) norm_part_forward_kernel(NormArgs a, Tiling t, Parts parts, int64_t first_point)
{
    constexpr int U = 4, NV = VEC / UNIT;
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, piece = blockIdx.x % t.pieces;
    const int64_t local = blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    const int cg_tile = t.slices == 1 ? cg : c.width;    // a slice is all that a tile has of its group
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg_tile};
    float *mean_of = lds + t.threads * NV, *m2_of = mean_of + c.groups;
    const Stretch stretch = stretch_of(t, piece, s.ty, a.shape.positions);
    Walk<BF16, VEC> x(a.x, n, stretch.first, c.first + s.at, t.down);
    float mean[NV], m2[NV], have = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) mean[i] = m2[i] = 0.f;
    for (int left = stretch.left; left > 0; left -= U, x.advance(U)) {
        typename C::raw raw[U];
        load_step<false>(raw, x, left);
        hold_step(raw);
        auto step = [&](auto all) {
            const int rows = all() ? U : left;
            float v[U][VEC], sum[NV];
#pragma unroll
            for (int i = 0; i < NV; ++i) sum[i] = 0.f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (!all() && u >= rows) break;
                C::widen(raw[u], v[u]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum[i / UNIT] += v[u][i];
            }
            const float fresh = static_cast<float>(rows * UNIT), share = 1.f / fresh, total = have + fresh;
            const float part = fresh / total;
            const float weight = have * part;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float m = sum[i] * share, apart = m - mean[i];
                float q = 0.f;
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (all() || u < rows) {
#pragma unroll
                        for (int j = 0; j < UNIT; ++j) {
                            const float d = v[u][i * UNIT + j] - m;
                            q = fmaf(d, d, q);
                        }
                    }
                mean[i] = fmaf(apart, part, mean[i]);
                m2[i] += fmaf(apart * apart, weight, q);
            }
            have = total;
        };
        if (left >= U) step(std::true_type());
        else step(std::false_type());
    }
    float brought[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) brought[i] = have * mean[i];
    sums(s, brought, mean_of);
    const int rows = min(t.down * t.k, a.shape.positions - piece * t.down * t.k);
    const float count = static_cast<float>(rows) * (c.width / c.groups);
    for (int g = threadIdx.x; g < c.groups; g += blockDim.x) mean_of[g] /= count;
    __syncthreads();
    float all[VEC];
    spread<VEC, UNIT>(all, mean_of, s, c, cg_tile);
#pragma unroll
    for (int i = 0; i < NV; ++i) brought[i] = have > 0.f ? fmaf(have * (mean[i] - all[i * UNIT]), mean[i] - all[i * UNIT], m2[i]) : 0.f;
    sums(s, brought, m2_of);
    for (int g = threadIdx.x; g < c.groups; g += blockDim.x) parts.pair[parts.at(t, local, tile, piece) + g] = f2{mean_of[g], m2_of[g]};
}

template <bool BF16, int VEC, int UNIT, int ACT> __global__ void __launch_bounds__(256) norm_join_forward_kernel(NormArgs a, Tiling t, Parts parts, int64_t first_point)
{
    constexpr int U = 4;
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y;
    const int piece = t.pieces - 1 - static_cast<int>(blockIdx.x % t.pieces);            // the last ones read are the likeliest in the caches
    const int64_t local = gridDim.x / t.pieces - 1 - blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    float *mean = lds, *rstd = mean + c.groups;
    const Stretch stretch = stretch_of(t, piece, s.ty, a.shape.positions);
    Walk<BF16, VEC> x(a.x, n, stretch.first, c.first + s.at, t.down), y(a.y, n, stretch.first, c.first + s.at, t.down);
    typename C::raw raw[U];
    load_step<true>(raw, x, stretch.left);               // on its way while the statistics are joined
    join_parts(parts, t, c, n, tile, [&](int g, int lane, int lanes, int first_tile) {
        // the values of piece i of slice j: rows times columns
        auto values = [&](int i, int j) {
            const int rows = min(t.down * t.k, a.shape.positions - i * t.down * t.k);
            const int columns = t.slices == 1 ? cg : slice_begin(t, cg, j + 1) - slice_begin(t, cg, j);
            return static_cast<double>(rows) * columns;
        };
        const double all = static_cast<double>(a.shape.positions) * cg;
        const int entries = t.pieces * t.slices;
        double sum = 0.0;
        for (int e = lane; e < entries; e += lanes) sum += values(e % t.pieces, e / t.pieces) * parts.pair[parts.at(t, local, first_tile + e / t.pieces, e % t.pieces) + g].x;
        for (int o = 1; o < lanes; o *= 2) sum += __shfl_xor(sum, o, 64);
        const double m = sum / all;
        sum = 0.0;
        for (int e = lane; e < entries; e += lanes) {
            const f2 p = parts.pair[parts.at(t, local, first_tile + e / t.pieces, e % t.pieces) + g];
            sum += p.y + values(e % t.pieces, e / t.pieces) * (p.x - m) * (p.x - m);
        }
        for (int o = 1; o < lanes; o *= 2) sum += __shfl_xor(sum, o, 64);
        if (lane == 0) {
            mean[g] = static_cast<float>(m);
            rstd[g] = 1.f / sqrtf(static_cast<float>(sum / all) + a.eps);
            if (a.mean && piece == 0 && tile == first_tile) {
                a.mean[n * a.groups + c.group + g] = mean[g];
                a.rstd[n * a.groups + c.group + g] = rstd[g];
            }
        }
    });
    __syncthreads();
    if (!s.has) return;
    float m[VEC], r[VEC];
    const int cg_tile = t.slices == 1 ? cg : c.width;
    spread<VEC, UNIT>(m, mean, s, c, cg_tile);
    spread<VEC, UNIT>(r, rstd, s, c, cg_tile);
    const Finish<BF16, VEC, ACT> finish(a, c.first + s.at, m, r);
    for (int left = stretch.left; left > 0; left -= U) {
        hold_step(raw);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= left) break;
            float v[VEC];
            C::widen(raw[u], v);
            finish(v);
            put_chunk<BF16, VEC>(y.at(u), v, c, s);
        }
        if (left <= U) break;
        x.advance(U);
        y.advance(U);
        load_step<true>(raw, x, left - U);
    }
}

template <bool BF16, int VEC, int UNIT, int ACT>
__global__ void __launch_bounds__(256) norm_part_backward_kernel(NormGradArgs a, Tiling t, Parts parts, int64_t first_point, float *parts_gamma, float *parts_beta)
{
    constexpr int U = 4, NV = VEC / UNIT;
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, piece = blockIdx.x % t.pieces;
    const int64_t local = blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    const int cg_tile = t.slices == 1 ? cg : c.width;
    GroupSum<VEC, UNIT> sums = {lds, t, c, cg_tile};
    const int room = t.threads * NV;
    float *A_of = lds + 2 * room, *B_of = A_of + c.groups;
    const Stretch stretch = stretch_of(t, piece, s.ty, a.shape.positions);
    Walk<BF16, VEC> x(a.x, n, stretch.first, c.first + s.at, t.down), dy(a.dy, n, stretch.first, c.first + s.at, t.down);
    Gradient<BF16, VEC, ACT> g;
    float s1[VEC], s2[VEC];
    read_floats(g.gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(g.beta, a.beta, c.first + s.at, 0.f);
    read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, n, cg);
#pragma unroll
    for (int v = 0; v < VEC; ++v) s1[v] = s2[v] = 0.f;
    for (int left = stretch.left; left > 0; left -= U, x.advance(U), dy.advance(U)) {
        typename C::raw raw[U], raw_d[U];
        load_step<false>(raw, x, left);
        load_step<false>(raw_d, dy, left);
        hold_step(raw);
        hold_step(raw_d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= left) break;
            float h[VEC], d[VEC];
            C::widen(raw[u], h);
            C::widen(raw_d[u], d);
            g.slopes(h, d);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                s1[v] += d[v];
                s2[v] = fmaf(d[v], h[v], s2[v]);
            }
        }
    }
    if (parts_gamma) {
        auto give = [&](float *to) { return [=](int col, float total) { to[int64_t(blockIdx.x) * a.shape.channels + c.first + col] = total; }; };
        add_columns(s2, s.has, s.at, s.ty, t.down, c.width, lds, give(parts_gamma));
        add_columns(s1, s.has, s.at, s.ty, t.down, c.width, lds, give(parts_beta));
    }
    bring<VEC, UNIT>(sums, s, g.gamma, s1, s2, room, A_of, B_of);
    for (int q = threadIdx.x; q < c.groups; q += blockDim.x) parts.pair[parts.at(t, local, tile, piece) + q] = f2{A_of[q], B_of[q]};
}

template <bool BF16, int VEC, int UNIT, int ACT> __global__ void __launch_bounds__(256) norm_join_backward_kernel(NormGradArgs a, Tiling t, Parts parts, int64_t first_point)
{
    constexpr int U = 4;
    using C = Chunk<BF16, VEC>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y;
    const int piece = t.pieces - 1 - static_cast<int>(blockIdx.x % t.pieces);
    const int64_t local = gridDim.x / t.pieces - 1 - blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    float *A_of = lds, *B_of = A_of + c.groups;
    const Stretch stretch = stretch_of(t, piece, s.ty, a.shape.positions);
    Walk<BF16, VEC> x(a.x, n, stretch.first, c.first + s.at, t.down), dy(a.dy, n, stretch.first, c.first + s.at, t.down), dx(a.dx, n, stretch.first, c.first + s.at, t.down);
    typename C::raw raw[U], raw_d[U];
    load_step<true>(raw, x, stretch.left);
    load_step<true>(raw_d, dy, stretch.left);
    const double all = static_cast<double>(a.shape.positions) * cg;
    join_parts(parts, t, c, n, tile, [&](int g, int lane, int lanes, int first_tile) {
        double sum_A = 0.0, sum_B = 0.0;
        for (int e = lane; e < t.pieces * t.slices; e += lanes) {
            const f2 p = parts.pair[parts.at(t, local, first_tile + e / t.pieces, e % t.pieces) + g];
            sum_A += p.x;
            sum_B += p.y;
        }
        for (int o = 1; o < lanes; o *= 2) {
            sum_A += __shfl_xor(sum_A, o, 64);
            sum_B += __shfl_xor(sum_B, o, 64);
        }
        if (lane == 0) {
            A_of[g] = static_cast<float>(sum_A / all);
            B_of[g] = static_cast<float>(sum_B / all);
        }
    });
    Gradient<BF16, VEC, ACT> g;
    float A[VEC], B[VEC];
    read_floats(g.gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(g.beta, a.beta, c.first + s.at, 0.f);
    read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, n, cg);
    __syncthreads();
    if (!s.has) return;
    const int cg_tile = t.slices == 1 ? cg : c.width;
    spread<VEC, UNIT>(A, A_of, s, c, cg_tile);
    spread<VEC, UNIT>(B, B_of, s, c, cg_tile);
    const Correction<VEC> dx_of(A, B, 1.f);
    for (int left = stretch.left; left > 0; left -= U) {
        hold_step(raw);
        hold_step(raw_d);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (u >= left) break;
            float h[VEC], d[VEC];
            C::widen(raw[u], h);
            C::widen(raw_d[u], d);
            g.slopes(h, d);
#pragma unroll
            for (int v = 0; v < VEC; ++v) d[v] = dx_of(g, h[v], d[v], v);
            put_chunk<BF16, VEC>(dx.at(u), d, c, s);
        }
        if (left <= U) break;
        x.advance(U);
        dy.advance(U);
        dx.advance(U);
        load_step<true>(raw, x, left - U);
        load_step<true>(raw_d, dy, left - U);
    }
}

// ---- which of them ----------------------------------------------------------------------------------------------------------------------------
// Rows of one position whose groups are whole chunks, a power of two of them: lanes per group, or 0.
int lanes_per_group(const LayerShape &s, int groups)
{
    const int vec = s.bf16 ? 8 : 4, cg = s.channels / groups, lanes = cg / vec;
    return s.positions == 1 && cg % vec == 0 && lanes <= 64 && (lanes & (lanes - 1)) == 0 ? lanes : 0;
}
// chunks of a row that a workgroup of norm_rows has: whole groups, as even as can be
int across_of(const LayerShape &s, int lanes)
{
    const int chunks = s.channels / (s.bf16 ? 8 : 4), tiles = (chunks + 255) / 256;
    return (chunks / lanes + tiles - 1) / tiles * lanes;
}

int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

constexpr int kMostGroups = 4096;                        // sums of a workgroup: with what they are made from they fit 64 KB of LDS
constexpr int kPartThreads = 256;                        // of norm_part_* and norm_join_*
constexpr int kForwardThreads = 1024, kBackwardThreads = 256;           // of norm_tile_*, at most; chunks of a thread: 8

int vec_of(const LayerShape &s) { return s.channels < (s.bf16 ? 8 : 4) ? 1 : s.bf16 ? 8 : 4; }
int across_for(const LayerShape &s, int groups, int tiles) { return ceil_div(int64_t(ceil_div(groups, tiles)) * (s.channels / groups), vec_of(s)); }
// Whether the seats of a column can be added up inside a wavefront; rounds `down` for it where there is room.
void fold_columns(Tiling *t)
{
    t->fold = 0;
    if (t->across > 32 || (t->across & (t->across - 1)) != 0) return;
    const int step = 64 / t->across, down = (t->down + step - 1) / step * step;
    if (t->side > 1 ? t->down % step != 0 : down * t->across > t->threads) return;
    t->down = t->side > 1 ? t->down : down;
    t->fold = 1;
}

// Tiles in registers: at most so many threads and chunks of each; k == 0: the point is too large, and is cut into pieces.  Small workgroups, of which
// several share a compute unit and one loads while others add up; so tiles get narrower (down to a cache line of columns) before they get more threads,
// and more threads rather than more chunks each where there are few of them.
Tiling tile(const LayerShape &s, int groups, bool backward)
{
    const int most_threads = backward ? kBackwardThreads : kForwardThreads, most_chunks = 8, vec = vec_of(s);
    const int cg = s.channels / groups, line = std::max(1, 128 / (cg * (s.bf16 ? 2 : 4)));
    Tiling t = {};
    t.slices = t.unit = t.side = t.pieces = 1;
    const int most_tiles = std::max(1, groups / line);
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
        while (t.threads < most_threads && s.points * tiles < 2 * kUnits && !fits(t.threads, 1, tiles)) t.threads *= 2;
        t.tiles = tiles;
        t.across = across_for(s, groups, tiles);
        t.k = 1;
        while (int64_t(t.threads / t.across) * t.k < s.positions) t.k *= 2;
        t.down = ceil_div(s.positions, t.k);             // as even as can be
        t.side = std::max(1, std::min(t.threads / (t.across * t.down), kMostGroups / ceil_div(groups, tiles)));
        t.side = static_cast<int>(std::min<int64_t>(t.side, std::max<int64_t>(1, s.points)));
        fold_columns(&t);
        // one position each: several points each, so long as there are enough for all workgroups and LDS for their sums
        if (t.k == 1 && t.threads <= 512) {
            const int values = cg % vec == 0 ? 1 : cg == vec / 2 ? 2 : vec;
            auto room = [&](int deep) { return (size_t(deep) * t.threads * values + size_t(2) * deep * t.side * ceil_div(groups, tiles)) * (backward ? 2 : 1) * sizeof(float); };
            // (the gradient of four, with a sum per channel, is more than the registers hold)
            for (int deep = backward && values > 1 ? 2 : 4; deep > 1 && !t.deep; deep /= 2)
                if (room(deep) <= size_t(48) << 10 && s.points * tiles >= int64_t(4) * kUnits * t.side * deep) t.deep = deep;
        }
        return t;
    }
    return t;
}
Tiling cut(const LayerShape &s, int groups)
{
    const int vec = vec_of(s), cg = s.channels / groups;
    Tiling t = {};
    t.side = t.slices = 1;
    t.threads = kPartThreads;
    t.unit = cg % vec == 0 ? vec : 1;
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
int most_groups(const Tiling &t, int groups) { return t.slices > 1 ? 1 : ceil_div(groups, t.tiles); }

// Points of a pair of launches: as many as a grid takes.  (Fewer, so that what is read twice comes from the last-level cache, cost more at the launches' ends
// than they gain: 64 x 4 096 x 512 bf16, points of 96 MB at a time / of 192 / all: forward 213 / 196 / 176 us, backward 365 / 320 / 279.)
int64_t batch_points(const LayerShape &s, const Tiling &t) { return std::max<int64_t>(1, std::min<int64_t>(s.points, (int64_t(1) << 22) / t.pieces)); }

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
    auto with = [&](auto bf16, auto v) {                 // a load's, half a load's, one
        constexpr int V = v(), HALF = V > 1 ? V / 2 : 1;
        if (cg % V == 0) f(bf16, v, v);
        else if (cg == HALF) f(bf16, v, std::integral_constant<int, HALF>());
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
template <typename F> void with_lanes(int lanes, F f)
{
    switch (lanes) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    case 8: f(std::integral_constant<int, 8>()); break;
    case 16: f(std::integral_constant<int, 16>()); break;
    case 32: f(std::integral_constant<int, 32>()); break;
    default: f(std::integral_constant<int, 64>()); break;
    }
}

// points of a workgroup of norm_rows
int64_t rows_of_workgroup(const LayerShape &s, int across, int workgroups_per_unit, int steps)
{
    const int64_t tiles = ceil_div(s.channels / (s.bf16 ? 8 : 4), across), step = 256 / across * 4;
    int64_t length = (s.points * tiles + kUnits * workgroups_per_unit - 1) / (kUnits * workgroups_per_unit);
    length = (length + step - 1) / step * step;
    return std::max<int64_t>({1, length, std::min(step * steps, (s.points + step - 1) / step * step)});
}
// points of a piece: a workgroup's sums of the parameters' gradients are over so many that they are little beside what it reads
int64_t points_of_piece(const LayerShape &s, const Tiling &t)
{
    const int64_t wanted = std::max<int64_t>(1, kUnits * 8 / t.tiles);
    int64_t length = std::max<int64_t>((s.points + wanted - 1) / wanted, std::min<int64_t>(32 / std::min(s.positions, 32), (s.points + kUnits - 1) / kUnits));
    const int at_once = t.side * std::max(t.deep, 1);
    return std::max<int64_t>((length + at_once - 1) / at_once * at_once, 1);
}

struct BackwardPlan {
    int lanes;                   // of norm_rows, or 0
    bool cut;                    // norm_part and norm_join
    Tiling t;
    int64_t units_per_point, length;                     // of the pieces
};
BackwardPlan plan_backward(const LayerShape &s, int groups)
{
    BackwardPlan p = {};
    p.units_per_point = 1;
    p.lanes = lanes_per_group(s, groups);
    if (p.lanes) {
        p.length = rows_of_workgroup(s, across_of(s, p.lanes), 4, 4);
        return p;
    }
    p.t = tile(s, groups, true);
    if (p.t.k) {
        p.length = points_of_piece(s, p.t);
        return p;
    }
    p.cut = true;
    p.t = cut(s, groups);
    p.units_per_point = p.t.pieces;
    p.length = 1;
    return p;
}

size_t align_up(size_t v) { return (v + 255) / 256 * 256; }

// What a backward call keeps in its workspace: rows of the pieces' sums for dgamma and dbeta, rows beside them, pairs of sums of the groups.
struct BackwardRoom {
    size_t table, beside, pairs;
    size_t bytes() const { return 2 * table + 2 * beside + pairs; }
};
BackwardRoom room_of(const LayerShape &s, int groups, const BackwardPlan &p, const int64_t *bounds, int runs)
{
    const int64_t most = most_pieces(bounds, runs, p.units_per_point, p.length), rows = p.cut ? s.points * p.units_per_point : most;
    BackwardRoom r;
    r.table = align_up(static_cast<size_t>(rows) * s.channels * sizeof(float));
    r.beside = align_up(static_cast<size_t>(rows_beside(most, runs)) * s.channels * sizeof(float));
    r.pairs = p.cut ? static_cast<size_t>(batch_points(s, p.t)) * p.t.tiles * p.t.pieces * most_groups(p.t, groups) * sizeof(f2) : 0;
    return r;
}

}  // namespace

size_t norm_forward_bytes(const LayerShape &s, int groups)
{
    if (s.points == 0 || lanes_per_group(s, groups) || tile(s, groups, false).k) return 0;
    const Tiling t = cut(s, groups);
    return static_cast<size_t>(batch_points(s, t)) * t.tiles * t.pieces * most_groups(t, groups) * sizeof(f2);
}

size_t norm_backward_bytes(const LayerShape &s, int groups, const int64_t *bounds, int runs)
{
    return s.points == 0 ? 0 : room_of(s, groups, plan_backward(s, groups), bounds, runs).bytes();
}

hipError_t launch_norm_forward(const NormArgs &a, void *workspace, hipStream_t stream)
{
    const LayerShape &s = a.shape;
    if (s.points == 0) return hipSuccess;
    if (const int lanes = lanes_per_group(s, a.groups)) {
        const int across = across_of(s, lanes);
        const int64_t length = rows_of_workgroup(s, across, 16, 1);
        const dim3 grid(ceil_div(s.channels / (s.bf16 ? 8 : 4), across), ceil_div(s.points, length));
        with_lanes(lanes, [&](auto l) {
            with_activation(a.activation, [&](auto act) {
                (s.bf16 ? norm_rows_forward_kernel<true, l(), act()> : norm_rows_forward_kernel<false, l(), act()>)<<<grid, 256, 0, stream>>>(a, across, length);
            });
        });
        return hipGetLastError();
    }
    const Tiling t = tile(s, a.groups, false);
    if (t.deep) {
        with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
            const int64_t at_once = t.side * t.deep;
            const dim3 grid(static_cast<unsigned>(std::min<int64_t>((s.points + at_once - 1) / at_once, 1 << 20)), t.tiles);
            const size_t lds = t.deep * (t.threads * (vec() / unit()) + 2 * t.side * most_groups(t, a.groups)) * sizeof(float);
            with_activation(a.activation, [&](auto act) {
                constexpr int B = bf16(), V = vec(), U = unit(), A = act();
                (t.deep == 4 ? norm_deep_forward_kernel<B, V, 4, U, A> : norm_deep_forward_kernel<B, V, 2, U, A>)<<<grid, t.threads, lds, stream>>>(a, t);
            });
        });
        return hipGetLastError();
    }
    if (t.k) {
        with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
            with_k(t.k, [&](auto k) {
                const dim3 grid(static_cast<unsigned>(std::min<int64_t>((s.points + t.side - 1) / t.side, 1 << 20)), t.tiles);
                const size_t lds = (t.threads * (vec() / unit()) + 2 * t.side * most_groups(t, a.groups)) * sizeof(float);
                with_activation(a.activation, [&](auto act) {
                    constexpr int B = bf16(), V = vec(), K = k(), U = unit(), A = act();
                    (t.threads > 512 || K < 8 ? norm_tile_forward_kernel<B, V, K, U, A, 1024> : norm_tile_forward_kernel<B, V, K, U, A, K < 8 ? 1024 : 512>)<<<grid, t.threads, lds, stream>>>(a, t);
                });
            });
        });
        return hipGetLastError();
    }
    const Tiling c = cut(s, a.groups);
    const Parts parts = {static_cast<f2 *>(workspace), most_groups(c, a.groups)};
    const int64_t batch = batch_points(s, c);
    for (int64_t n = 0; n < s.points; n += batch) {
        const dim3 grid(static_cast<unsigned>(std::min(batch, s.points - n) * c.pieces), c.tiles);
        with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
            const size_t tables = 2 * parts.stride * sizeof(float), lds = c.threads * (vec() / unit()) * sizeof(float) + tables;
            norm_part_forward_kernel<bf16(), vec(), unit()><<<grid, c.threads, lds, stream>>>(a, c, parts, n);
            with_activation(a.activation, [&](auto act) { norm_join_forward_kernel<bf16(), vec(), unit(), act()><<<grid, c.threads, tables, stream>>>(a, c, parts, n); });
        });
    }
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormGradArgs &a, void *workspace, hipStream_t stream)
{
    const LayerShape &s = a.shape;
    const bool sums = a.dgamma || a.dbeta;
    if (!sums && (!a.dx.p || s.points == 0)) return hipSuccess;
    BackwardPlan p = {};
    p.units_per_point = p.length = 1;
    float *parts_gamma = nullptr, *parts_beta = nullptr, *beside = nullptr;
    if (s.points > 0) {
        p = plan_backward(s, a.groups);
        const BackwardRoom room = room_of(s, a.groups, p, a.bounds, a.runs);
        char *at = static_cast<char *>(workspace);
        if (sums) {
            parts_gamma = reinterpret_cast<float *>(at);
            parts_beta = reinterpret_cast<float *>(at + room.table);
            beside = reinterpret_cast<float *>(at + 2 * room.table);
        }
        if (p.cut) {
            const Tiling &t = p.t;
            const Parts parts = {reinterpret_cast<f2 *>(at + 2 * room.table + 2 * room.beside), most_groups(t, a.groups)};
            const int64_t batch = batch_points(s, t);
            for (int64_t n = 0; n < s.points; n += batch) {
                const dim3 grid(static_cast<unsigned>(std::min(batch, s.points - n) * t.pieces), t.tiles);
                with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
                    const size_t tables = 2 * parts.stride * sizeof(float), columns = t.threads * vec() * sizeof(float);
                    const size_t lds = std::max(2 * t.threads * (vec() / unit()) * sizeof(float) + tables, columns);
                    float *to_gamma = sums ? parts_gamma + n * t.pieces * s.channels : nullptr, *to_beta = sums ? parts_beta + n * t.pieces * s.channels : nullptr;
                    with_activation(a.activation, [&](auto act) {
                        norm_part_backward_kernel<bf16(), vec(), unit(), act()><<<grid, t.threads, lds, stream>>>(a, t, parts, n, to_gamma, to_beta);
                        if (a.dx.p) norm_join_backward_kernel<bf16(), vec(), unit(), act()><<<grid, t.threads, tables, stream>>>(a, t, parts, n);
                    });
                });
            }
        }
    }
    for (int r = 0; r < a.runs; r += Pieces::kRuns) {
        Pieces pieces;
        const int count = lay_out_pieces(a.bounds + r, std::min(Pieces::kRuns, a.runs - r), p.units_per_point, p.length, &pieces);
        const float *from_gamma = parts_gamma, *from_beta = parts_beta;
        if (p.cut && sums) {                             // rows of all pieces lie in one table
            from_gamma += pieces.first[0] * s.channels;
            from_beta += pieces.first[0] * s.channels;
        } else if (p.cut) {
            break;
        } else if (count > 0 && p.lanes) {
            const int across = across_of(s, p.lanes);
            const dim3 grid(ceil_div(s.channels / (s.bf16 ? 8 : 4), across), count);
            with_lanes(p.lanes, [&](auto l) {
                with_activation(a.activation, [&](auto act) {
                    (s.bf16 ? norm_rows_backward_kernel<true, l(), act()> : norm_rows_backward_kernel<false, l(), act()>)<<<grid, 256, 0, stream>>>(a, across, pieces, parts_gamma, parts_beta);
                });
            });
        } else if (count > 0) {
            const Tiling &t = p.t;
            if (t.deep) {
                with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
                    const size_t columns = t.threads * vec() * sizeof(float);
                    const size_t lds = std::max(2 * t.deep * (t.threads * (vec() / unit()) + t.side * most_groups(t, a.groups)) * sizeof(float), columns);
                    with_activation(a.activation, [&](auto act) {
                        constexpr int B = bf16(), V = vec(), U = unit(), A = act();
                        (t.deep == 4 ? norm_deep_backward_kernel<B, V, U == V ? 4 : 2, U, A> : norm_deep_backward_kernel<B, V, 2, U, A>)
                            <<<dim3(count, t.tiles), t.threads, lds, stream>>>(a, t, pieces, parts_gamma, parts_beta);
                    });
                });
            } else with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
                with_k(t.k, [&](auto k) {
                    const size_t columns = t.threads * vec() * sizeof(float);
                    const size_t lds = std::max((2 * t.threads * (vec() / unit()) + 2 * t.side * most_groups(t, a.groups)) * sizeof(float), columns);
                    with_activation(a.activation, [&](auto act) {
                        norm_tile_backward_kernel<bf16(), vec(), k(), unit(), act()><<<dim3(count, t.tiles), t.threads, lds, stream>>>(a, t, pieces, parts_gamma, parts_beta);
                    });
                });
            });
        }
        if (sums)
            launch_sum_pieces(from_gamma, from_beta, s.channels, pieces, beside, a.dgamma ? a.dgamma + int64_t(r) * s.channels : nullptr,
                              a.dbeta ? a.dbeta + int64_t(r) * s.channels : nullptr, stream);
    }
    return hipGetLastError();
}

}  // namespace cr

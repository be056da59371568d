// Group norm with an activation, channels last, for gfx950.
//
// A thread has a chunk of 16 bytes of channels and goes down a point's positions, so that its gamma, beta and statistics stay in registers.  Sums over a
// group meet in LDS.  The variance is the mean of squared distances from the mean, taken from registers in a second step, never a difference of large
// sums; tiles of a group that several workgroups have meet by  M2 = sum M2_i + n_i (mean_i - mean)^2.
//
//   norm_rows_*    points of one position, groups of 1 to 64 chunks, a power of two: a group is a few lanes, no workgroup meets
//   norm_tile_*    a point's group (or some of them, or several points) in the registers of a workgroup, read once
//   norm_part_*, norm_join_*   larger groups: pieces of a group leave their sums, then every piece is read again
#include "runs_device.h"

namespace cr {

namespace {

constexpr int kUnits = 256;

// act(z), and d act'(z) from d and z
template <int VEC> __device__ __forceinline__ void activate(int kind, float (&z)[VEC])
{
    if (kind == 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) z[v] = z[v] < 0.f ? 0.f : z[v];
    } else if (kind == 2) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) z[v] = z[v] * __builtin_amdgcn_rcpf(1.f + __expf(-z[v]));
    }
}
template <int VEC> __device__ __forceinline__ void through_slope(int kind, const float (&z)[VEC], float (&d)[VEC])
{
    if (kind == 1) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) d[v] = z[v] > 0.f ? d[v] : z[v] <= 0.f ? 0.f : z[v];                // not 0 where z is not a number
    } else if (kind == 2) {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            const float s = __builtin_amdgcn_rcpf(1.f + __expf(-z[v]));
            d[v] *= s * fmaf(z[v], 1.f - s, 1.f);
        }
    }
}
template <int VEC> __device__ __forceinline__ void read_floats(float (&out)[VEC], const float *p, int at, float otherwise)
{
#pragma unroll
    for (int v = 0; v < VEC; ++v) out[v] = p ? p[at + v] : otherwise;
}

// ---- points of one position, groups of a few lanes ---------------------------------------------------------------------------------------
// A thread stays with its chunk and goes through the points, U at a time.  Its group is the LANES lanes around it.
template <bool BF16, int LANES> __global__ void __launch_bounds__(256) norm_rows_forward_kernel(NormArgs a, int across, int64_t length)
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
            for (int i = 0; i < VEC; ++i) v[i] = fmaf(v[i] * rstd, gamma[i], beta[i]);
            activate(a.activation, v);
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

template <bool BF16, int LANES>
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
                float h[VEC], d[VEC], z[VEC], A = 0.f, B = 0.f;
                C::widen(raw[u], h);
                C::widen(raw_d[u], d);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    h[i] = (h[i] - mean[u]) * rstd[u];
                    z[i] = fmaf(h[i], gamma[i], beta[i]);
                }
                through_slope(a.activation, z, d);
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
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
                    d[i] = rstd[u] * (fmaf(gamma[i], d[i], -A) - h[i] * B);
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

// Sums over the groups of a tile.  Each thread brings one value, of a chunk that lies in one group (WIDE), or VEC of them, one for each channel; the sum over
// the rows and the channels of a group goes to out[side * groups + group], where every thread finds it after the call.
template <int VEC, bool WIDE> struct GroupSum {
    float *lds;                  // threads * (WIDE ? 1 : VEC) floats
    const Tiling &t;
    const Columns &c;
    int cg;
    __device__ __forceinline__ void put(const Seat &s, const float (&value)[VEC], float *to)
    {
        const int row = s.side * t.down + s.ty;
        if (!s.has) return;
        if constexpr (WIDE) {
            float sum = 0.f;
#pragma unroll
            for (int v = 0; v < VEC; ++v) sum += value[v];
            to[row * (c.width / VEC) + s.at / VEC] = sum;
        } else {
#pragma unroll
            for (int v = 0; v < VEC; ++v) to[row * c.width + s.at + v] = value[v];
        }
    }
    // lanes per sum: a power of two, so that the sums share out the workgroup's threads
    __device__ __forceinline__ void add(const float *from, float *out)
    {
        const int per = WIDE ? cg / VEC : cg, width = WIDE ? c.width / VEC : c.width, sums = t.side * c.groups;
        int lanes = 64;
        while (lanes > 1 && lanes * sums > static_cast<int>(blockDim.x)) lanes /= 2;
        const int lane = threadIdx.x % lanes, step_row = lanes / per, step_col = lanes % per;
        for (int q = threadIdx.x / lanes; q < sums; q += blockDim.x / lanes) {
            const int side = q / c.groups, g = q % c.groups;
            const float *base = from + side * t.down * width + g * per;
            int row = lane / per, col = lane % per;
            float sum = 0.f;
            while (row < t.down) {
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
    __device__ __forceinline__ void operator()(const Seat &s, const float (&value)[VEC], float *out)
    {
        put(s, value, lds);
        __syncthreads();
        add(lds, out);
        __syncthreads();
    }
};
// what the groups' table has for the channels of a seat
template <int VEC, bool WIDE> __device__ __forceinline__ void spread(float (&out)[VEC], const float *table, const Seat &s, const Columns &c, int cg)
{
    const int first = s.side * c.groups;
    if constexpr (WIDE) {
        const float v = table[first + s.at / cg];
#pragma unroll
        for (int i = 0; i < VEC; ++i) out[i] = v;
    } else {
        int g = s.at / cg, r = s.at % cg;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            out[i] = table[first + g];
            if (++r == cg) {
                r = 0;
                ++g;
            }
        }
    }
}

template <bool BF16, int VEC, int K> struct TileLoad {
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    // positions first + ty + k down of a point (past the last one: the last one, not counted), the chunk at channel `channel`
    template <bool ONCE> static __device__ __forceinline__ void load(typename C::raw (&raw)[K], const Rows &v, int64_t point, int64_t first, int down, int positions, int channel)
    {
        const T *p = static_cast<const T *>(v.p) + point * v.point_stride + channel;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const T *at = p + min(first + k * down, int64_t(positions - 1)) * v.position_stride;
            raw[k] = ONCE ? C::load_once(at) : C::load(at);
        }
    }
};

// The mean and the sum of squared distances from it, for the groups of a tile: mean[side * groups + group], M2 likewise.
template <bool BF16, int VEC, int K, bool WIDE>
__device__ __forceinline__ void tile_moments(const typename Chunk<BF16, VEC>::raw (&raw)[K], const Seat &s, int64_t first, int positions, const Tiling &t, const Columns &c,
                                             int cg, float count, GroupSum<VEC, WIDE> &sums, float *mean, float *m2)
{
    using C = Chunk<BF16, VEC>;
    float sum[VEC], m[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (first + k * t.down < positions) {
            float x[VEC];
            C::widen(raw[k], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) sum[v] += x[v];
        }
    }
    sums(s, sum, mean);
    for (int q = threadIdx.x; q < t.side * c.groups; q += blockDim.x) mean[q] /= count;
    __syncthreads();
    spread<VEC, WIDE>(m, mean, s, c, cg);
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (first + k * t.down < positions) {
            float x[VEC];
            C::widen(raw[k], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                x[v] -= m[v];
                sum[v] = fmaf(x[v], x[v], sum[v]);
            }
        }
    }
    sums(s, sum, m2);
}

// y from x in registers, with the tables of mean and 1 / deviation
template <bool BF16, int VEC, int K, bool WIDE>
__device__ __forceinline__ void tile_out(const typename Chunk<BF16, VEC>::raw (&raw)[K], const NormArgs &a, const Seat &s, int64_t point, int64_t first, const Tiling &t,
                                         const Columns &c, int cg, const float *mean, const float *rstd)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    float m[VEC], r[VEC], gamma[VEC], beta[VEC];
    spread<VEC, WIDE>(m, mean, s, c, cg);
    spread<VEC, WIDE>(r, rstd, s, c, cg);
    read_floats(gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(beta, a.beta, c.first + s.at, 0.f);
#pragma unroll
    for (int v = 0; v < VEC; ++v) gamma[v] *= r[v];
    T *y = static_cast<T *>(a.y.p) + point * a.y.point_stride + c.first + s.at;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t p = first + k * t.down;
        if (p < a.shape.positions) {
            float x[VEC];
            C::widen(raw[k], x);
#pragma unroll
            for (int v = 0; v < VEC; ++v) x[v] = fmaf(x[v] - m[v], gamma[v], beta[v]);
            activate(a.activation, x);
            C::store(y + p * a.y.position_stride, C::narrow(x));
        }
    }
}

template <bool BF16, int VEC, int K, bool WIDE> __global__ void __launch_bounds__(1024) norm_tile_forward_kernel(NormArgs a, Tiling t)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, WIDE> sums = {lds, t, c, cg};
    float *mean = lds + t.threads * (WIDE ? 1 : VEC), *rstd = mean + t.side * c.groups;
    const float count = static_cast<float>(a.shape.positions) * cg;
    for (int64_t n0 = int64_t(blockIdx.x) * t.side; n0 < a.shape.points; n0 += int64_t(gridDim.x) * t.side) {
        const int64_t n = n0 + s.side;
        typename Chunk<BF16, VEC>::raw raw[K];
        L::template load<true>(raw, a.x, min(n, a.shape.points - 1), s.ty, t.down, a.shape.positions, c.first + s.at);
        tile_moments<BF16, VEC, K, WIDE>(raw, s, s.ty, a.shape.positions, t, c, cg, count, sums, mean, rstd);
        for (int q = threadIdx.x; q < t.side * c.groups; q += blockDim.x) {
            rstd[q] = 1.f / sqrtf(rstd[q] / count + a.eps);
            const int64_t point = n0 + q / c.groups;
            if (a.mean && point < a.shape.points) {
                a.mean[point * a.groups + c.group + q % c.groups] = mean[q];
                a.rstd[point * a.groups + c.group + q % c.groups] = rstd[q];
            }
        }
        __syncthreads();
        if (s.has && n < a.shape.points) tile_out<BF16, VEC, K, WIDE>(raw, a, s, n, s.ty, t, c, cg, mean, rstd);
        __syncthreads();                                 // before the tables are another point's
    }
}

// h and gamma dz of a tile: what the sums and dx are made of.  kept[k] = dz, raw keeps x.
template <bool BF16, int VEC, int K, bool WIDE>
__device__ __forceinline__ void tile_slopes(const typename Chunk<BF16, VEC>::raw (&raw)[K], const typename Chunk<BF16, VEC>::raw (&raw_d)[K], float (&dz)[K][VEC],
                                            const NormGradArgs &a, int64_t first, const Tiling &t, const float (&m)[VEC], const float (&r)[VEC],
                                            const float (&gamma)[VEC], const float (&beta)[VEC], float (&s1)[VEC], float (&s2)[VEC])
{
    using C = Chunk<BF16, VEC>;
#pragma unroll
    for (int v = 0; v < VEC; ++v) s1[v] = s2[v] = 0.f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (first + k * t.down < a.shape.positions) {
            float h[VEC], z[VEC];
            C::widen(raw[k], h);
            C::widen(raw_d[k], dz[k]);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                h[v] = (h[v] - m[v]) * r[v];
                z[v] = fmaf(h[v], gamma[v], beta[v]);
            }
            through_slope(a.activation, z, dz[k]);
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                s1[v] += dz[k][v];
                s2[v] = fmaf(dz[k][v], h[v], s2[v]);
            }
        }
    }
}
template <bool BF16, int VEC, int K>
__device__ __forceinline__ void tile_dx(const typename Chunk<BF16, VEC>::raw (&raw)[K], const float (&dz)[K][VEC], const NormGradArgs &a, const Seat &s, const Columns &c,
                                        int64_t point, int64_t first, const Tiling &t, const float (&m)[VEC], const float (&r)[VEC], const float (&gamma)[VEC],
                                        const float (&A)[VEC], const float (&B)[VEC])
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    T *dx = static_cast<T *>(a.dx.p) + point * a.dx.point_stride + c.first + s.at;
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int64_t p = first + k * t.down;
        if (p < a.shape.positions) {
            float h[VEC];
            C::widen(raw[k], h);
#pragma unroll
            for (int v = 0; v < VEC; ++v) h[v] = r[v] * (fmaf(gamma[v], dz[k][v], -A[v]) - (h[v] - m[v]) * r[v] * B[v]);
            C::store(dx + p * a.dx.position_stride, C::narrow(h));
        }
    }
}
// mean and 1 / deviation of a seat's channels, from the tensors
template <int VEC, bool WIDE> __device__ __forceinline__ void read_stats(float (&m)[VEC], float (&r)[VEC], const NormGradArgs &a, const Seat &s, const Columns &c, int64_t point, int cg)
{
    const float *mean = a.mean + point * a.groups + c.group, *rstd = a.rstd + point * a.groups + c.group;
    Columns one = c;
    Seat seat = s;
    one.groups = 0;                                      // the tables are this point's
    seat.side = 0;
    const int within = c.first - c.group * cg;           // a slice of a group begins inside it
    seat.at += within;
    spread<VEC, WIDE>(m, mean, seat, one, cg);
    spread<VEC, WIDE>(r, rstd, seat, one, cg);
}

// A workgroup goes through the points of a piece of a run, `side` at a time.
template <bool BF16, int VEC, int K, bool WIDE>
__global__ void __launch_bounds__(512) norm_tile_backward_kernel(NormGradArgs a, Tiling t, Pieces pieces, float *parts_gamma, float *parts_beta)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups;
    const Columns c = columns_of(a.shape, a.groups, t, blockIdx.y);
    const Seat s = take_seat<VEC>(t, c);
    GroupSum<VEC, WIDE> sums = {lds, t, c, cg};
    const int room = t.threads * (WIDE ? 1 : VEC);
    float *A_of = lds + 2 * room, *B_of = A_of + t.side * c.groups;
    const float share = 1.f / (static_cast<float>(a.shape.positions) * cg);
    float gamma[VEC], beta[VEC], sum_gamma[VEC], sum_beta[VEC];
    read_floats(gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(beta, a.beta, c.first + s.at, 0.f);
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum_gamma[v] = sum_beta[v] = 0.f;
    const Piece piece = find_piece(pieces, blockIdx.x);
    for (int64_t n0 = piece.begin; n0 < piece.end; n0 += t.side) {
        const int64_t n = min(n0 + s.side, piece.end - 1);
        const bool live = s.has && n0 + s.side < piece.end;
        typename Chunk<BF16, VEC>::raw raw[K], raw_d[K];
        float dz[K][VEC], m[VEC], r[VEC], s1[VEC], s2[VEC], A[VEC], B[VEC];
        L::template load<true>(raw, a.x, n, s.ty, t.down, a.shape.positions, c.first + s.at);
        L::template load<true>(raw_d, a.dy, n, s.ty, t.down, a.shape.positions, c.first + s.at);
        read_stats<VEC, WIDE>(m, r, a, s, c, n, cg);
        tile_slopes<BF16, VEC, K, WIDE>(raw, raw_d, dz, a, s.ty, t, m, r, gamma, beta, s1, s2);
        if (live) {
#pragma unroll
            for (int v = 0; v < VEC; ++v) {
                sum_beta[v] += s1[v];
                sum_gamma[v] += s2[v];
            }
        }
        if (!a.dx.p) continue;
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            s1[v] *= gamma[v];
            s2[v] *= gamma[v];
        }
        sums.put(s, s1, lds);
        sums.put(s, s2, lds + room);
        __syncthreads();
        sums.add(lds, A_of);
        sums.add(lds + room, B_of);
        __syncthreads();
        spread<VEC, WIDE>(A, A_of, s, c, cg);
        spread<VEC, WIDE>(B, B_of, s, c, cg);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            A[v] *= share;
            B[v] *= share;
        }
        if (live) tile_dx<BF16, VEC, K>(raw, dz, a, s, c, n, s.ty, t, m, r, gamma, A, B);
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

template <bool BF16, int VEC, int K, bool WIDE> __global__ void __launch_bounds__(512) norm_part_forward_kernel(NormArgs a, Tiling t, Parts parts, int64_t first_point)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, piece = blockIdx.x % t.pieces;
    const int64_t local = blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    const int cg_tile = t.slices == 1 ? cg : c.width;    // a slice is all that a tile has of its group
    GroupSum<VEC, WIDE> sums = {lds, t, c, cg_tile};
    float *mean = lds + t.threads * (WIDE ? 1 : VEC), *m2 = mean + c.groups;
    const int64_t begin = int64_t(piece) * t.down * K, first = begin + s.ty;
    const float count = static_cast<float>(min(int64_t(t.down) * K, a.shape.positions - begin)) * (c.width / c.groups);
    typename Chunk<BF16, VEC>::raw raw[K];
    L::template load<false>(raw, a.x, n, first, t.down, a.shape.positions, c.first + s.at);
    tile_moments<BF16, VEC, K, WIDE>(raw, s, first, a.shape.positions, t, c, cg_tile, count, sums, mean, m2);
    for (int g = threadIdx.x; g < c.groups; g += blockDim.x) parts.pair[parts.at(t, local, tile, piece) + g] = f2{mean[g], m2[g]};
}

template <bool BF16, int VEC, int K, bool WIDE> __global__ void __launch_bounds__(512) norm_join_forward_kernel(NormArgs a, Tiling t, Parts parts, int64_t first_point)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y;
    const int piece = t.pieces - 1 - static_cast<int>(blockIdx.x % t.pieces);            // the last ones read are the likeliest in the caches
    const int64_t local = gridDim.x / t.pieces - 1 - blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    float *mean = lds, *rstd = mean + c.groups;
    const int64_t first = int64_t(piece) * t.down * K + s.ty;
    typename Chunk<BF16, VEC>::raw raw[K];
    L::template load<true>(raw, a.x, n, first, t.down, a.shape.positions, c.first + s.at);
    join_parts(parts, t, c, n, tile, [&](int g, int lane, int lanes, int first_tile) {
        // the values of piece i of slice j: rows times columns
        auto values = [&](int i, int j) {
            const int rows = min(t.down * K, a.shape.positions - i * t.down * K);
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
    if (s.has) tile_out<BF16, VEC, K, WIDE>(raw, a, s, n, first, t, c, t.slices == 1 ? cg : c.width, mean, rstd);
}

template <bool BF16, int VEC, int K, bool WIDE>
__global__ void __launch_bounds__(512) norm_part_backward_kernel(NormGradArgs a, Tiling t, Parts parts, int64_t first_point, float *parts_gamma, float *parts_beta)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y, piece = blockIdx.x % t.pieces;
    const int64_t local = blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    const int cg_tile = t.slices == 1 ? cg : c.width;
    GroupSum<VEC, WIDE> sums = {lds, t, c, cg_tile};
    const int room = t.threads * (WIDE ? 1 : VEC);
    float *A_of = lds + 2 * room, *B_of = A_of + c.groups;
    const int64_t first = int64_t(piece) * t.down * K + s.ty;
    typename Chunk<BF16, VEC>::raw raw[K], raw_d[K];
    float dz[K][VEC], m[VEC], r[VEC], s1[VEC], s2[VEC], gamma[VEC], beta[VEC];
    L::template load<false>(raw, a.x, n, first, t.down, a.shape.positions, c.first + s.at);
    L::template load<false>(raw_d, a.dy, n, first, t.down, a.shape.positions, c.first + s.at);
    read_floats(gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(beta, a.beta, c.first + s.at, 0.f);
    read_stats<VEC, WIDE>(m, r, a, s, c, n, cg);
    tile_slopes<BF16, VEC, K, WIDE>(raw, raw_d, dz, a, first, t, m, r, gamma, beta, s1, s2);
    if (parts_gamma) {
        auto give = [&](float *to) { return [=](int col, float total) { to[int64_t(blockIdx.x) * a.shape.channels + c.first + col] = total; }; };
        add_columns(s2, s.has, s.at, s.ty, t.down, c.width, lds, give(parts_gamma));
        add_columns(s1, s.has, s.at, s.ty, t.down, c.width, lds, give(parts_beta));
    }
#pragma unroll
    for (int v = 0; v < VEC; ++v) {
        s1[v] *= gamma[v];
        s2[v] *= gamma[v];
    }
    sums.put(s, s1, lds);
    sums.put(s, s2, lds + room);
    __syncthreads();
    sums.add(lds, A_of);
    sums.add(lds + room, B_of);
    __syncthreads();
    for (int g = threadIdx.x; g < c.groups; g += blockDim.x) parts.pair[parts.at(t, local, tile, piece) + g] = f2{A_of[g], B_of[g]};
}

template <bool BF16, int VEC, int K, bool WIDE> __global__ void __launch_bounds__(512) norm_join_backward_kernel(NormGradArgs a, Tiling t, Parts parts, int64_t first_point)
{
    using L = TileLoad<BF16, VEC, K>;
    extern __shared__ float lds[];
    const int cg = a.shape.channels / a.groups, tile = blockIdx.y;
    const int piece = t.pieces - 1 - static_cast<int>(blockIdx.x % t.pieces);
    const int64_t local = gridDim.x / t.pieces - 1 - blockIdx.x / t.pieces, n = first_point + local;
    const Columns c = columns_of(a.shape, a.groups, t, tile);
    const Seat s = take_seat<VEC>(t, c);
    float *A_of = lds, *B_of = A_of + c.groups;
    const int64_t first = int64_t(piece) * t.down * K + s.ty;
    typename Chunk<BF16, VEC>::raw raw[K], raw_d[K];
    float dz[K][VEC], m[VEC], r[VEC], s1[VEC], s2[VEC], gamma[VEC], beta[VEC], A[VEC], B[VEC];
    L::template load<true>(raw, a.x, n, first, t.down, a.shape.positions, c.first + s.at);
    L::template load<true>(raw_d, a.dy, n, first, t.down, a.shape.positions, c.first + s.at);
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
    read_floats(gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(beta, a.beta, c.first + s.at, 0.f);
    read_stats<VEC, WIDE>(m, r, a, s, c, n, cg);
    __syncthreads();
    const int cg_tile = t.slices == 1 ? cg : c.width;
    spread<VEC, WIDE>(A, A_of, s, c, cg_tile);
    spread<VEC, WIDE>(B, B_of, s, c, cg_tile);
    tile_slopes<BF16, VEC, K, WIDE>(raw, raw_d, dz, a, first, t, m, r, gamma, beta, s1, s2);
    if (s.has) tile_dx<BF16, VEC, K>(raw, dz, a, s, c, n, first, t, m, r, gamma, A, B);
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

constexpr int kPartChunks = 8, kPartThreads = 512;       // of norm_part_* and norm_join_*
constexpr int kMostGroups = 4096;                        // sums of a workgroup: with what they are made from they fit 64 KB of LDS

// Tiles in registers: at most `threads` threads with `k` chunks each; k == 0: the point is too large, and is cut into pieces.
Tiling tile(const LayerShape &s, int groups, int most_threads, int most_chunks)
{
    const int vec = s.channels < (s.bf16 ? 8 : 4) ? 1 : s.bf16 ? 8 : 4, e = s.bf16 ? 2 : 4, cg = s.channels / groups;
    Tiling t = {};
    t.slices = t.unit = 1;
    t.side = 1;
    t.pieces = 1;
    // narrowest tiles: whole groups, a cache line of columns
    const int least = std::min(groups, std::max(1, 128 / (cg * e)));
    const int most_tiles = std::max(1, groups / least);
    auto across_for = [&](int tiles) { return ceil_div(int64_t(ceil_div(groups, tiles)) * cg, vec); };
    // as few tiles as fit, more where there are few points
    int tiles = 1;
    auto fits = [&](int n) {
        return across_for(n) <= most_threads && ceil_div(groups, n) <= kMostGroups && int64_t(s.positions) <= int64_t(most_threads / across_for(n)) * most_chunks;
    };
    while (tiles < most_tiles && !fits(tiles)) tiles = std::min(most_tiles, tiles * 2);
    if (!fits(tiles)) return t;
    while (tiles < most_tiles && s.points * tiles < kUnits) tiles = std::min(most_tiles, tiles * 2);
    t.tiles = tiles;
    t.across = across_for(tiles);
    // few threads with many chunks each where there are many tiles, else many threads
    const bool many = s.points * tiles >= 4 * kUnits;
    t.threads = 256;
    for (;;) {
        const int down = t.threads / t.across;
        if (down > 0 && (int64_t(down) * (many ? most_chunks : 2) >= s.positions || t.threads == most_threads)) break;
        t.threads *= 2;
    }
    t.down = std::min(t.threads / t.across, s.positions);
    t.k = 1;
    while (int64_t(t.down) * t.k < s.positions) t.k *= 2;
    t.down = ceil_div(s.positions, t.k);                 // as even as can be
    t.side = std::max(1, std::min(t.threads / (t.across * t.down), kMostGroups / ceil_div(groups, tiles)));
    t.side = static_cast<int>(std::min<int64_t>(t.side, std::max<int64_t>(1, s.points)));
    return t;
}
Tiling cut(const LayerShape &s, int groups)
{
    const int vec = s.channels < (s.bf16 ? 8 : 4) ? 1 : s.bf16 ? 8 : 4, cg = s.channels / groups;
    Tiling t = {};
    t.side = t.slices = 1;
    t.threads = kPartThreads;
    t.k = kPartChunks;
    t.unit = cg % vec == 0 ? vec : 1;
    if (ceil_div(cg, vec) > t.threads) {                 // a group is wider than a workgroup
        t.slices = ceil_div(cg, int64_t(t.threads) * vec);
        t.tiles = groups * t.slices;
        t.across = ceil_div(int64_t(ceil_div(cg / t.unit, t.slices)) * t.unit, vec);
    } else {
        auto across_for = [&](int tiles) { return ceil_div(int64_t(ceil_div(groups, tiles)) * cg, vec); };
        t.tiles = ceil_div(ceil_div(s.channels, vec), t.threads);
        while (across_for(t.tiles) > t.threads) ++t.tiles;
        t.across = across_for(t.tiles);
    }
    t.down = t.threads / t.across;
    t.pieces = ceil_div(s.positions, int64_t(t.down) * t.k);
    t.down = ceil_div(ceil_div(s.positions, t.pieces), t.k);
    t.pieces = ceil_div(s.positions, int64_t(t.down) * t.k);
    return t;
}
int most_groups(const Tiling &t, int groups) { return t.slices > 1 ? 1 : ceil_div(groups, t.tiles); }

// points of a pair of launches: what they read twice stays in the last-level cache
int64_t batch_points(const LayerShape &s, const Tiling &t, int tensors)
{
    const int64_t bytes = int64_t(s.positions) * s.channels * (s.bf16 ? 2 : 4) * tensors;
    const int64_t fit = (int64_t(96) << 20) / bytes;
    return std::max<int64_t>(1, std::min({s.points, std::max<int64_t>(fit, 1), (int64_t(1) << 22) / t.pieces}));
}

template <typename F> void with_k(int k, F f)
{
    switch (k) {
    case 1: f(std::integral_constant<int, 1>()); break;
    case 2: f(std::integral_constant<int, 2>()); break;
    case 4: f(std::integral_constant<int, 4>()); break;
    default: f(std::integral_constant<int, 8>()); break;
    }
}
// f(bf16, vec, wide)
template <typename F> void with_types(const LayerShape &s, int groups, F f)
{
    using Yes = std::true_type;
    using No = std::false_type;
    const int vec = s.bf16 ? 8 : 4;
    const bool wide = s.channels / groups % vec == 0;
    if (s.channels < vec) s.bf16 ? f(Yes(), std::integral_constant<int, 1>(), No()) : f(No(), std::integral_constant<int, 1>(), No());
    else if (s.bf16) wide ? f(Yes(), std::integral_constant<int, 8>(), Yes()) : f(Yes(), std::integral_constant<int, 8>(), No());
    else wide ? f(No(), std::integral_constant<int, 4>(), Yes()) : f(No(), std::integral_constant<int, 4>(), No());
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
constexpr int kForwardChunks = 8, kForwardThreads = 1024, kBackwardChunks = 8, kBackwardThreads = 512;
// points of a piece: a workgroup's sums of the parameters' gradients are over so many that they are little beside what it reads
int64_t points_of_piece(const LayerShape &s, const Tiling &t)
{
    const int64_t wanted = std::max<int64_t>(1, kUnits * 8 / t.tiles);
    int64_t length = std::max<int64_t>((s.points + wanted - 1) / wanted, std::min<int64_t>(32 / std::min(s.positions, 32), (s.points + kUnits - 1) / kUnits));
    return std::max<int64_t>((length + t.side - 1) / t.side * t.side, 1);
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
    p.t = tile(s, groups, kBackwardThreads, kBackwardChunks);
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

}  // namespace

size_t norm_forward_bytes(const LayerShape &s, int groups)
{
    if (s.points == 0 || lanes_per_group(s, groups) || tile(s, groups, kForwardThreads, kForwardChunks).k) return 0;
    const Tiling t = cut(s, groups);
    return static_cast<size_t>(batch_points(s, t, 1)) * t.tiles * t.pieces * most_groups(t, groups) * sizeof(f2);
}

size_t norm_backward_bytes(const LayerShape &s, int groups, const int64_t *bounds, int runs)
{
    if (s.points == 0) return 0;
    const BackwardPlan p = plan_backward(s, groups);
    const int64_t rows = p.cut ? s.points * p.units_per_point : most_pieces(bounds, runs, p.units_per_point, p.length);
    size_t bytes = 2 * align_up(static_cast<size_t>(rows) * s.channels * sizeof(float));
    if (p.cut) bytes += static_cast<size_t>(batch_points(s, p.t, 2)) * p.t.tiles * p.t.pieces * most_groups(p.t, groups) * sizeof(f2);
    return bytes;
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
            (s.bf16 ? norm_rows_forward_kernel<true, l()> : norm_rows_forward_kernel<false, l()>)<<<grid, 256, 0, stream>>>(a, across, length);
        });
        return hipGetLastError();
    }
    const Tiling t = tile(s, a.groups, kForwardThreads, kForwardChunks);
    if (t.k) {
        with_types(s, a.groups, [&](auto bf16, auto vec, auto wide) {
            with_k(t.k, [&](auto k) {
                const dim3 grid(static_cast<unsigned>(std::min<int64_t>((s.points + t.side - 1) / t.side, 1 << 20)), t.tiles);
                const size_t lds = (t.threads * (wide() ? 1 : vec()) + 2 * t.side * most_groups(t, a.groups)) * sizeof(float);
                norm_tile_forward_kernel<bf16(), vec(), k(), wide()><<<grid, t.threads, lds, stream>>>(a, t);
            });
        });
        return hipGetLastError();
    }
    const Tiling c = cut(s, a.groups);
    const Parts parts = {static_cast<f2 *>(workspace), most_groups(c, a.groups)};
    const int64_t batch = batch_points(s, c, 1);
    for (int64_t n = 0; n < s.points; n += batch) {
        const dim3 grid(static_cast<unsigned>(std::min(batch, s.points - n) * c.pieces), c.tiles);
        with_types(s, a.groups, [&](auto bf16, auto vec, auto wide) {
            const size_t tables = 2 * parts.stride * sizeof(float), lds = c.threads * (wide() ? 1 : vec()) * sizeof(float) + tables;
            norm_part_forward_kernel<bf16(), vec(), kPartChunks, wide()><<<grid, c.threads, lds, stream>>>(a, c, parts, n);
            norm_join_forward_kernel<bf16(), vec(), kPartChunks, wide()><<<grid, c.threads, tables, stream>>>(a, c, parts, n);
        });
    }
    return hipGetLastError();
}

hipError_t launch_norm_backward(const NormGradArgs &a, void *workspace, hipStream_t stream)
{
    const LayerShape &s = a.shape;
    const bool sums = a.dgamma || a.dbeta;
    if (!sums && (!a.dx.p || s.points == 0)) return hipSuccess;
    if (s.points == 0) {                                 // sums of nothing
        for (int r = 0; r < a.runs; r += Pieces::kRuns) {
            Pieces p;
            lay_out_pieces(a.bounds + r, std::min(Pieces::kRuns, a.runs - r), 1, 1, &p);
            launch_sum_pieces<true>(nullptr, nullptr, s.channels, p, a.dgamma ? a.dgamma + int64_t(r) * s.channels : nullptr,
                                    a.dbeta ? a.dbeta + int64_t(r) * s.channels : nullptr, stream);
        }
        return hipGetLastError();
    }
    const BackwardPlan p = plan_backward(s, a.groups);
    const int64_t rows = p.cut ? s.points * p.units_per_point : most_pieces(a.bounds, a.runs, p.units_per_point, p.length);
    const size_t table = align_up(static_cast<size_t>(rows) * s.channels * sizeof(float));
    float *parts_gamma = sums ? static_cast<float *>(workspace) : nullptr;
    float *parts_beta = sums ? reinterpret_cast<float *>(static_cast<char *>(workspace) + table) : nullptr;
    if (p.cut) {
        const Tiling &t = p.t;
        const Parts parts = {reinterpret_cast<f2 *>(static_cast<char *>(workspace) + 2 * table), most_groups(t, a.groups)};
        const int64_t batch = batch_points(s, t, 2);
        for (int64_t n = 0; n < s.points; n += batch) {
            const dim3 grid(static_cast<unsigned>(std::min(batch, s.points - n) * t.pieces), t.tiles);
            with_types(s, a.groups, [&](auto bf16, auto vec, auto wide) {
                const size_t tables = 2 * parts.stride * sizeof(float), room = t.threads * vec() * sizeof(float);
                const size_t lds = 2 * (wide() ? t.threads * sizeof(float) : room) + tables;
                float *to_gamma = sums ? parts_gamma + n * t.pieces * s.channels : nullptr, *to_beta = sums ? parts_beta + n * t.pieces * s.channels : nullptr;
                norm_part_backward_kernel<bf16(), vec(), kPartChunks, wide()><<<grid, t.threads, std::max(lds, room), stream>>>(a, t, parts, n, to_gamma, to_beta);
                if (a.dx.p) norm_join_backward_kernel<bf16(), vec(), kPartChunks, wide()><<<grid, t.threads, tables, stream>>>(a, t, parts, n);
            });
        }
    }
    for (int r = 0; r < a.runs; r += Pieces::kRuns) {
        Pieces pieces;
        const int count = lay_out_pieces(a.bounds + r, std::min(Pieces::kRuns, a.runs - r), p.units_per_point, p.length, &pieces);
        const float *from_gamma = parts_gamma, *from_beta = parts_beta;
        if (p.cut) {                                     // rows of all pieces lie in one table
            from_gamma += pieces.first[0] * s.channels;
            from_beta += pieces.first[0] * s.channels;
        } else if (count > 0 && p.lanes) {
            const int across = across_of(s, p.lanes);
            const dim3 grid(ceil_div(s.channels / (s.bf16 ? 8 : 4), across), count);
            with_lanes(p.lanes, [&](auto l) {
                (s.bf16 ? norm_rows_backward_kernel<true, l()> : norm_rows_backward_kernel<false, l()>)<<<grid, 256, 0, stream>>>(a, across, pieces, parts_gamma, parts_beta);
            });
        } else if (count > 0) {
            const Tiling &t = p.t;
            with_types(s, a.groups, [&](auto bf16, auto vec, auto wide) {
                with_k(t.k, [&](auto k) {
                    const size_t room = t.threads * vec() * sizeof(float);
                    const size_t lds = 2 * (wide() ? t.threads * sizeof(float) : room) + 2 * t.side * most_groups(t, a.groups) * sizeof(float);
                    norm_tile_backward_kernel<bf16(), vec(), k(), wide()><<<dim3(count, t.tiles), t.threads, std::max(lds, room), stream>>>(a, t, pieces, parts_gamma, parts_beta);
                });
            });
        }
        if (sums)
            launch_sum_pieces<true>(from_gamma, from_beta, s.channels, pieces, a.dgamma ? a.dgamma + int64_t(r) * s.channels : nullptr,
                                    a.dbeta ? a.dbeta + int64_t(r) * s.channels : nullptr, stream);
    }
    return hipGetLastError();
}

}  // namespace cr

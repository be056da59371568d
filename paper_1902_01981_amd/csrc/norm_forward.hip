// Group norm with an activation, channels last, for gfx950: the forward pass.
//
// A thread has a chunk of 16 bytes of channels and goes down a point's positions, so that its gamma, beta and statistics stay in registers.  Sums over a
// group meet in LDS.  The variance is the mean of squared distances from the mean, taken from registers in a second step, never a difference of large
// sums; pieces of a group that several workgroups have meet by  M2 = sum M2_i + n_i (mean_i - mean)^2.
//
//   norm_tile_forward_kernel   a point's groups (or some of them, or several points) in the registers of a workgroup, read once
//   norm_deep_forward_kernel   the same for several points of few positions at a time
//   norm_part_forward_kernel, norm_join_forward_kernel   larger groups: pieces leave their moments, then every piece is read again
//   (points of one position: norm_rows.hip)
//
// Fewer than ten operations per byte, so the reads and writes are the floor.  A tile is bound by its chain of loads, sums and barriers, of which a compute
// unit has a few at a time: 2 000 x 49 x 512 bf16, 32 groups, 46 us, 4.3 TB/s.  20 000 x 4 x 320, 29 us, 3.5 TB/s.  One group of more channels than norm_rows.hip takes has 1 024 threads
// and a chunk each: 16 384 x 8 192 bf16 500 us, 1.1 TB/s.  Pieces are read twice: 64 x 4 096 x 512 bf16, 170 us, 4.7 TB/s of what moves, 3.2 of what has to; where
// points are few, every workgroup adding up all pieces' moments before it goes on is most of it: 1 x 4 454 x 2 240, 37 us, 29 of them the second kernel.
#include "norm_device.h"

namespace cr {

namespace {

// The mean of a group as its user gets it: not an infinity, which is what a group with one in it may have for a mean (its rstd is NaN then).
__device__ __forceinline__ float known(float mean, float rstd) { return rstd != rstd ? rstd : mean; }

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

// y from x: gamma h + beta and the activation.  gamma rstd is one number, rounded by itself: half a unit of gamma h.
template <int VEC, int ACT> struct Finish {
    float shift[VEC], scale[VEC], beta[VEC];
    __device__ __forceinline__ Finish(const NormArgs &a, int channel, const float (&mean)[VEC], const float (&rstd)[VEC])
    {
        read_floats(scale, a.gamma, channel, 1.f);
        read_floats(beta, a.beta, channel, 0.f);
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            scale[v] *= rstd[v];
            shift[v] = mean[v];
        }
    }
    __device__ __forceinline__ void operator()(float (&x)[VEC]) const
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) x[v] = activated<ACT>(fmaf(x[v] - shift[v], scale[v], beta[v]));
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
                a.mean[point * a.groups + c.group + q % c.groups] = known(mean[q], rstd[q]);
                a.rstd[point * a.groups + c.group + q % c.groups] = rstd[q];
            }
        }
        __syncthreads();
        if (s.has && n < a.shape.points) {
            float m[VEC], r[VEC];
            spread<VEC, UNIT>(m, mean, s, c, cg);
            spread<VEC, UNIT>(r, rstd, s, c, cg);
            const Finish<VEC, ACT> finish(a, c.first + s.at, m, r);
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
    // in scalar registers: one more vector register would cost a wavefront a unit
    auto scalar_of = [](float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); };
    const float count = scalar_of(static_cast<float>(positions) * cg), share = scalar_of(1.f / count);
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
                v[i] -= quotient(m[i], count, share);
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
            mean[q] = quotient(mean[q], count, share);
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
                const Finish<VEC, ACT> finish(a, c.first + s.at, m, r);
                C::widen(raw[k], v);
                finish(v);
                const Walk<BF16, VEC> y(a.y, n + k * t.side, s.ty, c.first + s.at, t.down);
                C::store(y.base + y.offset, C::narrow(v));
            }
        }
        __syncthreads();                                 // before the tables are other points'
    }
}

// ---- pieces of a point's groups ------------------------------------------------------------------------------------------------------------
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
            const float fresh = static_cast<float>(rows * UNIT), total = have + fresh;
            const float part = fresh / total;
            const float weight = have * part;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const float m = all() ? sum[i] * (1.f / (U * UNIT)) : sum[i] / fresh, apart = m - mean[i];          // the first is exact: a power of two
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
                a.mean[n * a.groups + c.group + g] = known(mean[g], rstd[g]);
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
    const Finish<VEC, ACT> finish(a, c.first + s.at, m, r);
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

}  // namespace

size_t norm_forward_bytes(const LayerShape &s, int groups)
{
    if (s.points == 0 || rows_plan(s, groups, false).lanes || tile(s, groups, false).k) return 0;
    const Tiling t = cut(s, groups);
    return static_cast<size_t>(batch_points(s, t)) * t.tiles * t.pieces * most_groups(t, groups) * sizeof(f2);
}

hipError_t launch_norm_forward(const NormArgs &a, void *workspace, hipStream_t stream)
{
    const LayerShape &s = a.shape;
    if (s.points == 0) return hipSuccess;
    if (const RowsPlan p = rows_plan(s, a.groups, false); p.lanes) {
        launch_norm_rows_forward(a, p, stream);
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

}  // namespace cr

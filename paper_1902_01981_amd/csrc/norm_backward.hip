// Group norm with an activation, channels last, for gfx950: the gradient.
//
// With dz = dy act'(z) and M values in a group, A = sum gamma dz / M and B = sum gamma dz h / M over the group, dx = rstd (gamma dz - A - h B); the parameters'
// gradients are sums of dz h and dz over the points of a run.  Threads and tiles are those of the forward pass; a thread's sums for the parameters stay in
// its registers over all points of its piece of a run.
//
//   norm_tile_backward_kernel   points' groups in the registers of a workgroup, read once
//   norm_deep_backward_kernel   the same for several points of few positions at a time
//   norm_part_backward_kernel, norm_join_backward_kernel   larger groups: pieces leave their sums, then every piece is read again
//   sum_parts_kernel, sum_pieces_kernel   the parameters' gradients per run
//   (points of one position: norm_rows.hip)
//
// Bound as the forward pass is, with twice the sums: 2 000 x 49 x 512 bf16, 32 groups, 95 us, 3.2 TB/s, two launches for 4 096 sums of a run among them;
// 20 000 x 4 x 320 72 us, 2.1 TB/s.  Pieces are read twice, and the slopes of an activation formed twice: 64 x 4 096 x 512 bf16, 269 us, 5.0 TB/s of what
// moves, 3.0 of what has to.  1 x 4 454 x 2 240: 54 us, 28 of them the second kernel, as in the forward pass.
#include "norm_device.h"

namespace cr {

namespace {

// What a thread needs of its channels for the gradient.  x - mean stands for h where rstd can be multiplied in later, in sums and once per channel.  (Not
// x rstd - mean rstd: where a group's values are close together the rounding of one product would be left over.)
template <int VEC, int ACT> struct Gradient {
    float mean[VEC], rstd[VEC], gamma[VEC], beta[VEC];
    // dz from dy; x - mean is left in x
    __device__ __forceinline__ void slopes(float (&x)[VEC], float (&d)[VEC]) const
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            x[v] -= mean[v];
            d[v] = through_slope<ACT>(fmaf(x[v] * rstd[v], gamma[v], beta[v]), d[v]);
        }
    }
};
// dx = rstd (gamma dz - A - h B) from x - mean and dz; where a group is one value gamma dz and A are the same, and what is left of them is the rounding of
// that product
template <int VEC> struct Correction {
    float A[VEC], B[VEC];
    template <typename G> __device__ __forceinline__ Correction(const G &g, const float (&sum_A)[VEC], const float (&sum_B)[VEC], float share)
    {
#pragma unroll
        for (int v = 0; v < VEC; ++v) {
            A[v] = sum_A[v] * share;
            B[v] = sum_B[v] * share * g.rstd[v];
        }
    }
    template <typename G> __device__ __forceinline__ float operator()(const G &g, float from_mean, float dz, int v) const
    {
        return g.rstd[v] * fmaf(-from_mean, B[v], fmaf(g.gamma[v], dz, -A[v]));
    }
};
// mean and 1 / deviation of a seat's channels, from the tensors
template <int VEC, int UNIT, bool WAIT = false> __device__ __forceinline__ void read_stats(float (&m)[VEC], float (&r)[VEC], const NormGradArgs &a, const Seat &s, const Columns &c, int64_t point, int cg)
{
    const float *mean = a.mean + point * a.groups + c.group, *rstd = a.rstd + point * a.groups + c.group;
    Columns one = c;
    Seat seat = s;
    one.groups = 0;                                      // the tables are this point's
    seat.side = 0;
    const int within = c.first - c.group * cg;           // a slice of a group begins inside it
    seat.at += within;
    spread<VEC, UNIT, WAIT>(m, mean, seat, one, cg);
    spread<VEC, UNIT, WAIT>(r, rstd, seat, one, cg);
}

// The groups' sums of gamma s1 and gamma s2, s1 over dz and s2 over dz h, for every thread.
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
__global__ void __launch_bounds__(K == 1 ? 512 : 256) norm_tile_backward_kernel(NormGradArgs a, Tiling t, Pieces pieces, float *parts_gamma, float *parts_beta)
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
    Gradient<VEC, ACT> g;
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
        read_stats<VEC, UNIT, true>(g.mean, g.rstd, a, s, c, n, cg);
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
#pragma unroll
        for (int v = 0; v < VEC; ++v) s2[v] *= g.rstd[v];
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
            const Correction<VEC> dx_of(g, A, B, share);
            const Walk<BF16, VEC> dx(a.dx, n, s.ty, c.first + s.at, t.down);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (exists(s.ty, k, t.down, positions)) {
                    float h[VEC];
                    C::widen(raw[k], h);
#pragma unroll
                    for (int v = 0; v < VEC; ++v) h[v] = dx_of(g, h[v] - g.mean[v], dz[k][v], v);
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
__global__ void __launch_bounds__(512) norm_deep_backward_kernel(NormGradArgs a, Tiling t, Pieces pieces, float *parts_gamma, float *parts_beta)
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
    Gradient<VEC, ACT> g;
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
                h[v] *= g.rstd[v];
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
                const Correction<VEC> dx_of(g, A, B, share);
#pragma unroll
                for (int v = 0; v < VEC; ++v) h[v] = dx_of(g, h[v] - g.mean[v], dz[k][v], v);
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
    Gradient<VEC, ACT> g;
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
#pragma unroll
    for (int v = 0; v < VEC; ++v) s2[v] *= g.rstd[v];
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
    Gradient<VEC, ACT> g;
    float A[VEC], B[VEC];
    read_floats(g.gamma, a.gamma, c.first + s.at, 1.f);
    read_floats(g.beta, a.beta, c.first + s.at, 0.f);
    read_stats<VEC, UNIT>(g.mean, g.rstd, a, s, c, n, cg);
    __syncthreads();
    if (!s.has) return;
    const int cg_tile = t.slices == 1 ? cg : c.width;
    spread<VEC, UNIT>(A, A_of, s, c, cg_tile);
    spread<VEC, UNIT>(B, B_of, s, c, cg_tile);
    const Correction<VEC> dx_of(g, A, B, 1.f);
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

bool norm_backward_numbered(const LayerShape &s, int groups)
{
    return s.points == 0 || s.points < (int64_t(1) << 31) / plan_backward(s, groups).units_per_point;
}

size_t norm_backward_bytes(const LayerShape &s, int groups, const int64_t *bounds, int runs)
{
    return s.points == 0 ? 0 : room_of(s, groups, plan_backward(s, groups), bounds, runs).bytes();
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
        float *to_gamma = parts_gamma, *to_beta = parts_beta;
        float *dgamma = a.dgamma ? a.dgamma + int64_t(r) * s.channels : nullptr, *dbeta = a.dbeta ? a.dbeta + int64_t(r) * s.channels : nullptr;
        const bool direct = sums && !p.cut && one_each(pieces);
        if (direct) {                                    // what is not wanted has its place in the workspace all the same
            if (dgamma) to_gamma = dgamma;
            if (dbeta) to_beta = dbeta;
        }
        if (p.cut && sums) {                             // rows of all pieces lie in one table
            from_gamma += pieces.first[0] * s.channels;
            from_beta += pieces.first[0] * s.channels;
        } else if (p.cut) {
            break;
        } else if (count > 0 && p.rows.lanes) {
            launch_norm_rows_backward(a, p.rows, pieces, count, to_gamma, to_beta, stream);
        } else if (count > 0) {
            const Tiling &t = p.t;
            if (t.deep) {
                with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
                    const size_t columns = t.threads * vec() * sizeof(float);
                    const size_t lds = std::max(2 * t.deep * (t.threads * (vec() / unit()) + t.side * most_groups(t, a.groups)) * sizeof(float), columns);
                    with_activation(a.activation, [&](auto act) {
                        constexpr int B = bf16(), V = vec(), U = unit(), A = act();
                        (t.deep == 4 ? norm_deep_backward_kernel<B, V, U == V ? 4 : 2, U, A> : norm_deep_backward_kernel<B, V, 2, U, A>)
                            <<<dim3(count, t.tiles), t.threads, lds, stream>>>(a, t, pieces, to_gamma, to_beta);
                    });
                });
            } else with_types(s, a.groups, [&](auto bf16, auto vec, auto unit) {
                with_k(t.k, [&](auto k) {
                    const size_t columns = t.threads * vec() * sizeof(float);
                    const size_t lds = std::max((2 * t.threads * (vec() / unit()) + 2 * t.side * most_groups(t, a.groups)) * sizeof(float), columns);
                    with_activation(a.activation, [&](auto act) {
                        norm_tile_backward_kernel<bf16(), vec(), k(), unit(), act()><<<dim3(count, t.tiles), t.threads, lds, stream>>>(a, t, pieces, to_gamma, to_beta);
                    });
                });
            });
        }
        if (sums && !direct) launch_sum_pieces(from_gamma, from_beta, s.channels, pieces, beside, dgamma, dbeta, stream);
    }
    return hipGetLastError();
}

}  // namespace cr

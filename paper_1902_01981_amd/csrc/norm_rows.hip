// Group norm of points of one position, forward and gradient, for gfx950: a group is a row of neighbouring channels, and a few lanes of a wavefront have it.
//
// LANES lanes (a power of two) have the group, CHUNKS chunks of 16 bytes each; sums over the group go from lane to lane, and no workgroup meets.  A team
// stays with its group and goes through the points, U at a time, so that gamma, beta and the sums of their gradients stay in registers.  Where the group is no
// whole number of chunks (or lanes are left over), the last chunk is moved back to end with it: what it shares with its neighbour is summed up there, and
// comes out the same in both.
//
// The reads and writes bound it: 16 384 x 4 096 bf16, 32 groups, forward 49 us, 5.4 TB/s, gradient 80 us, 5.0 TB/s with the sums over the run after it;
// 65 536 x 1 027 fp32, one group, 109 us, 4.9 TB/s, and 150 us, 5.4 TB/s.  (By workgroups that meet in
// LDS, as points of more positions: 294 and 1 243 us.)
#include "norm_device.h"

namespace cr {

namespace {

// What a lane has of its group.
template <int VEC, int LANES, int CHUNKS, bool EXACT> struct GroupLane {
    int at[CHUNKS];              // channel in the group
    int skip;                    // elements of the last chunk that do not count
    __device__ __forceinline__ GroupLane(int cg)
    {
        const int lane = threadIdx.x % LANES, chunks = (cg + VEC - 1) / VEC;
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) at[k] = min((lane + k * LANES) * VEC, cg - VEC);
        const int q = lane + (CHUNKS - 1) * LANES;
        skip = q < chunks - 1 ? 0 : q == chunks - 1 ? chunks * VEC - cg : VEC;
    }
    // does element v of chunk k count in sums over the group?  (All chunks but a lane's last are whole ones.)
    __device__ __forceinline__ bool counts(int k, int v) const { return EXACT || k < CHUNKS - 1 || v >= skip; }
};
// Which group and points a team has.
struct Team {
    int group, ty;
    bool has;
};
__device__ __forceinline__ Team take_team(int lanes, int groups, int wide, int down)
{
    const int team = threadIdx.x / lanes;
    Team t;
    t.group = blockIdx.x * wide + team % wide;
    t.ty = team / wide;
    t.has = t.group < groups && t.ty < down;
    t.group = min(t.group, groups - 1);
    return t;
}
template <bool BF16, int LANES, int CHUNKS, bool EXACT, int ACT>
__global__ void __launch_bounds__(256) norm_rows_forward_kernel(NormArgs a, int wide, int down, int64_t length)
{
    constexpr int VEC = BF16 ? 8 : 4, U = points_at_once(CHUNKS);
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int cg = a.shape.channels / a.groups;
    const Team team = take_team(LANES, a.groups, wide, down);
    if (!team.has) return;                               // whole teams
    const GroupLane<VEC, LANES, CHUNKS, EXACT> lane(cg);
    const int first = team.group * cg;
    // parameters of few chunks stay in registers, of more they are read again, from the caches
    float gamma[CHUNKS <= 2 ? CHUNKS : 1][VEC], beta[CHUNKS <= 2 ? CHUNKS : 1][VEC];
    if constexpr (CHUNKS <= 2) {
#pragma unroll
        for (int k = 0; k < CHUNKS; ++k) {
            read_floats(gamma[k], a.gamma, first + lane.at[k], 1.f);
            read_floats(beta[k], a.beta, first + lane.at[k], 0.f);
        }
    }
    const float share = 1.f / cg;
    const int64_t begin = blockIdx.y * length, end = min(begin + length, a.shape.points);
    const T *x = static_cast<const T *>(a.x.p) + first;
    T *y = static_cast<T *>(a.y.p) + first;
    for (int64_t n0 = begin + team.ty; n0 < end; n0 += U * down) {
        typename C::raw raw[U][CHUNKS];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) raw[u][k] = C::load_once(x + min(n0 + u * down, end - 1) * a.x.point_stride + lane.at[k]);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t n = n0 + u * down;
            float v[CHUNKS][VEC], sum = 0.f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                C::widen(raw[u][k], v[k]);
#pragma unroll
                for (int i = 0; i < VEC; ++i) sum += lane.counts(k, i) ? v[k][i] : 0.f;
            }
            const float mean = quotient(lanes_total<LANES>(sum), static_cast<float>(cg), share);
            sum = 0.f;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) {
                    v[k][i] -= mean;
                    sum = fmaf(lane.counts(k, i) ? v[k][i] : 0.f, v[k][i], sum);
                }
            const float rstd = 1.f / sqrtf(fmaf(lanes_total<LANES>(sum), share, a.eps));
            if (n >= end) continue;
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k) {
                constexpr bool kHeld = CHUNKS <= 2;
                if constexpr (!kHeld) {
                    read_floats(gamma[0], a.gamma, first + lane.at[k], 1.f);
                    read_floats(beta[0], a.beta, first + lane.at[k], 0.f);
                }
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[k][i] = activated<ACT>(fmaf(v[k][i] * rstd, gamma[kHeld ? k : 0][i], beta[kHeld ? k : 0][i]));
                C::store(y + n * a.y.point_stride + lane.at[k], C::narrow(v[k]));
            }
            if (a.mean && threadIdx.x % LANES == 0) {
                a.mean[n * a.groups + team.group] = mean;
                a.rstd[n * a.groups + team.group] = rstd;
            }
        }
    }
}

template <bool BF16, int LANES, int CHUNKS, bool EXACT, int ACT>
__global__ void __launch_bounds__(256) norm_rows_backward_kernel(NormGradArgs a, int wide, int down, Pieces pieces, float *parts_gamma, float *parts_beta)
{
    constexpr int VEC = BF16 ? 8 : 4, U = points_at_once(CHUNKS);
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float lds[256 * VEC * CHUNKS];
    const int cg = a.shape.channels / a.groups;
    const Team team = take_team(LANES, a.groups, wide, down);
    const GroupLane<VEC, LANES, CHUNKS, EXACT> lane(cg);
    const int first = team.group * cg;
    float gamma[CHUNKS][VEC], beta[CHUNKS][VEC], sum_gamma[CHUNKS][VEC], sum_beta[CHUNKS][VEC];
#pragma unroll
    for (int k = 0; k < CHUNKS; ++k) {
        read_floats(gamma[k], a.gamma, first + lane.at[k], 1.f);
        read_floats(beta[k], a.beta, first + lane.at[k], 0.f);
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum_gamma[k][i] = sum_beta[k][i] = 0.f;
    }
    const float share = 1.f / cg;
    const Piece piece = find_piece(pieces, blockIdx.y);
    const T *x = static_cast<const T *>(a.x.p) + first, *dy = static_cast<const T *>(a.dy.p) + first;
    T *dx = static_cast<T *>(a.dx.p) + first;
    if (team.has) {
        for (int64_t n0 = piece.begin + team.ty; n0 < piece.end; n0 += U * down) {
            typename C::raw raw[U][CHUNKS], raw_d[U][CHUNKS];
            float mean[U], rstd[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t n = min(n0 + u * down, piece.end - 1);
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    raw[u][k] = C::load_once(x + n * a.x.point_stride + lane.at[k]);
                    raw_d[u][k] = C::load_once(dy + n * a.dy.point_stride + lane.at[k]);
                }
                mean[u] = a.mean[n * a.groups + team.group];
                rstd[u] = a.rstd[n * a.groups + team.group];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t n = n0 + u * down;
                float h[CHUNKS][VEC], d[CHUNKS][VEC], A = 0.f, B = 0.f;
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
                    C::widen(raw[u][k], h[k]);
                    C::widen(raw_d[u][k], d[k]);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        h[k][i] = (h[k][i] - mean[u]) * rstd[u];
                        d[k][i] = through_slope<ACT>(fmaf(h[k][i], gamma[k][i], beta[k][i]), d[k][i]);
                        const float t = lane.counts(k, i) ? gamma[k][i] * d[k][i] : 0.f;
                        A += t;
                        B = fmaf(t, h[k][i], B);
                    }
                }
                A = lanes_total<LANES>(A) * share;
                B = lanes_total<LANES>(B) * share;
                if (n >= piece.end) continue;
#pragma unroll
                for (int k = 0; k < CHUNKS; ++k) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        sum_beta[k][i] += d[k][i];
                        sum_gamma[k][i] = fmaf(d[k][i], h[k][i], sum_gamma[k][i]);
                        d[k][i] = rstd[u] * fmaf(-h[k][i], B, fmaf(gamma[k][i], d[k][i], -A));
                    }
                    if (a.dx.p) C::store(dx + n * a.dx.point_stride + lane.at[k], C::narrow(d[k]));
                }
            }
        }
    }
    if (!parts_gamma) return;
    const int columns = min(wide, a.groups - static_cast<int>(blockIdx.x) * wide) * cg, from = blockIdx.x * wide * cg, column = (team.group - blockIdx.x * wide) * cg;
    auto total = [&](const float (&sum)[CHUNKS][VEC], float *parts) {
        if (team.has) {
#pragma unroll
            for (int k = 0; k < CHUNKS; ++k)
#pragma unroll
                for (int i = 0; i < VEC; ++i) lds[team.ty * columns + column + lane.at[k] + i] = sum[k][i];
        }
        add_columns_in_lds(down, columns, lds, [&](int col, float t) { parts[int64_t(blockIdx.y) * a.shape.channels + from + col] = t; });
    };
    total(sum_gamma, parts_gamma);
    total(sum_beta, parts_beta);
}

template <typename F> void with_team(const LayerShape &s, int groups, const RowsPlan &p, F f)
{
    const int cg = s.channels / groups, vec = s.bf16 ? 8 : 4;
    const bool exact = cg == p.lanes * p.chunks * vec;
    auto lanes = [&](auto l) {                           // one chunk each
        if (exact) f(l, std::integral_constant<int, 1>(), std::true_type());
        else f(l, std::integral_constant<int, 1>(), std::false_type());
    };
    auto chunks = [&](auto k) { f(std::integral_constant<int, 64>(), k, std::false_type()); };
    switch (p.lanes) {
    case 1: f(std::integral_constant<int, 1>(), std::integral_constant<int, 1>(), std::true_type()); return;
    case 2: lanes(std::integral_constant<int, 2>()); return;
    case 4: lanes(std::integral_constant<int, 4>()); return;
    case 8: lanes(std::integral_constant<int, 8>()); return;
    case 16: lanes(std::integral_constant<int, 16>()); return;
    case 32: lanes(std::integral_constant<int, 32>()); return;
    }
    switch (p.chunks) {
    case 1: lanes(std::integral_constant<int, 64>()); return;
    case 2: chunks(std::integral_constant<int, 2>()); return;
    case 3: chunks(std::integral_constant<int, 3>()); return;
    case 4: chunks(std::integral_constant<int, 4>()); return;
    case 5: chunks(std::integral_constant<int, 5>()); return;
    case 6: chunks(std::integral_constant<int, 6>()); return;
    case 7: chunks(std::integral_constant<int, 7>()); return;
    default: chunks(std::integral_constant<int, 8>()); return;
    }
}

}  // namespace

void launch_norm_rows_forward(const NormArgs &a, const RowsPlan &p, hipStream_t stream)
{
    const int64_t length = points_of_workgroup(a.shape, a.groups, p, 16, 1);
    const dim3 grid(ceil_div(a.groups, p.wide), ceil_div(a.shape.points, length));
    with_team(a.shape, a.groups, p, [&](auto lanes, auto chunks, auto exact) {
        with_activation(a.activation, [&](auto act) {
            constexpr int L = lanes(), K = chunks(), E = exact(), A = act();
            (a.shape.bf16 ? norm_rows_forward_kernel<true, L, K, E, A> : norm_rows_forward_kernel<false, L, K, E, A>)<<<grid, 256, 0, stream>>>(a, p.wide, p.down, length);
        });
    });
}

void launch_norm_rows_backward(const NormGradArgs &a, const RowsPlan &p, const Pieces &pieces, int count, float *parts_gamma, float *parts_beta, hipStream_t stream)
{
    const dim3 grid(ceil_div(a.groups, p.wide), count);
    with_team(a.shape, a.groups, p, [&](auto lanes, auto chunks, auto exact) {
        with_activation(a.activation, [&](auto act) {
            constexpr int L = lanes(), K = chunks(), E = exact(), A = act();
            (a.shape.bf16 ? norm_rows_backward_kernel<true, L, K < 4 ? K : 4, E, A> : norm_rows_backward_kernel<false, L, K, E, A>)
                <<<grid, 256, 0, stream>>>(a, p.wide, p.down, pieces, parts_gamma, parts_beta);
        });
    });
}

}  // namespace cr

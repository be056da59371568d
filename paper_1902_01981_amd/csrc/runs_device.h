// Sums over the points of a run, in two steps: workgroups add up pieces of a run's rows and leave a row of sums each; these are added up per run.
#pragma once
#include <algorithm>

#include "layers_device.h"

namespace cr {

// Runs in pieces, as a kernel argument: run r has `units` first[r] .. first[r + 1] (points, or rows of channels), cut into pieces of `length` units;
// they are pieces piece[r] .. piece[r + 1] of the launch.  A launch takes a batch of at most kRuns runs.
struct Pieces {
    static constexpr int kRuns = 128;
    int runs;
    int64_t length;
    int64_t first[kRuns + 1];
    int piece[kRuns + 1];
};
struct Piece {
    int64_t begin, end;
};
#ifdef __HIPCC__
// The units of a piece.  Every wavefront finds its run for itself: the number of runs that begin at or before the piece.
__device__ __forceinline__ Piece find_piece(const Pieces &p, int piece)
{
    int r = 0;
    if (p.runs > 1) {
        const int lane = threadIdx.x % 64;
        int before = 0;
#pragma unroll
        for (int i = 0; i < Pieces::kRuns; i += 64) before += __popcll(__ballot(i + lane < p.runs && p.piece[i + lane] <= piece));
        r = __builtin_amdgcn_readfirstlane(before) - 1;
        // runs of no pieces begin where the next one does: the last of them that begins here is the one that has it
    }
    Piece q;
    q.begin = p.first[r] + (piece - p.piece[r]) * p.length;
    q.end = min(q.begin + p.length, p.first[r + 1]);
    return q;
}
#endif
// Fills in a batch of runs from bounds[0 .. runs]; per_point units per point.  Returns the number of pieces.
inline int lay_out_pieces(const int64_t *bounds, int runs, int64_t per_point, int64_t length, Pieces *out)
{
    out->runs = runs;
    out->length = length;
    out->piece[0] = 0;
    for (int r = 0; r <= runs; ++r) out->first[r] = bounds[r] * per_point;
    for (int r = 0; r < runs; ++r) out->piece[r + 1] = out->piece[r] + static_cast<int>((out->first[r + 1] - out->first[r] + length - 1) / length);
    return out->piece[runs];
}
// The most pieces of a batch that these bounds give.
inline int64_t most_pieces(const int64_t *bounds, int runs, int64_t per_point, int64_t length)
{
    int64_t most = 0;
    for (int r = 0; r < runs; r += Pieces::kRuns) {
        int64_t n = 0;
        for (int i = r; i < std::min(runs, r + Pieces::kRuns); ++i) n += ((bounds[i + 1] - bounds[i]) * per_point + length - 1) / length;
        most = std::max(most, n);
    }
    return most;
}

#ifdef __HIPCC__
// out[r][c] = the sum over run r's pieces of parts[piece][c], added up in 64 bits in a fixed order; a workgroup has 64 columns of a run.  TWO: the same of
// a second table behind the first.
template <int THREADS, bool TWO>
__global__ void __launch_bounds__(THREADS) sum_pieces_kernel(const float *parts, const float *parts2, int columns, Pieces p, float *out, float *out2)
{
    __shared__ double meet[TWO ? 2 : 1][THREADS / 64][64];
    const int r = blockIdx.y, lane = threadIdx.x % 64, wave = threadIdx.x / 64, c = blockIdx.x * 64 + lane, at = min(c, columns - 1);
    double sum = 0.0, sum2 = 0.0;
    for (int i = p.piece[r] + wave; i < p.piece[r + 1]; i += THREADS / 64) {
        sum += parts[int64_t(i) * columns + at];
        if constexpr (TWO) sum2 += parts2[int64_t(i) * columns + at];
    }
    meet[0][wave][lane] = sum;
    if constexpr (TWO) meet[1][wave][lane] = sum2;
    __syncthreads();
    if (wave == 0 && c < columns) {
        for (int w = 1; w < THREADS / 64; ++w) sum += meet[0][w][lane];
        if (out) out[int64_t(r) * columns + c] = static_cast<float>(sum);
        if constexpr (TWO) {
            for (int w = 1; w < THREADS / 64; ++w) sum2 += meet[1][w][lane];
            if (out2) out2[int64_t(r) * columns + c] = static_cast<float>(sum2);
        }
    }
}
template <bool TWO> void launch_sum_pieces(const float *parts, const float *parts2, int columns, const Pieces &p, float *out, float *out2, hipStream_t stream)
{
    const dim3 grid((columns + 63) / 64, p.runs);
    // as many wavefronts as there are pieces to share out
    if (p.piece[p.runs] >= 16 * p.runs) sum_pieces_kernel<1024, TWO><<<grid, 1024, 0, stream>>>(parts, parts2, columns, p, out, out2);
    else sum_pieces_kernel<256, TWO><<<grid, 256, 0, stream>>>(parts, parts2, columns, p, out, out2);
}
#endif

}  // namespace cr

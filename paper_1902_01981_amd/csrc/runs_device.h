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
// Whether every run is one piece: what its workgroup adds up is the run's sum already.
inline bool one_each(const Pieces &p)
{
    for (int r = 0; r < p.runs; ++r)
        if (p.piece[r] != r) return false;
    return p.piece[p.runs] == p.runs;
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

// Pieces of a run that a first launch adds up where a run has so many that one workgroup per 64 columns would be long at it, or 0: one launch does.
// 2 048 pieces of 512 columns, two tables: 97 us in one launch, 6 in two; 768 of 320, 12 runs, with the gradient before it: 41.6 in two, 38.4
// in one.
inline int64_t sum_in_parts(const Pieces &p)
{
    int64_t longest = 0, length = 64;
    for (int r = 0; r < p.runs; ++r) longest = std::max<int64_t>(longest, p.piece[r + 1] - p.piece[r]);
    while (length * length < longest) length *= 2;
    return longest > 512 ? length : 0;
}
// Rows of floats that the sums of any batch of at most `pieces` pieces need beside them, per table.
inline int64_t rows_beside(int64_t pieces, int runs) { return pieces / 64 + std::min(runs, Pieces::kRuns); }

#ifdef __HIPCC__
// Sums of rows [begin, end) of a table with so many columns, a workgroup per 64 columns, in a fixed order; for the first wavefront.
template <int THREADS> __device__ __forceinline__ double sum_rows(const float *table, int64_t columns, int64_t begin, int64_t end, double (*meet)[64])
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int64_t at = min(int64_t(blockIdx.x) * 64 + lane, columns - 1);
    constexpr int WAVES = THREADS / 64, U = 8;
    double sum = 0.0;
    for (int64_t i = begin + wave; i < end; i += U * WAVES) {
        float v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = table[min(i + u * WAVES, end - 1) * columns + at];
#pragma unroll
        for (int u = 0; u < U; ++u) sum += i + u * WAVES < end ? v[u] : 0.f;
    }
    meet[wave][lane] = sum;
    __syncthreads();
    if (wave == 0)
        for (int w = 1; w < WAVES; ++w) sum += meet[w][lane];
    __syncthreads();
    return sum;
}
// out[r][c] = the sum over run r's pieces of parts[piece][c]; blockIdx.z: of one or the other table
template <int THREADS> __global__ void __launch_bounds__(THREADS) sum_pieces_kernel(const float *parts, const float *parts2, int columns, Pieces p, float *out, float *out2)
{
    __shared__ double meet[THREADS / 64][64];
    const int r = blockIdx.y, c = blockIdx.x * 64 + threadIdx.x % 64;
    float *to = blockIdx.z ? out2 : out;
    if (!to) return;
    const double sum = sum_rows<THREADS>(blockIdx.z ? parts2 : parts, columns, p.piece[r], p.piece[r + 1], meet);
    if (threadIdx.x < 64 && c < columns) to[int64_t(r) * columns + c] = static_cast<float>(sum);
}
// the same of a run's parts: piece q of `p` is rows of the tables, its sum goes to row q of the others
static __global__ void __launch_bounds__(256) sum_parts_kernel(const float *parts, const float *parts2, int columns, Pieces p, float *out, float *out2)
{
    __shared__ double meet[4][64];
    const int c = blockIdx.x * 64 + threadIdx.x % 64;
    const Piece q = find_piece(p, blockIdx.y);
    const double sum = sum_rows<256>(blockIdx.z ? parts2 : parts, columns, q.begin, q.end, meet);
    if (threadIdx.x < 64 && c < columns) (blockIdx.z ? out2 : out)[int64_t(blockIdx.y) * columns + c] = static_cast<float>(sum);
}
// The sums of a batch's runs, of one table or two; `beside` holds rows_beside rows per table.
inline void launch_sum_pieces(const float *parts, const float *parts2, int columns, const Pieces &pieces, float *beside, float *out, float *out2, hipStream_t stream)
{
    Pieces p = pieces;
    const unsigned tables = parts2 || out2 ? 2 : 1;
    const unsigned across = (columns + 63) / 64;
    if (const int64_t length = sum_in_parts(pieces)) {
        int64_t bounds[Pieces::kRuns + 1];
        for (int r = 0; r <= p.runs; ++r) bounds[r] = pieces.piece[r];
        const int count = lay_out_pieces(bounds, p.runs, 1, length, &p);
        float *beside2 = beside + int64_t(count) * columns;
        sum_parts_kernel<<<dim3(across, count, tables), 256, 0, stream>>>(parts, parts2, columns, p, beside, beside2);
        parts = beside;
        parts2 = beside2;
    }
    const dim3 grid(across, p.runs, tables);
    // as many wavefronts as there are pieces to share out
    if (p.piece[p.runs] > 16 * p.runs) sum_pieces_kernel<1024><<<grid, 1024, 0, stream>>>(parts, parts2, columns, p, out, out2);
    else sum_pieces_kernel<256><<<grid, 256, 0, stream>>>(parts, parts2, columns, p, out, out2);
}
#endif

}  // namespace cr

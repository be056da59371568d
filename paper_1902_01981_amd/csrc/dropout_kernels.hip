// Bias, dropout and residual, the mask drawn from a counter, for gfx950.
//
// A word of 64 bits has the draws of four neighbouring channels.  Word number i is mix(key + (i + 1) golden): from row to row a thread's number
// moves on by a constant, so that golden times it is one 64-bit addition, and a word costs the two products of the mixing function.
//
//   dropout_forward_kernel, dropout_backward_kernel   a thread has a chunk of 16 bytes of channels and goes down the rows, four at a time; bias and sums
//                          of the bias's gradient stay in its registers
//   sum_pieces_kernel      the bias's gradient per run, where runs are more than a piece each
//
// The reads and writes bound it where there are enough rows, 64 x 512 x 4 096 bf16: forward with residual 129 us, 6.2 TB/s, backward with the bias's
// gradient 92 us, 5.8 TB/s; the two products of 64 bits per word hide behind them.  683 x 9 x 1 027 fp32, 12 runs: 11.8 us, 4.3 TB/s, and 17.7 us, 2.9 TB/s,
// the second launch among them.  Small calls take what the host's part of a launch takes, 7 us.
#include "row_step.h"
#include "runs_device.h"

namespace cr {

namespace {

constexpr int kThreads = 256;
constexpr int kRowsAtOnce = 4, kTailsAtOnce = 2;       // of a thread

__device__ __forceinline__ uint64_t mask_key(const Mask &m) { return splitmix_mix(m.key_state + (m.draw_dev ? kGolden * *m.draw_dev : 0)); }
__device__ __forceinline__ bool kept(uint64_t word, int field, uint32_t least)
{
    const uint32_t half = field < 2 ? static_cast<uint32_t>(word) : static_cast<uint32_t>(word >> 32);
    return field % 2 ? half >= least << 16 : (half & 0xffffu) >= least;      // the low half decides nothing: least << 16 ends in zeros
}

// The columns that a workgroup has: `across` chunks from first_chunk on, rows side by side in the rest of its threads; the last of a row of workgroups also
// has the `left` channels behind the whole chunks: forward an element per thread, whose loads and stores lie side by side (65 536 x 5 x 37 bf16 19.8 us, a row per
// thread 30.4), in the gradient a row per thread, which draws once and sums in its registers (65 536 x 10 x 12 33.5 us, an element per thread 48.5).
struct Columns {
    int chunks, across, down;    // whole chunks of a row, chunks of a workgroup, rows side by side
};
Columns columns_of(int channels, int vec)
{
    Columns c;
    c.chunks = channels / vec;
    const int tiles = std::max(1, (c.chunks + kThreads - 1) / kThreads);
    c.across = (c.chunks + tiles - 1) / tiles;
    c.down = c.across ? kThreads / c.across : kThreads;
    return c;
}
int tiles_of(const Columns &c) { return c.across ? (c.chunks + c.across - 1) / c.across : 1; }

// A row of all points' positions.  FLAT: rows have one stride and the points follow each other, and its number is all there is to it.
template <bool FLAT> struct Row {
    int64_t r, point;
    int position;
};
// The rows of a thread, so many apart: one division at the start, an addition and a comparison each.  (20 000 points of 9 x 256 bf16 with
// indices, forward 37.0 us and backward 45.9; with a division per row 38.8 and 49.6.)
template <bool FLAT> struct RowWalk {
    const Mask &mask;
    int positions, apart, points_on, positions_on;
    __device__ __forceinline__ RowWalk(const Mask &mask, int positions, int apart) : mask(mask), positions(positions), apart(apart), points_on(apart / positions), positions_on(apart % positions) {}
    __device__ __forceinline__ Row<FLAT> start(int64_t r) const { return FLAT ? Row<FLAT>{r, 0, 0} : Row<FLAT>{r, r / positions, static_cast<int>(r % positions)}; }
    __device__ __forceinline__ Row<FLAT> next(Row<FLAT> row) const
    {
        row.r += apart;
        if (!FLAT) {
            const RowPlace to = row_place_on(RowPlace{row.point, row.position}, points_on, positions_on, positions);
            row.point = to.point;
            row.position = to.position;
        }
        return row;
    }
    __device__ __forceinline__ int64_t at(const Rows &v, const Row<FLAT> &row) const
    {
        return FLAT ? row.r * v.position_stride : row.point * v.point_stride + row.position * v.position_stride;
    }
    __device__ __forceinline__ uint64_t number(const Row<FLAT> &row) const          // of the row among all rows of all data points
    {
        if (FLAT || !mask.point_dev) return static_cast<uint64_t>(mask.first_point) * positions + row.r;
        return static_cast<uint64_t>(mask.point_dev[row.point]) * positions + row.position;
    }
    // the next U rows; those past the end are the first one once more
    template <int U> __device__ __forceinline__ void rows(Row<FLAT> (&out)[U], Row<FLAT> &row, int64_t end) const
    {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            out[u] = row;
            if (u > 0 && row.r >= end) out[u] = out[0];
            row = next(row);
        }
    }
};

// the elements behind a row's whole chunks, fewer than a chunk has, and their draws
template <bool BF16, int VEC> __device__ __forceinline__ void read_tail(float (&v)[VEC], const typename Element<BF16>::type *from, int left)
{
#pragma unroll
    for (int i = 0; i < VEC - 1; ++i)
        if (i < left) v[i] = Element<BF16>::get(from + i);
}
template <int WORDS> __device__ __forceinline__ void tail_words(uint64_t (&word)[WORDS], uint64_t state, int left)
{
    word[0] = splitmix_mix(state);
    if constexpr (WORDS > 1) word[1] = left > 4 ? splitmix_mix(state + kGolden) : 0;
}

template <bool BF16, bool FLAT, bool RESIDUAL>
__global__ void __launch_bounds__(kThreads) dropout_forward_kernel(DropoutArgs a, Columns c, int64_t length)
{
    constexpr int VEC = BF16 ? 8 : 4, U = kRowsAtOnce;
    using C = Chunk<BF16, VEC>;
    using E = Element<BF16>;
    using T = typename C::element;
    const int words = (a.shape.channels + 3) / 4;
    const int64_t begin = blockIdx.y * length, end = min(begin + length, a.shape.points * a.shape.positions);
    const uint64_t key = mask_key(a.mask);
    const T *x = static_cast<const T *>(a.x.p), *residual = static_cast<const T *>(a.residual.p);
    T *y = static_cast<T *>(a.y.p);

    const int across = min(c.across, c.chunks - static_cast<int>(blockIdx.x) * c.across);
    const int tx = threadIdx.x % max(c.across, 1), ty = threadIdx.x / max(c.across, 1);
    if (tx < across && ty < c.down) {
        const int channel = (blockIdx.x * c.across + tx) * VEC;
        float bias[VEC];
#pragma unroll
        for (int v = 0; v < VEC; ++v) bias[v] = a.bias ? a.bias[channel + v] : 0.f;
        const RowWalk<FLAT> walk(a.mask, a.shape.positions, c.down);
        for (Row<FLAT> row = walk.start(begin + ty); row.r < end;) {
            Row<FLAT> rows[U];
            const int64_t first = row.r;
            walk.rows(rows, row, end);
            typename C::raw in[U], add[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                in[u] = C::load_once(x + walk.at(a.x, rows[u]) + channel);
                if constexpr (RESIDUAL) add[u] = C::load_once(residual + walk.at(a.residual, rows[u]) + channel);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (first + u * c.down >= end) break;
                float v[VEC], s[VEC];
                C::widen(in[u], v);
                if constexpr (RESIDUAL) C::widen(add[u], s);
                const uint64_t state = key + (walk.number(rows[u]) * words + channel / 4 + 1) * kGolden;
#pragma unroll
                for (int w = 0; w < VEC / 4; ++w) {
                    const uint64_t word = splitmix_mix(state + w * kGolden);
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const int i = 4 * w + f;
                        const float t = kept(word, f, a.mask.least) ? (v[i] + bias[i]) * a.mask.scale : 0.f;
                        v[i] = RESIDUAL ? s[i] + t : t;
                    }
                }
                C::store(y + walk.at(a.y, rows[u]) + channel, C::narrow(v));
            }
        }
    }
    const int left = a.shape.channels - c.chunks * VEC;
    if (left > 0 && blockIdx.x == gridDim.x - 1) {
        // a thread stays with its channel: rows side by side in what a multiple of `left` threads leaves
        const int down = kThreads / left, at = c.chunks * VEC + threadIdx.x % left;
        if (static_cast<int>(threadIdx.x) >= down * left) return;
        const RowWalk<FLAT> walk(a.mask, a.shape.positions, down);
        const float bias = a.bias ? a.bias[at] : 0.f;
        for (Row<FLAT> r = walk.start(begin + threadIdx.x / left); r.r < end; r = walk.next(r)) {
            const uint64_t word = splitmix_mix(key + (walk.number(r) * words + at / 4 + 1) * kGolden);
            float t = kept(word, at % 4, a.mask.least) ? (E::get(x + walk.at(a.x, r) + at) + bias) * a.mask.scale : 0.f;
            if constexpr (RESIDUAL) t += E::get(residual + walk.at(a.residual, r) + at);
            E::put(y + walk.at(a.y, r) + at, t);
        }
    }
}

// dx, and the sums of a piece's columns into its row of parts.
template <bool BF16, bool FLAT, bool DX, bool SUMS>
__global__ void __launch_bounds__(kThreads) dropout_backward_kernel(DropoutGradArgs a, Columns c, Pieces pieces, float *parts)
{
    constexpr int VEC = BF16 ? 8 : 4, U = kRowsAtOnce;
    using C = Chunk<BF16, VEC>;
    using E = Element<BF16>;
    using T = typename C::element;
    __shared__ float lds[kThreads * VEC];
    const int words = (a.shape.channels + 3) / 4;
    const Piece piece = find_piece(pieces, blockIdx.y);
    const uint64_t key = mask_key(a.mask);
    const T *dy = static_cast<const T *>(a.dy.p);
    T *dx = static_cast<T *>(a.dx.p);

    const int across = min(c.across, c.chunks - static_cast<int>(blockIdx.x) * c.across);
    const int tx = threadIdx.x % max(c.across, 1), ty = threadIdx.x / max(c.across, 1);
    const int channel = (blockIdx.x * c.across + tx) * VEC;
    float sum[VEC];
#pragma unroll
    for (int v = 0; v < VEC; ++v) sum[v] = 0.f;
    if (tx < across && ty < c.down) {
        const RowWalk<FLAT> walk(a.mask, a.shape.positions, c.down);
        for (Row<FLAT> row = walk.start(piece.begin + ty); row.r < piece.end;) {
            Row<FLAT> rows[U];
            const int64_t first = row.r;
            walk.rows(rows, row, piece.end);
            typename C::raw in[U];
#pragma unroll
            for (int u = 0; u < U; ++u) in[u] = C::load_once(dy + walk.at(a.dy, rows[u]) + channel);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (first + u * c.down >= piece.end) break;
                float v[VEC];
                C::widen(in[u], v);
                const uint64_t state = key + (walk.number(rows[u]) * words + channel / 4 + 1) * kGolden;
#pragma unroll
                for (int w = 0; w < VEC / 4; ++w) {
                    const uint64_t word = splitmix_mix(state + w * kGolden);
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const int i = 4 * w + f;
                        v[i] = kept(word, f, a.mask.least) ? v[i] * a.mask.scale : 0.f;
                        sum[i] += v[i];
                    }
                }
                if constexpr (DX) C::store(dx + walk.at(a.dx, rows[u]) + channel, C::narrow(v));
            }
        }
    }
    if constexpr (SUMS) {
        if (c.across > 0) {
            const int width = c.across * VEC;
            if (ty < c.down) {
#pragma unroll
                for (int v = 0; v < VEC; ++v) lds[ty * width + tx * VEC + v] = sum[v];
            }
            // columns' sums, side by side by as many threads as there are, then by one each
            const int shares = max(1, kThreads / width);
            __syncthreads();
            float s = 0.f;
            if (shares > 1) {
                const int col = threadIdx.x % width, share = threadIdx.x / width;
                if (share < shares)
                    for (int r = share; r < c.down; r += shares) s += lds[r * width + col];
                __syncthreads();
                if (share < shares) lds[share * width + col] = s;
                __syncthreads();
            }
            const int rows = shares > 1 ? min(shares, c.down) : c.down;
            for (int col = threadIdx.x; col < across * VEC; col += kThreads) {
                s = 0.f;
                for (int r = 0; r < rows; ++r) s += lds[r * width + col];
                parts[int64_t(blockIdx.y) * a.shape.channels + blockIdx.x * width + col] = s;
            }
        }
    }
    const int left = a.shape.channels - c.chunks * VEC;
    if (left > 0 && blockIdx.x == gridDim.x - 1) {
        const int at = c.chunks * VEC;
#pragma unroll
        for (int v = 0; v < VEC; ++v) sum[v] = 0.f;
        const RowWalk<FLAT> walk(a.mask, a.shape.positions, kThreads);
        for (Row<FLAT> row = walk.start(piece.begin + threadIdx.x); row.r < piece.end;) {
            Row<FLAT> rows[kTailsAtOnce];
            const int64_t first = row.r;
            walk.rows(rows, row, piece.end);
            float v[kTailsAtOnce][VEC];
#pragma unroll
            for (int u = 0; u < kTailsAtOnce; ++u) read_tail<BF16>(v[u], dy + walk.at(a.dy, rows[u]) + at, left);
#pragma unroll
            for (int u = 0; u < kTailsAtOnce; ++u) {
                if (first + u * kThreads >= piece.end) break;
                uint64_t word[VEC / 4];
                tail_words(word, key + (walk.number(rows[u]) * words + at / 4 + 1) * kGolden, left);
#pragma unroll
                for (int i = 0; i < VEC - 1; ++i) {
                    if (i >= left) break;
                    const float t = kept(word[i / 4], i % 4, a.mask.least) ? v[u][i] * a.mask.scale : 0.f;
                    sum[i] += t;
                    if constexpr (DX) E::put(dx + walk.at(a.dx, rows[u]) + at + i, t);
                }
            }
        }
        if constexpr (SUMS) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < VEC - 1; ++i) {
                if (i >= left) break;
                const float s = lanes_total<64>(sum[i]);
                if (threadIdx.x % 64 == 0) lds[threadIdx.x / 64 * VEC + i] = s;
            }
            __syncthreads();
            if (static_cast<int>(threadIdx.x) < left) {
                float s = 0.f;
                for (int w = 0; w < kThreads / 64; ++w) s += lds[w * VEC + threadIdx.x];
                parts[int64_t(blockIdx.y) * a.shape.channels + at + threadIdx.x] = s;
            }
        }
    }
}

constexpr int kUnits = 256;

// rows of a workgroup: enough workgroups to fill the chip several times, and a few steps for each
int64_t rows_of_workgroup(int64_t rows, const Columns &c, int workgroups_per_unit, int steps)
{
    const int64_t step = int64_t(c.down) * kRowsAtOnce;
    const int64_t wanted = std::max<int64_t>(1, kUnits * workgroups_per_unit / tiles_of(c));
    int64_t length = (rows + wanted - 1) / wanted;
    length = (length + step - 1) / step * step;
    length = std::max<int64_t>(length, std::min(step * steps, (rows + step - 1) / step * step));
    return std::max<int64_t>(length, 1);
}

bool one_stride(const Rows &v, const LayerShape &s) { return s.points <= 1 || s.positions == 1 || v.point_stride == v.position_stride * s.positions; }
// with one position per point it is the points that have the stride
Rows flattened(Rows v, const LayerShape &s)
{
    if (s.positions == 1) v.position_stride = v.point_stride;
    return v;
}

int64_t piece_length(const LayerShape &shape)
{
    const Columns c = columns_of(shape.channels, shape.bf16 ? 8 : 4);
    return rows_of_workgroup(shape.points * shape.positions, c, 4, 4);
}

}  // namespace

size_t dropout_backward_bytes(const LayerShape &shape, const int64_t *bounds, int runs)
{
    const int64_t pieces = most_pieces(bounds, runs, shape.positions, piece_length(shape));
    return static_cast<size_t>(pieces + rows_beside(pieces, runs)) * shape.channels * sizeof(float);
}

hipError_t launch_dropout_forward(const DropoutArgs &args, hipStream_t stream)
{
    if (args.shape.points == 0) return hipSuccess;
    DropoutArgs a = args;
    const bool residual = a.residual.p != nullptr;
    const bool flat = !a.mask.point_dev && one_stride(a.x, a.shape) && one_stride(a.y, a.shape) && (!residual || one_stride(a.residual, a.shape));
    if (flat) {
        a.x = flattened(a.x, a.shape);
        a.y = flattened(a.y, a.shape);
        a.residual = flattened(a.residual, a.shape);
    }
    const Columns c = columns_of(a.shape.channels, a.shape.bf16 ? 8 : 4);
    const int64_t rows = a.shape.points * a.shape.positions, length = rows_of_workgroup(rows, c, 16, 1);
    const dim3 grid(tiles_of(c), static_cast<unsigned>((rows + length - 1) / length));
    auto pick = [&](auto bf16, auto is_flat) {
        constexpr bool B = decltype(bf16)::value, F = decltype(is_flat)::value;
        (residual ? dropout_forward_kernel<B, F, true> : dropout_forward_kernel<B, F, false>)<<<grid, kThreads, 0, stream>>>(a, c, length);
    };
    using Yes = std::true_type;
    using No = std::false_type;
    a.shape.bf16 ? flat ? pick(Yes(), Yes()) : pick(Yes(), No()) : flat ? pick(No(), Yes()) : pick(No(), No());
    return hipGetLastError();
}

hipError_t launch_dropout_backward(const DropoutGradArgs &args, void *workspace, hipStream_t stream)
{
    DropoutGradArgs a = args;
    if (!a.dx.p && !a.dbias) return hipSuccess;
    const bool flat = !a.mask.point_dev && one_stride(a.dy, a.shape) && (!a.dx.p || one_stride(a.dx, a.shape));
    if (flat) {
        a.dy = flattened(a.dy, a.shape);
        a.dx = flattened(a.dx, a.shape);
    }
    const Columns c = columns_of(a.shape.channels, a.shape.bf16 ? 8 : 4);
    const int64_t length = piece_length(a.shape);
    float *parts = static_cast<float *>(workspace), *beside = a.dbias ? parts + most_pieces(a.bounds, a.runs, a.shape.positions, length) * a.shape.channels : nullptr;
    for (int r = 0; r < a.runs; r += Pieces::kRuns) {
        Pieces p;
        const int count = lay_out_pieces(a.bounds + r, std::min(Pieces::kRuns, a.runs - r), a.shape.positions, length, &p);
        float *sums = a.dbias ? a.dbias + int64_t(r) * a.shape.channels : nullptr;
        const bool direct = one_each(p);
        if (count > 0) {
            // far fewer than the grid's second dimension takes: at most one for each wanted workgroup and run
            const dim3 grid(tiles_of(c), count);
            auto pick = [&](auto bf16, auto is_flat) {
                constexpr bool B = decltype(bf16)::value, F = decltype(is_flat)::value;
                (!a.dbias ? dropout_backward_kernel<B, F, true, false> : a.dx.p ? dropout_backward_kernel<B, F, true, true> : dropout_backward_kernel<B, F, false, true>)
                    <<<grid, kThreads, 0, stream>>>(a, c, p, direct ? sums : parts);
            };
            using Yes = std::true_type;
            using No = std::false_type;
            a.shape.bf16 ? flat ? pick(Yes(), Yes()) : pick(Yes(), No()) : flat ? pick(No(), Yes()) : pick(No(), No());
        }
        if (sums && !direct) launch_sum_pieces(parts, nullptr, a.shape.channels, p, beside, sums, nullptr, stream);
    }
    return hipGetLastError();
}

}  // namespace cr

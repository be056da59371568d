// Rows of a table looked up by tokens, and the table's gradient, for gfx950.
//
// A row of the gradient is a sum over the positions that have its token.  Their order is made fixed by sorting the positions by token, stably: a token's
// positions, and with them the runs, ascend within its stretch.
//
//   embedding_forward_kernel   chunks of 16 bytes of the rows of y, side by side
//   sort_count_kernel, sort_place_kernel   a stable sort by eight bits of the tokens, in as many passes as the vocabulary has bytes
//   embedding_sums_kernel      pieces of the sorted positions: sums of a cell (a run's token) that lies in a piece go to the gradient, others to the workspace
//   embedding_join_kernel      cells of several pieces
//   embedding_zeros_kernel     the rows of the gradient that no position has
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256;

// n / d for n < 2^31, by a product
struct Divisor {
    uint32_t d, magic, shift;
    explicit Divisor(uint32_t divisor) : d(divisor), shift(0)
    {
        while ((uint64_t(1) << shift) < d) ++shift;
        magic = static_cast<uint32_t>(((uint64_t(1) << 32) * ((uint64_t(1) << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t n) const { return (__umulhi(n, magic) + n) >> shift; }
};

// Rows numbered through points and positions.
struct Walk {
    int64_t point_stride, position_stride;
    Divisor positions;
    Walk(const Rows &r, int per_point) : point_stride(r.point_stride), position_stride(r.position_stride), positions(per_point) {}
    __device__ __forceinline__ int64_t at(uint32_t row) const
    {
        const uint32_t n = positions.of(row);
        return n * point_stride + (row - n * positions.d) * position_stride;
    }
};

// ---- forward ---------------------------------------------------------------------------------------------------------------------
constexpr int kChunks = 4;       // of a thread

template <bool TABLE_BF16, int VEC> __device__ __forceinline__ void load_table(const void *table, int64_t at, float (&v)[VEC])
{
    using T = typename Element<TABLE_BF16>::type;
    const T *p = static_cast<const T *>(table) + at;
    if constexpr (VEC == 1) {
        v[0] = Element<TABLE_BF16>::get(p);
    } else if constexpr (TABLE_BF16) {
        static_assert(VEC == 8);
        Chunk<true, 8>::widen(Chunk<true, 8>::load(p), v);
    } else {
#pragma unroll
        for (int h = 0; h < VEC / 4; ++h) {
            float w[4];
            Chunk<false, 4>::widen(Chunk<false, 4>::load(p + 4 * h), w);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = w[i];
        }
    }
}
template <bool BF16, int VEC> __device__ __forceinline__ void store_row(void *y, int64_t at, const float (&v)[VEC])
{
    using T = typename Element<BF16>::type;
    T *p = static_cast<T *>(y) + at;
    if constexpr (VEC == 1) {
        Element<BF16>::put(p, v[0]);
    } else if constexpr (BF16) {
        static_assert(VEC == 8);
        Chunk<true, 8>::store(p, Chunk<true, 8>::narrow(v));
    } else {
#pragma unroll
        for (int h = 0; h < VEC / 4; ++h) Chunk<false, 4>::store(p + 4 * h, f4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]});
    }
}

// VEC channels a chunk: 8 where either side is bf16, else 4; the last chunk of a row is moved back to end with it, and stores the same bits twice.
template <bool BF16, bool TABLE_BF16, int VEC>
__global__ void __launch_bounds__(kThreads) embedding_forward_kernel(EmbeddingArgs a, Walk tokens, Walk out, Divisor per_row, int64_t chunks)
{
    const int C = a.shape.channels, nq = per_row.d;
    constexpr int kBlock = kThreads * kChunks;
    for (int64_t first = int64_t(blockIdx.x) * kBlock; first < chunks; first += int64_t(gridDim.x) * kBlock) {
        const int64_t row0 = first / nq;
        const uint32_t inside = static_cast<uint32_t>(first - row0 * nq);
        uint32_t row[kChunks];
        int64_t token[kChunks];
        int at[kChunks];
        float v[kChunks][VEC];
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int64_t last = chunks - 1 - first;
            const uint32_t l = inside + static_cast<uint32_t>(std::min<int64_t>(threadIdx.x + k * kThreads, last)), r = per_row.of(l);
            row[k] = static_cast<uint32_t>(row0) + r;
            const int q = l - r * nq;
            at[k] = q < nq - 1 ? q * VEC : C - VEC;
            token[k] = static_cast<const int64_t *>(a.tokens.p)[tokens.at(row[k])];
        }
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
            const int64_t t = token[k] >= 0 && token[k] < a.vocabulary ? token[k] : 0;
            load_table<TABLE_BF16, VEC>(a.table, t * C + at[k], v[k]);
        }
#pragma unroll
        for (int k = 0; k < kChunks; ++k) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[k][i] = token[k] < 0 ? 0.f : token[k] >= a.vocabulary ? __builtin_nanf("") : v[k][i] * a.scale;
            store_row<BF16, VEC>(a.y.p, out.at(row[k]) + at[k], v[k]);
        }
    }
}

template <bool BF16, bool TABLE_BF16> void launch_forward(const EmbeddingArgs &a, hipStream_t stream)
{
    constexpr int VEC = BF16 || TABLE_BF16 ? 8 : 4;
    const int C = a.shape.channels, nq = C < VEC ? C : (C + VEC - 1) / VEC;
    const int64_t chunks = a.shape.points * a.shape.positions * nq;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>((chunks + kThreads * kChunks - 1) / (kThreads * kChunks), 1 << 20));
    const Walk tokens(a.tokens, a.shape.positions), out(a.y, a.shape.positions);
    (C < VEC ? embedding_forward_kernel<BF16, TABLE_BF16, 1> : embedding_forward_kernel<BF16, TABLE_BF16, VEC>)<<<grid, kThreads, 0, stream>>>(a, tokens, out, Divisor(nq), chunks);
}

// ---- the sort --------------------------------------------------------------------------------------------------------------------
constexpr int kDigits = 256;                             // of a pass
constexpr int kWaves = kThreads / 64, kKeysOfLane = 16;
constexpr int kTile = kThreads * kKeysOfLane;            // positions that a workgroup sorts at once: a stretch of 1 024 per wavefront
constexpr int kMostBlocks = 512;                         // of a pass, each with as many tiles as it takes

// Runs of a batch, by the first of their points in it.
struct BatchRuns {
    static constexpr int kRuns = 128;
    int runs;
    int first[kRuns + 1];
    __device__ __forceinline__ int of(int point) const   // the last run that begins at or before the point: those before it that begin there are empty
    {
        int lo = 0, hi = runs;
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (first[mid] <= point) lo = mid;
            else hi = mid;
        }
        return lo;
    }
};

struct SortPass {
    const int64_t *tokens;                               // of the first pass, null later
    Walk walk;
    uint32_t vocabulary;
    const uint32_t *keys, *order;                        // of later passes: tokens, `vocabulary` for none, and positions
    uint32_t *keys_out, *order_out;
    uint8_t *run_out;                                    // of the last pass, if there are several runs
    uint32_t *counts;                                    // [workgroup][digit]
    uint32_t n;                                          // positions
    int tiles, shift;                                    // tiles of a workgroup
    __device__ __forceinline__ uint32_t key(uint32_t i) const
    {
        if (!tokens) return keys[i];
        const int64_t t = tokens[walk.at(i)];
        return t >= 0 && t < vocabulary ? static_cast<uint32_t>(t) : vocabulary;
    }
};

__global__ void __launch_bounds__(kThreads) sort_count_kernel(SortPass s, uint64_t *bits, int64_t words)
{
    __shared__ uint32_t count[kDigits];
    for (int64_t w = int64_t(blockIdx.x) * kThreads + threadIdx.x; w < words; w += int64_t(gridDim.x) * kThreads) bits[w] = 0;
    count[threadIdx.x] = 0;
    __syncthreads();
    const uint64_t begin = uint64_t(blockIdx.x) * s.tiles * kTile, end = std::min<uint64_t>(begin + uint64_t(s.tiles) * kTile, s.n);
    for (uint64_t i = begin + threadIdx.x; i < end; i += kThreads) atomicAdd(&count[s.key(static_cast<uint32_t>(i)) >> s.shift & (kDigits - 1)], 1u);
    __syncthreads();
    s.counts[blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

// A key's place: keys with smaller digits, keys with its digit in earlier workgroups, in earlier tiles, wavefronts, and steps of its wavefront, and in
// lower lanes.
__global__ void __launch_bounds__(kThreads) sort_place_kernel(SortPass s, BatchRuns runs)
{
    __shared__ uint32_t place[kWaves][kDigits], totals[kWaves];
    const int digit = threadIdx.x, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t total = 0, before = 0;
    for (unsigned b = 0; b < gridDim.x; ++b) {
        const uint32_t c = s.counts[b * kDigits + digit];
        if (b < blockIdx.x) before += c;
        total += c;
    }
    uint32_t sum = total;                                // inclusive over the digits
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == 63) totals[wave] = sum;
    __syncthreads();
    uint32_t next = before + sum - total;                // the place of the next key with this thread's digit
    for (int w = 0; w < wave; ++w) next += totals[w];

    const uint64_t begin = uint64_t(blockIdx.x) * s.tiles * kTile;
    for (int tile = 0; tile < s.tiles; ++tile) {
        const uint64_t first = begin + uint64_t(tile) * kTile;
        if (first >= s.n) break;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) place[w][digit] = 0;
        __syncthreads();
        uint32_t key[kKeysOfLane], order[kKeysOfLane], rank[kKeysOfLane];
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            const uint64_t i = first + wave * (kTile / kWaves) + u * 64 + lane;
            const uint32_t j = static_cast<uint32_t>(std::min<uint64_t>(i, s.n - 1));
            key[u] = s.key(j);
            order[u] = s.tokens ? j : s.order[j];
        }
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            const bool is = first + wave * (kTile / kWaves) + u * 64 + lane < s.n;
            const uint32_t d = key[u] >> s.shift & (kDigits - 1);
            uint64_t same = __ballot(is);
#pragma unroll
            for (int b = 0; b < 8; ++b) {
                const uint64_t set = __ballot(d >> b & 1);
                same &= d >> b & 1 ? set : ~set;
            }
            const int leader = is ? __ffsll(static_cast<long long>(same)) - 1 : lane;
            uint32_t old = 0;
            if (is && lane == leader) old = atomicAdd(&place[wave][d], static_cast<uint32_t>(__popcll(same)));
            rank[u] = __shfl(old, leader) + __popcll(same & ((uint64_t(1) << lane) - 1));
        }
        __syncthreads();
        for (int w = 0; w < kWaves; ++w) {
            const uint32_t c = place[w][digit];
            place[w][digit] = next;
            next += c;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            if (first + wave * (kTile / kWaves) + u * 64 + lane >= s.n) continue;
            const uint32_t to = place[wave][key[u] >> s.shift & (kDigits - 1)] + rank[u];
            s.keys_out[to] = key[u];
            s.order_out[to] = order[u];
            if (s.run_out) s.run_out[to] = static_cast<uint8_t>(runs.of(static_cast<int>(s.walk.positions.of(order[u]))));
        }
    }
}

// ---- the sums --------------------------------------------------------------------------------------------------------------------
// Positions in the order of their cells; a cell is a token of a run.
struct Sorted {
    const uint32_t *keys, *order;
    const uint8_t *run;                                  // or null: one run
    uint32_t n, vocabulary;
    int length;                                          // positions of a piece
    unsigned pieces;
};
struct Cell {
    uint32_t key, run;
    __device__ __forceinline__ bool operator==(const Cell &o) const { return key == o.key && run == o.run; }
};
__device__ __forceinline__ Cell cell_at(const Sorted &s, uint32_t i) { return {s.keys[i], s.run ? s.run[i] : 0u}; }

struct Gradient {
    const void *dy;
    Walk walk;
    int channels;
    float scale;
    float *dtable, *parts;                               // parts: two rows a piece, what began before it and what goes on behind it
    uint64_t *bits;                                      // a bit for each cell that has positions
    int64_t words;                                       // of a run
};

constexpr int kRowsAtOnce = 8;

// TS lanes per piece, each with a chunk of the channels; a wavefront per piece and 64 chunks where there are more.
template <bool BF16, int VEC, int TS> __global__ void __launch_bounds__(kThreads) embedding_sums_kernel(Gradient g, Sorted s, int nq, unsigned slabs)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const uint64_t teams = uint64_t(s.pieces) * slabs;
    for (uint64_t team = uint64_t(blockIdx.x) * (kThreads / TS) + threadIdx.x / TS; team < teams; team += uint64_t(gridDim.x) * (kThreads / TS)) {
        const unsigned piece = static_cast<unsigned>(team / slabs);
        const int q = static_cast<int>(team % slabs) * TS + threadIdx.x % TS;
        if (q >= nq) continue;
        const uint32_t begin = piece * s.length, end = min(begin + s.length, s.n);
        const int at = q < nq - 1 ? q * VEC : g.channels - VEC;
        const T *dy = static_cast<const T *>(g.dy) + at;
        Cell now = cell_at(s, begin);
        if (now.key >= s.vocabulary) continue;               // nothing but positions without a row from here on
        bool begun = begin == 0 || !(cell_at(s, begin - 1) == now);
        float acc[VEC];
    #pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
        auto leave = [&](bool ends) {
            if (now.key >= s.vocabulary) return;
            if (begun && q == 0) atomicOr(reinterpret_cast<unsigned long long *>(g.bits + now.run * g.words + now.key / 64), 1ull << now.key % 64);
            float *to;
            float by = 1.f;
            if (begun && ends) {
                to = g.dtable + (int64_t(now.run) * s.vocabulary + now.key) * g.channels;
                by = g.scale;
            } else {
                to = g.parts + (2 * int64_t(piece) + begun) * g.channels;
            }
            float v[VEC];
    #pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = acc[i] * by;
            store_row<false, VEC>(to, at, v);
        };
        for (uint32_t e = begin; e < end; e += kRowsAtOnce) {
            Cell cell[kRowsAtOnce];
            typename C::raw raw[kRowsAtOnce];
    #pragma unroll
            for (int u = 0; u < kRowsAtOnce; ++u) {
                const uint32_t i = min(e + u, end - 1);
                cell[u] = cell_at(s, i);
                raw[u] = C::load(dy + g.walk.at(s.order[i]));
            }
    #pragma unroll
            for (int u = 0; u < kRowsAtOnce; ++u) {
                if (e + u < end) {
                    if (!(cell[u] == now)) {
                        leave(true);
                        now = cell[u];
                        begun = true;
    #pragma unroll
                        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
                    }
                    float v[VEC];
                    C::widen(raw[u], v);
    #pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] += v[i];
                }
            }
        }
        leave(end == s.n || !(cell_at(s, end) == now));
    }
}

// The cell that begins in a piece and goes on behind it: its parts, added up in 64 bits.
__global__ void __launch_bounds__(kThreads) embedding_join_kernel(Gradient g, Sorted s)
{
    __shared__ double meet[kWaves][64 * 4];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const unsigned piece = blockIdx.x;
    const uint32_t begin = piece * s.length, end = min(begin + s.length, s.n);
    if (end == s.n) return;
    const Cell now = cell_at(s, end - 1);
    if (now.key >= s.vocabulary || !(cell_at(s, end) == now)) return;
    if (begin > 0 && cell_at(s, begin - 1) == now) return;           // it began before
    unsigned more = 0;                                   // pieces behind this one that the cell reaches into
    for (;;) {
        const unsigned i = piece + 1 + more + threadIdx.x;
        const int count = __syncthreads_count(i < s.pieces && cell_at(s, i * s.length) == now);
        more += count;
        if (count < kThreads) break;
    }
    for (int64_t c0 = int64_t(blockIdx.y) * 256; c0 < g.channels; c0 += int64_t(gridDim.y) * 256) {
        double sum[4] = {};
        constexpr int U = 4;
        for (unsigned p = wave; p <= more; p += U * kWaves) {
            float v[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const unsigned pu = min(p + u * kWaves, more);
                const float *row = g.parts + (2 * int64_t(piece + pu) + (pu == 0)) * g.channels;
#pragma unroll
                for (int i = 0; i < 4; ++i) v[u][i] = row[std::min<int64_t>(c0 + i * 64 + lane, g.channels - 1)];
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] += p + u * kWaves <= more ? v[u][i] : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) meet[wave][i * 64 + lane] = sum[i];
        __syncthreads();
        double total = 0.0;
        for (int w = 0; w < kWaves; ++w) total += meet[w][threadIdx.x];
        const int64_t c = c0 + threadIdx.x;
        if (c < g.channels) g.dtable[(int64_t(now.run) * s.vocabulary + now.key) * g.channels + c] = static_cast<float>(total) * g.scale;
        __syncthreads();
    }
}

// Rows without positions, a few neighbours at a time; bits null: all rows.
__global__ void __launch_bounds__(kThreads) embedding_zeros_kernel(float *dtable, int channels, int vocabulary, int runs, const uint64_t *bits, int64_t words, int neighbours)
{
    const f4 none = {0.f, 0.f, 0.f, 0.f};
    const int64_t groups = (vocabulary + neighbours - 1) / neighbours, all = groups * runs;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const int64_t run = i / groups;
        const int first = static_cast<int>(i - run * groups) * neighbours, count = min(neighbours, vocabulary - first);
        float *rows = dtable + (run * vocabulary + first) * channels;
        uint64_t have = bits ? bits[run * words + first / 64] >> first % 64 : 0;
        if (count < 64) have &= (uint64_t(1) << count) - 1;
        auto clear = [&](float *from, int64_t floats) {
            const int64_t whole = floats / 4;
            for (int64_t c = int64_t(blockIdx.y) * kThreads + threadIdx.x; c < whole; c += int64_t(gridDim.y) * kThreads) Chunk<false, 4>::store(from + 4 * c, none);
            if (blockIdx.y == 0 && threadIdx.x < floats - 4 * whole) from[4 * whole + threadIdx.x] = 0.f;
        };
        if (have == 0) {
            clear(rows, int64_t(count) * channels);
        } else {
            for (int r = 0; r < count; ++r)
                if (!(have >> r & 1)) clear(rows + int64_t(r) * channels, channels);
        }
    }
}

// ---- what a gradient needs -------------------------------------------------------------------------------------------------------
struct GradPlan {
    uint32_t n;                  // positions of the largest batch of runs
    int passes;
    int vec, nq, team;           // channels of a chunk, chunks of a row, lanes of a piece
    unsigned slabs;
    int64_t words;               // of bits, per run
    size_t keys[2], order[2], run, counts, parts, bits, bytes;       // offsets
};
unsigned blocks_of(uint32_t n) { return std::min<unsigned>((uint64_t(n) + kTile - 1) / kTile, kMostBlocks); }
// Pieces that give some 8 192 wavefronts, of 16 to 256 positions.
int piece_length(uint32_t n, int team, unsigned slabs)
{
    int length = 16;
    while (length < 256 && uint64_t(n) * slabs * team / 64 > uint64_t(length) * 8192) length *= 2;
    return length;
}

GradPlan plan_gradient(const LayerShape &shape, int vocabulary, const int64_t *bounds, int runs, uint32_t n)
{
    GradPlan p = {};
    p.n = n;
    for (p.passes = 1; p.passes < 4 && (uint64_t(vocabulary) >> (8 * p.passes)) != 0; ++p.passes) {}
    p.vec = shape.bf16 ? 8 : 4;
    if (shape.channels < p.vec) p.vec = 1;
    p.nq = (shape.channels + p.vec - 1) / p.vec;
    for (p.team = 1; p.team < 64 && p.team < p.nq;) p.team *= 2;
    p.slabs = (p.nq + p.team - 1) / p.team;
    p.words = (int64_t(vocabulary) + 63) / 64;
    const int length = piece_length(n, p.team, p.slabs);
    const uint64_t pieces = (uint64_t(n) + length - 1) / length;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        p.keys[i] = take(size_t(n) * 4);
        p.order[i] = take(size_t(n) * 4);
    }
    p.run = take(runs > 1 ? n : 0);
    p.counts = take(size_t(blocks_of(n)) * kDigits * 4);
    p.parts = take(pieces * 2 * shape.channels * 4);
    p.bits = take(size_t(std::min(runs, BatchRuns::kRuns)) * p.words * 8);
    p.bytes = at;
    return p;
}
uint32_t most_positions(const LayerShape &shape, const int64_t *bounds, int runs)
{
    int64_t most = 0;
    for (int r = 0; r < runs; r += BatchRuns::kRuns) most = std::max(most, bounds[std::min(runs, r + BatchRuns::kRuns)] - bounds[r]);
    return static_cast<uint32_t>(most * shape.positions);
}

template <bool BF16, int VEC> void launch_sums(const Gradient &g, const Sorted &s, const GradPlan &p, hipStream_t stream)
{
    auto go = [&](auto kernel, int team) {
        const uint64_t teams = uint64_t(s.pieces) * p.slabs, per_block = kThreads / team;
        kernel<<<static_cast<unsigned>(std::min<uint64_t>((teams + per_block - 1) / per_block, 1 << 20)), kThreads, 0, stream>>>(g, s, p.nq, p.slabs);
    };
    switch (p.team) {
    case 1: return go(embedding_sums_kernel<BF16, VEC, 1>, 1);
    case 2: return go(embedding_sums_kernel<BF16, VEC, 2>, 2);
    case 4: return go(embedding_sums_kernel<BF16, VEC, 4>, 4);
    case 8: return go(embedding_sums_kernel<BF16, VEC, 8>, 8);
    }
    if constexpr (VEC > 1) {                             // rows of single channels are shorter
        if (p.team == 16) go(embedding_sums_kernel<BF16, VEC, 16>, 16);
        else if (p.team == 32) go(embedding_sums_kernel<BF16, VEC, 32>, 32);
        else go(embedding_sums_kernel<BF16, VEC, 64>, 64);
    }
}

void launch_zeros(const EmbeddingGradArgs &a, float *dtable, int runs, const uint64_t *bits, int64_t words, hipStream_t stream)
{
    int neighbours = 64;                                 // at most 64 KB of a workgroup
    while (neighbours > 1 && int64_t(neighbours) * a.shape.channels > 16384) neighbours /= 2;
    const int64_t groups = (int64_t(a.vocabulary) + neighbours - 1) / neighbours * runs;
    const dim3 grid(static_cast<unsigned>(std::min<int64_t>(groups, 1 << 20)), std::max(1, std::min(1024, a.shape.channels / 16384)));
    embedding_zeros_kernel<<<grid, kThreads, 0, stream>>>(dtable, a.shape.channels, a.vocabulary, runs, bits, words, neighbours);
}

}  // namespace

size_t embedding_backward_bytes(const LayerShape &shape, int vocabulary, const int64_t *bounds, int runs)
{
    const uint32_t n = most_positions(shape, bounds, runs);
    if (n == 0) return 0;
    size_t most = 0;                                     // pieces are shorter where there are fewer positions: every batch has to fit
    for (int r = 0; r < runs; r += BatchRuns::kRuns) {
        const int64_t points = bounds[std::min(runs, r + BatchRuns::kRuns)] - bounds[r];
        most = std::max(most, plan_gradient(shape, vocabulary, bounds, runs, static_cast<uint32_t>(points * shape.positions)).bytes);
    }
    return most;
}

hipError_t launch_embedding_forward(const EmbeddingArgs &a, hipStream_t stream)
{
    if (a.shape.points == 0) return hipSuccess;
    if (a.shape.bf16) a.table_bf16 ? launch_forward<true, true>(a, stream) : launch_forward<true, false>(a, stream);
    else a.table_bf16 ? launch_forward<false, true>(a, stream) : launch_forward<false, false>(a, stream);
    return hipGetLastError();
}

hipError_t launch_embedding_backward(const EmbeddingGradArgs &a, void *workspace, hipStream_t stream)
{
    const LayerShape &shape = a.shape;
    for (int r0 = 0; r0 < a.runs; r0 += BatchRuns::kRuns) {
        BatchRuns runs;
        runs.runs = std::min(a.runs - r0, BatchRuns::kRuns);
        const int64_t first = a.bounds[r0];
        for (int r = 0; r <= runs.runs; ++r) runs.first[r] = static_cast<int>(a.bounds[r0 + r] - first);
        float *dtable = a.dtable + int64_t(r0) * a.vocabulary * shape.channels;
        const uint32_t n = static_cast<uint32_t>((a.bounds[r0 + runs.runs] - first) * shape.positions);
        if (n == 0) {
            launch_zeros(a, dtable, runs.runs, nullptr, 0, stream);
            continue;
        }
        const GradPlan p = plan_gradient(shape, a.vocabulary, a.bounds, a.runs, n);
        char *ws = static_cast<char *>(workspace);
        auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(ws + at); };
        uint64_t *bits = reinterpret_cast<uint64_t *>(ws + p.bits);
        const unsigned blocks = blocks_of(n);
        const int tiles = static_cast<int>(((uint64_t(n) + kTile - 1) / kTile + blocks - 1) / blocks);
        for (int pass = 0; pass < p.passes; ++pass) {
            const int to = pass % 2, from = 1 - to;
            const bool last = pass == p.passes - 1;
            const SortPass s = {pass == 0 ? static_cast<const int64_t *>(a.tokens.p) + first * a.tokens.point_stride : nullptr, Walk(a.tokens, shape.positions),
                                static_cast<uint32_t>(a.vocabulary), words(p.keys[from]), words(p.order[from]), words(p.keys[to]), words(p.order[to]),
                                last && a.runs > 1 ? reinterpret_cast<uint8_t *>(ws + p.run) : nullptr, words(p.counts), n, tiles, 8 * pass};
            sort_count_kernel<<<blocks, kThreads, 0, stream>>>(s, bits, pass == 0 ? p.words * runs.runs : 0);
            sort_place_kernel<<<blocks, kThreads, 0, stream>>>(s, runs);
        }
        const int end = (p.passes - 1) % 2, length = piece_length(n, p.team, p.slabs);
        const Sorted s = {words(p.keys[end]), words(p.order[end]), a.runs > 1 ? reinterpret_cast<const uint8_t *>(ws + p.run) : nullptr, n,
                          static_cast<uint32_t>(a.vocabulary), length, static_cast<unsigned>((uint64_t(n) + length - 1) / length)};
        const size_t e = shape.bf16 ? 2 : 4;
        const Gradient g = {static_cast<const char *>(a.dy.p) + first * a.dy.point_stride * static_cast<int64_t>(e), Walk(a.dy, shape.positions), shape.channels, a.scale,
                            dtable, reinterpret_cast<float *>(ws + p.parts), bits, p.words};
        if (p.vec == 1) shape.bf16 ? launch_sums<true, 1>(g, s, p, stream) : launch_sums<false, 1>(g, s, p, stream);
        else if (shape.bf16) launch_sums<true, 8>(g, s, p, stream);
        else launch_sums<false, 4>(g, s, p, stream);
        if (s.pieces > 1) embedding_join_kernel<<<dim3(s.pieces, std::min((shape.channels + 255) / 256, 1024)), kThreads, 0, stream>>>(g, s);
        launch_zeros(a, dtable, runs.runs, bits, p.words, stream);
    }
    return hipGetLastError();
}

}  // namespace cr

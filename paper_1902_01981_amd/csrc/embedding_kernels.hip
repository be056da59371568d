// Rows of a table looked up by tokens, and the table's gradient, for gfx950.
//
// A row of the gradient is a sum over the positions that have its token.  Their order is made fixed by sorting the positions by token, stably: a token's
// positions, and with them the runs, ascend within its stretch.
//
//   embedding_forward_kernel   chunks of 16 bytes of the rows of y, side by side
//   sort_few_kernel            a stable sort of the positions by token, nine bits of it or fewer a pass, by one workgroup;
//   sort_count_kernel, sort_place_kernel   by many, a pair of launches a pass
//   embedding_sums_kernel, embedding_wide_sums_kernel   pieces of the sorted positions: sums of a cell (a run's token) that lies in a piece go to the
//                              gradient, others to the workspace; rows of the gradient that no position has are cleared beside them
//   embedding_join_kernel      cells of several pieces
//
// Reads and writes bound it.  Forward: y is written past the caches, which then keep the rows of frequent tokens: where the i-th is met as 1 / (i + 2.7),
// 8 192 x 120 x 512 bf16 of 50 008 rows takes 300 us with ordinary stores and 195 with these, 5.2 TB/s of what is written, 64 x 512 x 4 096 of 131 072 rows 79 and 64; where all
// are met as often, 281 and 273, 100 and 82.  What reads y next finds less of it in the caches: forward and dropout behind it, tokens all as frequent, 16 x 512 x 4 096 44 us and 45,
// 64 x 512 x 4 096 202 and 207, 256 x 512 x 4 096 798 and 768, 8 192 x 120 x 512 683 and 671.  Gradient: 64 x 512 x 4 096 bf16 of 131 072 rows 482 us, 5.0 TB/s, most
// of it the rows of zeros, which the sums hide behind; 8 192 x 120 x 512 of 50 008 rows 315 us, 3.5 TB/s: gathering rows of 1 KB 210, the two passes of the sort 70,
// the parts of frequent tokens 24; 683 x 9 x 1 027 fp32 with twelve runs of 5 003 rows 62 us, 4.4 TB/s.  600 positions 22 us, 3 launches; of a
// gradient of 50 MB 27 us with 1 027 channels, but 53 with 64 and 96 with 8, whose zeros go out 64 rows, 2 KB of 8 channels, a step.
#include "layers_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256;

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
constexpr int kChunks = 2;       // of a thread

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
// ONCE: past the caches
template <bool BF16, int VEC, bool ONCE = false> __device__ __forceinline__ void store_row(void *y, int64_t at, const float (&v)[VEC])
{
    constexpr int kChunk = VEC == 1 ? 1 : BF16 ? 8 : 4;
    using C = Chunk<BF16, kChunk>;
    typename C::element *p = static_cast<typename C::element *>(y) + at;
#pragma unroll
    for (int h = 0; h < VEC / kChunk; ++h) {
        float w[kChunk];
#pragma unroll
        for (int i = 0; i < kChunk; ++i) w[i] = v[h * kChunk + i];
        if constexpr (ONCE) C::store_once(p + h * kChunk, C::narrow(w));
        else C::store(p + h * kChunk, C::narrow(w));
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
            store_row<BF16, VEC, true>(a.y.p, out.at(row[k]) + at[k], v[k]);
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

// ---- rows of zeros ---------------------------------------------------------------------------------------------------------------
// Rows without positions, `neighbours` at a time; met: a byte for each row, 1 where it has positions; null: all rows are cleared.
struct Zeros {
    float *dtable;
    int channels, vocabulary, runs, neighbours, parts;   // parts: workgroups that share such rows
    const uint8_t *met;
    int64_t workgroups;
};
__device__ __forceinline__ void clear_rows(const Zeros &z, int64_t workgroup)
{
    const f4 none = {0.f, 0.f, 0.f, 0.f};
    const int part = static_cast<int>(workgroup % z.parts);
    const int64_t groups = (z.vocabulary + z.neighbours - 1) / z.neighbours, all = groups * z.runs, others = z.workgroups / z.parts;
    for (int64_t i = workgroup / z.parts; i < all; i += others) {
        const int64_t run = i / groups;
        const int first = static_cast<int>(i - run * groups) * z.neighbours, count = min(z.neighbours, z.vocabulary - first);
        float *rows = z.dtable + (run * z.vocabulary + first) * z.channels;
        uint64_t have = 0;
        if (z.met) {
            const int lane = threadIdx.x % 64;
            have = __ballot(lane < count && z.met[run * z.vocabulary + first + min(lane, count - 1)]);
        }
        auto clear = [&](float *from, int64_t floats) {
            const int64_t whole = floats / 4;
            for (int64_t c = int64_t(part) * static_cast<int>(blockDim.x) + threadIdx.x; c < whole; c += int64_t(z.parts) * static_cast<int>(blockDim.x)) Chunk<false, 4>::store(from + 4 * c, none);
            if (part == 0 && threadIdx.x < floats - 4 * whole) from[4 * whole + threadIdx.x] = 0.f;
        };
        if (have == 0) {
            clear(rows, int64_t(count) * z.channels);
        } else {
            for (int r = 0; r < count; ++r)
                if (!(have >> r & 1)) clear(rows + int64_t(r) * z.channels, z.channels);
        }
    }
}
// ---- the sort --------------------------------------------------------------------------------------------------------------------
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kKeysOfLane = 8;
constexpr int kMostTile = kSortThreads * kKeysOfLane;    // positions that a workgroup sorts at once, a stretch of them per wavefront
constexpr int kDigits = 512;                             // of a pass, at most
constexpr int kMostBlocks = 256;                         // of a pass, each with as many tiles as it takes (64 or 128: the same time, 983 040 positions)

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
    int tiles, steps, bits, shift;                       // tiles of a workgroup; steps of a wavefront in a tile; bits of a digit
    uint8_t *met;                                        // cleared and written by the first pass: see Zeros
    int64_t cells;
    __device__ __forceinline__ int tile() const { return steps * kSortThreads; }
    __device__ __forceinline__ uint32_t key(uint32_t i) const
    {
        if (!tokens) return keys[i];
        const int64_t t = tokens[walk.at(i)];
        return t >= 0 && t < vocabulary ? static_cast<uint32_t>(t) : vocabulary;
    }
    __device__ __forceinline__ void put(const BatchRuns &runs, uint32_t to, uint32_t k, uint32_t i) const
    {
        keys_out[to] = k;
        order_out[to] = i;
        if (run_out) run_out[to] = static_cast<uint8_t>(runs.of(static_cast<int>(walk.positions.of(i))));
    }
};

// A key's rank among the keys of its wavefront with its digit: those of earlier steps, and of lower lanes.  count[digit]: such keys so far.
__device__ __forceinline__ uint32_t rank_of(uint32_t digit, int bits, bool is, uint32_t *count)
{
    const int lane = threadIdx.x % 64;
    uint64_t same = __ballot(is);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot(digit >> b & 1);
        same &= digit >> b & 1 ? set : ~set;
    }
    const int leader = is ? __ffsll(static_cast<long long>(same)) - 1 : lane;
    uint32_t old = 0;
    if (is && lane == leader) old = atomicAdd(&count[digit], static_cast<uint32_t>(__popcll(same)));
    return __shfl(old, leader) + __popcll(same & ((uint64_t(1) << lane) - 1));
}
// The sum of `mine` over the digits before this thread's, a digit each of the first kDigits threads; sums: a place for each of their wavefronts.
__device__ __forceinline__ uint32_t digits_before(uint32_t mine, uint32_t *sums)
{
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    uint32_t sum = mine;                                 // up to and with this digit
    for (int d = 1; d < 64; d *= 2) {
        const uint32_t other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == 63 && wave < kDigits / 64) sums[wave] = sum;
    __syncthreads();
    uint32_t before = sum - mine;
    for (int w = 0; w < std::min(wave, kDigits / 64); ++w) before += sums[w];
    return before;
}

__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(SortPass s)
{
    __shared__ uint32_t count[kDigits];
    if (s.tokens)
        for (int64_t c = int64_t(blockIdx.x) * kSortThreads + threadIdx.x; c < s.cells; c += int64_t(gridDim.x) * kSortThreads) s.met[c] = 0;
    if (threadIdx.x < kDigits) count[threadIdx.x] = 0;
    __syncthreads();
    const uint64_t begin = uint64_t(blockIdx.x) * s.tiles * s.tile(), end = std::min<uint64_t>(begin + uint64_t(s.tiles) * s.tile(), s.n);
    for (uint64_t i = begin + threadIdx.x; i < end; i += kSortThreads) atomicAdd(&count[s.key(static_cast<uint32_t>(i)) >> s.shift & ((1u << s.bits) - 1)], 1u);
    __syncthreads();
    if (threadIdx.x < kDigits) s.counts[blockIdx.x * kDigits + threadIdx.x] = count[threadIdx.x];
}

// A key's place: keys with smaller digits, keys with its digit in earlier workgroups, in earlier tiles and wavefronts, and its rank in its own.
__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(SortPass s, BatchRuns runs)
{
    __shared__ uint32_t place[kSortWaves][kDigits], sums[kDigits / 64], halves[2][kDigits];
    const int digit = threadIdx.x % kDigits, half = threadIdx.x / kDigits, lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint32_t mask = (1u << s.bits) - 1;
    static_assert(kSortThreads == 2 * kDigits);
    uint32_t total = 0, before = 0;
    constexpr int U = 8;
    for (unsigned b = half; b < gridDim.x; b += 2 * U) {
        uint32_t c[U];
#pragma unroll
        for (int u = 0; u < U; ++u) c[u] = s.counts[std::min(b + 2 * u, gridDim.x - 1) * kDigits + digit];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            total += b + 2 * u < gridDim.x ? c[u] : 0;
            before += b + 2 * u < blockIdx.x ? c[u] : 0;
        }
    }
    if (half) {
        halves[0][digit] = total;
        halves[1][digit] = before;
    }
    __syncthreads();
    if (!half) {
        total += halves[0][digit];
        before += halves[1][digit];
    }
    uint32_t next = before + digits_before(total, sums); // the place of the next key with this thread's digit, in the first kDigits threads

    const uint64_t begin = uint64_t(blockIdx.x) * s.tiles * s.tile();
    for (int tile = 0; tile < s.tiles; ++tile) {
        const uint64_t first = begin + uint64_t(tile) * s.tile();
        if (first >= s.n) break;
        __syncthreads();
        for (int w = half; w < kSortWaves; w += 2) place[w][digit] = 0;
        __syncthreads();
        uint32_t key[kKeysOfLane], order[kKeysOfLane], rank[kKeysOfLane];
        const uint64_t own = first + wave * s.steps * 64 + lane, end = std::min<uint64_t>(s.n, first + (wave + 1) * s.steps * 64);
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            if (u >= s.steps) break;
            const uint32_t j = static_cast<uint32_t>(std::min<uint64_t>(own + u * 64, s.n - 1));
            key[u] = s.key(j);
            order[u] = s.tokens ? j : s.order[j];
        }
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            if (u >= s.steps) break;
            rank[u] = rank_of(key[u] >> s.shift & mask, s.bits, own + u * 64 < end, place[wave]);
        }
        __syncthreads();
        if (!half)
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = place[w][digit];
                place[w][digit] = next;
                next += c;
            }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u)
            if (own + u * 64 < end) {
                s.put(runs, place[wave][key[u] >> s.shift & mask] + rank[u], key[u], order[u]);
                if (s.tokens && key[u] < s.vocabulary) {
                    const int64_t run = runs.runs > 1 ? runs.of(static_cast<int>(s.walk.positions.of(order[u]))) : 0;
                    s.met[run * s.vocabulary + key[u]] = 1;
                }
            }
    }
}

// Positions that one workgroup holds: all passes in one launch.  The others clear the whole gradient meanwhile: rows that positions have are written twice,
// 8 192 of them at most.
__global__ void __launch_bounds__(kSortThreads) sort_few_kernel(SortPass s, BatchRuns runs, int passes, Zeros z)
{
    __shared__ uint32_t place[kSortWaves][kDigits], sums[kDigits / 64], keys[kMostTile];
    __shared__ uint16_t orders[kMostTile];
    if (blockIdx.x > 0) {
        clear_rows(z, blockIdx.x - 1);
        return;
    }
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64, n = static_cast<int>(s.n), steps = (n + kSortThreads - 1) / kSortThreads;
    const int own = wave * steps * 64 + lane, end = std::min(n, (wave + 1) * steps * 64);
    const uint32_t mask = (1u << s.bits) - 1;
    uint32_t key[kKeysOfLane], rank[kKeysOfLane];
    int order[kKeysOfLane];
#pragma unroll
    for (int u = 0; u < kKeysOfLane; ++u) {
        order[u] = own + u * 64;
        key[u] = u < steps ? s.key(std::min(own + u * 64, n - 1)) : 0;
    }
    for (int pass = 0; pass < passes; ++pass) {
        const int shift = pass * s.bits;
        for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) place[i / kDigits][i % kDigits] = 0;
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            if (u >= steps) break;
            rank[u] = rank_of(key[u] >> shift & mask, s.bits, own + u * 64 < end, place[wave]);
        }
        __syncthreads();
        uint32_t total = 0;
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kSortWaves; ++w) total += place[w][threadIdx.x];
        uint32_t next = digits_before(total, sums);
        if (threadIdx.x < kDigits)
            for (int w = 0; w < kSortWaves; ++w) {
                const uint32_t c = place[w][threadIdx.x];
                place[w][threadIdx.x] = next;
                next += c;
            }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u)
            if (own + u * 64 < end) {
                const uint32_t to = place[wave][key[u] >> shift & mask] + rank[u];
                keys[to] = key[u];
                orders[to] = static_cast<uint16_t>(order[u]);
            }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kKeysOfLane; ++u) {
            key[u] = keys[std::min(own + u * 64, n - 1)];
            order[u] = orders[std::min(own + u * 64, n - 1)];
        }
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kKeysOfLane; ++u)
        if (own + u * 64 < end) s.put(runs, own + u * 64, key[u], order[u]);
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
};

constexpr int kRowsAtOnce = 8;
template <int VEC> __device__ __forceinline__ int chunk_of(int q, int nq, int channels) { return q < nq - 1 ? q * VEC : channels - VEC; }

// TS lanes per piece, each with a chunk of the channels, for rows of up to 32 chunks.
template <bool BF16, int VEC, int TS> __global__ void __launch_bounds__(kThreads) embedding_sums_kernel(Gradient g, Sorted s, int nq, unsigned slabs, unsigned workgroups, Zeros z)
{
    if (blockIdx.x >= workgroups) {                      // rows that no position has, behind the sums: there is room in their gaps
        clear_rows(z, blockIdx.x - workgroups);
        return;
    }
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const uint64_t teams = uint64_t(s.pieces) * slabs;
    for (uint64_t team = uint64_t(blockIdx.x) * (kThreads / TS) + threadIdx.x / TS; team < teams; team += uint64_t(workgroups) * (kThreads / TS)) {
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

// Wider rows: a wavefront per piece and 64 chunks.  Its lanes look up 64 positions at once, what is at them is a scalar then; a row's place in the registers
// takes the row eight further on as soon as it is added.
template <bool BF16, int VEC> __global__ void __launch_bounds__(kThreads) embedding_wide_sums_kernel(Gradient g, Sorted s, int nq, unsigned slabs, unsigned workgroups, Zeros z)
{
    if (blockIdx.x >= workgroups) {                      // rows that no position has, behind the sums: there is room in their gaps
        clear_rows(z, blockIdx.x - workgroups);
        return;
    }
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int lane = threadIdx.x % 64;
    const uint64_t teams = uint64_t(s.pieces) * slabs;
    for (uint64_t team = uint64_t(blockIdx.x) * (kThreads / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); team < teams; team += uint64_t(workgroups) * (kThreads / 64)) {
        const unsigned piece = static_cast<unsigned>(team / slabs);
        const int q = static_cast<int>(team % slabs) * 64 + lane;
        const uint32_t begin = piece * s.length, end = min(begin + s.length, s.n);
        const int at = chunk_of<VEC>(min(q, nq - 1), nq, g.channels);
        const unsigned lane_byte = at * sizeof(T);       // channels of 2^24 at most
        // 64 positions: a lane's own, and before which of them another cell begins
        struct Look {
            uint32_t key, run;
            int64_t offset;
            uint64_t border;
        };
        auto look = [&](uint32_t first) {
            const uint32_t i = min(first + lane, end - 1);
            Look l;
            const Cell own = cell_at(s, i), before = cell_at(s, max(i, 1u) - 1);
            l.key = own.key;
            l.run = own.run;
            l.offset = g.walk.at(s.order[i]);
            l.border = __ballot(first + lane < end && i > begin && !(own == before));
            return l;
        };
        Look ahead = look(begin), here = ahead;
        Cell now = {static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(ahead.key)), static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(ahead.run))};
        if (now.key >= s.vocabulary) continue;           // nothing but positions without a row from here on
        bool begun = begin == 0 || !(cell_at(s, begin - 1) == now);
        float acc[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
        auto leave = [&](bool ends) {
            if (now.key >= s.vocabulary) return;
            const bool whole = begun && ends;
            float *to = whole ? g.dtable + (int64_t(now.run) * s.vocabulary + now.key) * g.channels : g.parts + (2 * int64_t(piece) + begun) * g.channels;
            const float by = whole ? g.scale : 1.f;
            float v[VEC];
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = acc[i] * by;
            if (q < nq) store_row<false, VEC>(to, at, v);
        };
        typename C::raw raw[kRowsAtOnce];
        auto fetch = [&](int u, int of) {                // the row of position `of` of the 64 ahead
            const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(ahead.offset), of), hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(ahead.offset >> 32), of);
            const char *row = static_cast<const char *>(g.dy) + static_cast<int64_t>(uint64_t(hi) << 32 | lo) * static_cast<int64_t>(sizeof(T));
            raw[u] = C::load_once(reinterpret_cast<const T *>(scalar(row) + lane_byte));
        };
#pragma unroll
        for (int u = 0; u < kRowsAtOnce; ++u) fetch(u, u);
        const int steps = (end - begin + kRowsAtOnce - 1) / kRowsAtOnce;
        for (int step = 0; step < steps; ++step) {
            const int first = step * kRowsAtOnce % 64;   // of the 64 here
            if (first == 0) here = ahead;
            if (first == 64 - kRowsAtOnce && step + 1 < steps) ahead = look(begin + (step + 1) * kRowsAtOnce);
#pragma unroll
            for (int u = 0; u < kRowsAtOnce; ++u) {
                const int e = first + u;
                if (begin + step * kRowsAtOnce + u < end) {
                    if (here.border >> e & 1) {
                        leave(true);
                        now = {static_cast<uint32_t>(__builtin_amdgcn_readlane(here.key, e)), static_cast<uint32_t>(__builtin_amdgcn_readlane(here.run, e))};
                        begun = true;
#pragma unroll
                        for (int i = 0; i < VEC; ++i) acc[i] = 0.f;
                    }
                    float v[VEC];
                    C::widen(raw[u], v);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) acc[i] += v[i];
                }
                if (step + 1 < steps) fetch(u, (e + kRowsAtOnce) % 64);
            }
        }
        leave(end == s.n || !(cell_at(s, end) == now));
    }
}

// The cell that begins in a piece and goes on behind it: its parts, added up in 64 bits.  A thread has two chunks of VEC channels; what threads a workgroup has
// beside those across a part's channels (512 at most) share the pieces out.
template <int VEC> __global__ void __launch_bounds__(kThreads) embedding_join_kernel(Gradient g, Sorted s, int nq, int across, int parts)
{
    constexpr int J = 2, U = 4;
    __shared__ double meet[J][VEC][kThreads];
    const int64_t all = int64_t(s.pieces) * parts;
    const int team = threadIdx.x / across, teams = kThreads / across, lane = threadIdx.x % across;
    for (int64_t i = blockIdx.x; i < all; i += gridDim.x) {
        const unsigned piece = static_cast<unsigned>(i / parts);
        const uint32_t begin = piece * s.length, end = min(begin + s.length, s.n);
        const Cell before = cell_at(s, max(begin, 1u) - 1), now = cell_at(s, end - 1), behind = cell_at(s, min(end, s.n - 1));
        if (end == s.n || now.key >= s.vocabulary || !(behind == now) || (begin > 0 && before == now)) continue;
        unsigned more = 0;                               // pieces behind this one that the cell reaches into
        for (;;) {
            const unsigned p = piece + 1 + more + threadIdx.x;
            const int count = __syncthreads_count(p < s.pieces && cell_at(s, std::min(p, s.pieces - 1) * s.length) == now);
            more += count;
            if (count < kThreads) break;
        }
        for (int q0 = static_cast<int>(i % parts) * J * across; q0 < nq; q0 += parts * J * across) {
            double sum[J][VEC] = {};
            int at[J];
#pragma unroll
            for (int j = 0; j < J; ++j) at[j] = chunk_of<VEC>(min(q0 + j * across + lane, nq - 1), nq, g.channels);
            for (unsigned p = team; p <= more; p += U * teams) {
                typename Chunk<false, VEC>::raw raw[U][J];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const unsigned pu = min(p + u * teams, more);
                    const float *row = g.parts + (2 * int64_t(piece + pu) + (pu == 0)) * g.channels;
#pragma unroll
                    for (int j = 0; j < J; ++j) raw[u][j] = Chunk<false, VEC>::load(row + at[j]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (p + u * teams > more) break;
#pragma unroll
                    for (int j = 0; j < J; ++j) {
                        float v[VEC];
                        Chunk<false, VEC>::widen(raw[u][j], v);
#pragma unroll
                        for (int c = 0; c < VEC; ++c) sum[j][c] += v[c];
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < J; ++j) {
#pragma unroll
                for (int c = 0; c < VEC; ++c) meet[j][c][threadIdx.x] = sum[j][c];
            }
            __syncthreads();
            for (int half = teams / 2; half > 0; half /= 2) {
                if (team < half) {
#pragma unroll
                    for (int j = 0; j < J; ++j) {
#pragma unroll
                        for (int c = 0; c < VEC; ++c) meet[j][c][threadIdx.x] += meet[j][c][threadIdx.x + half * across];
                    }
                }
                __syncthreads();
            }
            if (team == 0) {
#pragma unroll
                for (int j = 0; j < J; ++j) {
                    float v[VEC];
#pragma unroll
                    for (int c = 0; c < VEC; ++c) v[c] = static_cast<float>(meet[j][c][lane]) * g.scale;
                    if (q0 + j * across + lane < nq) store_row<false, VEC>(g.dtable, (int64_t(now.run) * s.vocabulary + now.key) * g.channels + at[j], v);
                }
            }
            __syncthreads();
        }
    }
}

// ---- what a gradient needs -------------------------------------------------------------------------------------------------------
struct GradPlan {
    int passes, digit_bits;      // of the sort; of a digit of it
    int vec, nq, team;           // channels of a chunk, chunks of a row, lanes of a piece
    unsigned slabs;
    size_t keys[2], order[2], run, counts, parts, met, bytes;        // offsets
};
// Workgroups of the sort: one where it holds all positions, else so many that a tile of each is as small as their number allows.
unsigned blocks_of(uint32_t n) { return n <= kMostTile ? 1 : static_cast<unsigned>(std::min<int64_t>((int64_t(n) + kSortThreads - 1) / kSortThreads, kMostBlocks)); }
// Pieces of 16 to 256 positions that fill the chip a whole number of times, once if they can: 983 040 rows of 1 KB in pieces of 128, which left 7 % of the
// wavefronts for a second time, took 287 us.
int piece_length(uint32_t n, int team, unsigned slabs)
{
    constexpr int64_t kWavefronts = 256 * 28;            // compute units, and what their registers take at once
    const int64_t work = (int64_t(n) * slabs * team + 63) / 64, times = std::max<int64_t>(1, (work + 256 * kWavefronts - 1) / (256 * kWavefronts));
    const int64_t length = (work + times * kWavefronts - 1) / (times * kWavefronts);
    return static_cast<int>(std::min<int64_t>(256, std::max<int64_t>(team < 64 ? 64 : 16, (length + 7) / 8 * 8)));
}

GradPlan plan_gradient(const LayerShape &shape, int vocabulary, int runs, uint32_t n)
{
    GradPlan p = {};
    int bits = 1;                                        // that the numbers 0 to `vocabulary` take
    while (uint64_t(vocabulary) >> bits) ++bits;
    p.passes = (bits + 8) / 9;
    p.digit_bits = (bits + p.passes - 1) / p.passes;
    p.vec = shape.bf16 ? 8 : 4;
    if (shape.channels < p.vec) p.vec = 1;
    p.nq = (shape.channels + p.vec - 1) / p.vec;
    for (p.team = 1; p.team < 64 && p.team < p.nq;) p.team *= 2;
    p.slabs = (p.nq + p.team - 1) / p.team;
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
    p.met = take(size_t(std::min(runs, BatchRuns::kRuns)) * vocabulary);
    p.bytes = at;
    return p;
}
template <bool BF16, int VEC> void launch_sums(const Gradient &g, const Sorted &s, const GradPlan &p, const Zeros &z, hipStream_t stream)
{
    auto go = [&](auto kernel, int team) {
        const uint64_t teams = uint64_t(s.pieces) * p.slabs, per_block = kThreads / team;
        const unsigned workgroups = static_cast<unsigned>(std::min<uint64_t>((teams + per_block - 1) / per_block, 1 << 20));
        kernel<<<workgroups + static_cast<unsigned>(z.workgroups), kThreads, 0, stream>>>(g, s, p.nq, p.slabs, workgroups, z);
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
        else go(embedding_wide_sums_kernel<BF16, VEC>, 64);
    }
}

Zeros plan_zeros(const EmbeddingGradArgs &a, float *dtable, int runs, const uint8_t *met, int64_t most_workgroups)
{
    Zeros z = {dtable, a.shape.channels, a.vocabulary, runs, 64, 1, met, 0};
    while (z.neighbours > 1 && int64_t(z.neighbours) * z.channels > 16384) z.neighbours /= 2;          // at most 64 KB of a workgroup
    z.parts = std::max(1, std::min(1024, z.channels / 16384));
    const int64_t groups = (int64_t(a.vocabulary) + z.neighbours - 1) / z.neighbours * runs;
    z.workgroups = std::min<int64_t>(groups, std::max<int64_t>(1, most_workgroups / z.parts)) * z.parts;
    return z;
}
constexpr int64_t kFewZeros = 511;
__global__ void __launch_bounds__(kThreads) embedding_zeros_kernel(Zeros z) { clear_rows(z, blockIdx.x); }

}  // namespace

size_t embedding_backward_bytes(const LayerShape &shape, int vocabulary, const int64_t *bounds, int runs)
{
    size_t most = 0;                                     // pieces are shorter where there are fewer positions: every batch has to fit
    for (int r = 0; r < runs; r += BatchRuns::kRuns) {
        const int64_t points = bounds[std::min(runs, r + BatchRuns::kRuns)] - bounds[r];
        if (points > 0) most = std::max(most, plan_gradient(shape, vocabulary, runs, static_cast<uint32_t>(points * shape.positions)).bytes);
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
            const Zeros z = plan_zeros(a, dtable, runs.runs, nullptr, 1 << 20);
            embedding_zeros_kernel<<<static_cast<unsigned>(z.workgroups), kThreads, 0, stream>>>(z);
            continue;
        }
        const GradPlan p = plan_gradient(shape, a.vocabulary, a.runs, n);
        char *ws = static_cast<char *>(workspace);
        auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(ws + at); };
        uint8_t *met = reinterpret_cast<uint8_t *>(ws + p.met);
        const unsigned blocks = blocks_of(n);
        const int64_t own = (int64_t(n) + blocks - 1) / blocks;          // positions of a workgroup
        const int steps = static_cast<int>(std::min<int64_t>(kKeysOfLane, (own + kSortThreads - 1) / kSortThreads));
        const int tiles = static_cast<int>((own + steps * kSortThreads - 1) / (steps * kSortThreads));
        int end = 0;                                     // of the two buffers, the one that holds the sorted positions
        for (int pass = 0; pass < (blocks == 1 ? 1 : p.passes); ++pass) {
            const int to = pass % 2, from = 1 - to;
            const bool last = blocks == 1 || pass == p.passes - 1;
            const SortPass s = {pass == 0 ? static_cast<const int64_t *>(a.tokens.p) + first * a.tokens.point_stride : nullptr, Walk(a.tokens, shape.positions),
                                static_cast<uint32_t>(a.vocabulary), words(p.keys[from]), words(p.order[from]), words(p.keys[to]), words(p.order[to]),
                                last && a.runs > 1 ? reinterpret_cast<uint8_t *>(ws + p.run) : nullptr, words(p.counts), n, tiles, steps, p.digit_bits, p.digit_bits * pass, met,
                                int64_t(runs.runs) * a.vocabulary};
            if (blocks == 1) {
                const Zeros z = plan_zeros(a, dtable, runs.runs, nullptr, kFewZeros);        // these stay
                sort_few_kernel<<<1 + static_cast<unsigned>(z.workgroups), kSortThreads, 0, stream>>>(s, runs, p.passes, z);
            } else {
                sort_count_kernel<<<blocks, kSortThreads, 0, stream>>>(s);
                sort_place_kernel<<<blocks, kSortThreads, 0, stream>>>(s, runs);
            }
            end = to;
        }
        const int length = piece_length(n, p.team, p.slabs);
        const Sorted s = {words(p.keys[end]), words(p.order[end]), a.runs > 1 ? reinterpret_cast<const uint8_t *>(ws + p.run) : nullptr, n,
                          static_cast<uint32_t>(a.vocabulary), length, static_cast<unsigned>((uint64_t(n) + length - 1) / length)};
        const size_t e = shape.bf16 ? 2 : 4;
        const Gradient g = {static_cast<const char *>(a.dy.p) + first * a.dy.point_stride * static_cast<int64_t>(e), Walk(a.dy, shape.positions), shape.channels, a.scale,
                            dtable, reinterpret_cast<float *>(ws + p.parts)};
        Zeros z = {};
        if (blocks > 1) z = plan_zeros(a, dtable, runs.runs, met, 1 << 20);
        if (p.vec == 1) shape.bf16 ? launch_sums<true, 1>(g, s, p, z, stream) : launch_sums<false, 1>(g, s, p, z, stream);
        else if (shape.bf16) launch_sums<true, 8>(g, s, p, z, stream);
        else launch_sums<false, 4>(g, s, p, z, stream);
        if (s.pieces > 1) {
            const int vec = shape.channels < 4 ? 1 : 4, nq = (shape.channels + vec - 1) / vec;
            int across = 2;
            while (across < 64 && 2 * across < nq) across *= 2;
            const int parts = std::min((nq + 2 * across - 1) / (2 * across), 64);
            const unsigned groups = static_cast<unsigned>(std::min<int64_t>(int64_t(s.pieces) * parts, 1 << 22));
            (vec == 1 ? embedding_join_kernel<1> : embedding_join_kernel<4>)<<<groups, kThreads, 0, stream>>>(g, s, nq, across, parts);
        }
    }
    return hipGetLastError();
}

}  // namespace cr

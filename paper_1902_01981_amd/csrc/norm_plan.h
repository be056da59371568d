// Which kernels a call of the group norm takes, and how they cut its points: host code, without the device's.
#pragma once
#include <algorithm>

#include "layers.h"

namespace cr {

constexpr int kUnits = 256;                              // compute units
inline int ceil_div(int64_t a, int64_t b) { return static_cast<int>((a + b - 1) / b); }

// ---- points of one position (norm_rows.hip) ---------------------------------------------------------------------------------------------------
struct RowsPlan {
    int lanes, chunks;           // lanes of a group, chunks of a lane; no lanes: not these kernels
    int wide, down;              // groups side by side in a workgroup, points
};
constexpr int points_at_once(int chunks) { return chunks == 1 ? 4 : chunks == 2 ? 2 : 1; }
// points of a workgroup: enough workgroups to fill the chip several times, and a few steps for each
inline int64_t points_of_workgroup(const LayerShape &s, int groups, const RowsPlan &p, int workgroups_per_unit, int steps)
{
    const int64_t tiles = ceil_div(groups, p.wide), step = p.down * points_at_once(p.chunks);
    int64_t length = (s.points * tiles + kUnits * workgroups_per_unit - 1) / (kUnits * workgroups_per_unit);
    length = (length + step - 1) / step * step;
    return std::max<int64_t>({1, length, std::min(step * steps, (s.points + step - 1) / step * step)});
}
// The gradient of more channels than 32 a lane is more than the registers hold beside the sums for gamma and beta.
inline RowsPlan rows_plan(const LayerShape &s, int groups, bool backward)
{
    const int vec = s.bf16 ? 8 : 4, cg = s.channels / groups, chunks = ceil_div(cg, vec);
    RowsPlan p = {};
    if (s.positions != 1 || cg < vec || chunks > 64 * (backward && s.bf16 ? 4 : 8)) return p;
    p.lanes = 1;
    while (p.lanes < 64 && p.lanes < chunks) p.lanes *= 2;
    p.chunks = ceil_div(chunks, p.lanes);
    const int teams = 256 / p.lanes;
    p.wide = ceil_div(groups, ceil_div(groups, teams));
    p.down = teams / p.wide;
    return p;
}
// points of a piece of a run
inline int64_t rows_piece(const LayerShape &s, int groups, const RowsPlan &p) { return points_of_workgroup(s, groups, p, 4, 4); }

// ---- tiles and pieces (norm_forward.hip, norm_backward.hip) -----------------------------------------------------------------------------------
// How a launch cuts points into tiles.  Columns: `tiles` of them, each some whole groups, or (slices > 1) a part of one group.  Rows: `down` positions side
// by side, K below each other in a thread; `side` points side by side.
struct Tiling {
    int tiles, slices, unit, across, down, side, threads, k;             // slices begin at multiples of `unit` channels of the group
    int pieces;                  // of a point's positions, down * k each
    int deep;                    // points of a thread, or 0: it has one point's positions (k of them)
    int fold;                    // the seats of a column in a wavefront are `across` lanes apart, and the wavefront has one point's: they are added up before LDS
};

constexpr int kMostGroups = 4096;                        // sums of a workgroup: with what they are made from they fit 64 KB of LDS
constexpr int kPartThreads = 256;                        // of norm_part_* and norm_join_*
constexpr int kForwardThreads = 1024, kBackwardThreads = 256;           // of norm_tile_*, at most

inline int vec_of(const LayerShape &s) { return s.channels < (s.bf16 ? 8 : 4) ? 1 : s.bf16 ? 8 : 4; }
// of a load of vec channels, the neighbours that always lie in one group: the largest power of two that divides both
inline int unit_of(int cg, int vec)
{
    while (cg % vec != 0) vec /= 2;
    return vec;
}
inline int across_for(const LayerShape &s, int groups, int tiles) { return ceil_div(int64_t(ceil_div(groups, tiles)) * (s.channels / groups), vec_of(s)); }
// Whether the seats of a column can be added up inside a wavefront; rounds `down` for it where there is room.
inline void fold_columns(Tiling *t)
{
    t->fold = 0;
    if (t->across > 32 || (t->across & (t->across - 1)) != 0) return;
    const int step = 64 / t->across, down = (t->down + step - 1) / step * step;
    if (t->side > 1 ? t->down % step != 0 : down * t->across > t->threads) return;
    t->down = t->side > 1 ? t->down : down;
    t->fold = 1;
}

// Tiles in registers: at most so many threads and chunks of each; k == 0: the point is too large, and is cut into pieces.  Small workgroups, of which
// several share a compute unit and one loads while others add up; so tiles get more chunks of a thread, then narrower (down to a cache line of columns), and only
// then more threads.  320 x 1 024 x 16 bf16 forward, 256 threads with 8 chunks each 11.8 us, 1 024 with two 17.0; 1 000 x 196 x 256 47 with 8 chunks, 59 with 4;
// its gradient 102 with 8 chunks and 256 threads, 145 with 4 and 512, 112 in pieces.  Columns of half a line rather than pieces, a point's tiles as far apart in
// the grid as there are points: 500 x 400 x 96 fp32 gradient 110 us against 77 in pieces, 64 x 1 800 x 160 forward 74 against 42.
inline Tiling tile(const LayerShape &s, int groups, bool backward)
{
    // (the gradient of one position each leaves room for a group of 512 chunks)
    const int most_threads = !backward ? kForwardThreads : s.positions == 1 ? 2 * kBackwardThreads : kBackwardThreads, most_chunks = 8, vec = vec_of(s);
    const int cg = s.channels / groups, line = std::max(1, 128 / (cg * (s.bf16 ? 2 : 4)));
    Tiling t = {};
    t.slices = t.unit = t.side = t.pieces = 1;
    const int most_tiles = std::max(1, std::min(groups / line, 65535));      // of a grid's second dimension
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
        t.tiles = tiles;
        t.across = across_for(s, groups, tiles);
        t.k = 1;
        while (int64_t(t.threads / t.across) * t.k < s.positions) t.k *= 2;
        // Where there are points enough, more chunks of a thread and more points side by side: a thread adds up its own rows of a group before it meets others,
        // and a step of a workgroup is that much more.  (Not where over two fifths of what a thread could have would be empty.)  Forward and gradient, us,
        // with the fewest chunks and so: 20 000 x 4 x 320 bf16 54 and 121, 29 and 72; 45 575 x 17 x 90 246 and 336, 77 and 196; 4 096 x 16 x 33 fp32 12 and
        // 32, 9 and 19.  Sums per channel of eight channels: the gradient's registers are full at four chunks (45 575 x 17 x 90 with eight: 247).
        const int values = vec / unit_of(cg, vec), side = t.threads / (t.across * ceil_div(s.positions, t.k)), fewest = t.k;
        for (int k = 2 * fewest; k <= (backward && values == 8 ? 4 : most_chunks) && k / 2 < s.positions; k *= 2) {
            const int more_side = t.threads / (t.across * ceil_div(s.positions, k));
            if (5 * more_side * fewest >= 3 * side * k && s.points * tiles >= int64_t(kUnits) * more_side) t.k = k;
        }
        t.down = ceil_div(s.positions, t.k);             // as even as can be
        t.side = std::max(1, std::min(t.threads / (t.across * t.down), kMostGroups / ceil_div(groups, tiles)));
        t.side = static_cast<int>(std::min<int64_t>(t.side, std::max<int64_t>(1, s.points)));
        fold_columns(&t);
        // one position each: several points each, so long as there are enough for all workgroups and LDS for their sums
        if (t.k == 1 && t.threads <= 512) {
            auto room = [&](int deep) { return (size_t(deep) * t.threads * values + size_t(2) * deep * t.side * ceil_div(groups, tiles)) * (backward ? 2 : 1) * sizeof(float); };
            // (the gradient of four, with a sum per channel, is more than the registers hold)
            for (int deep = backward && values > 1 ? 2 : 4; deep > 1 && !t.deep; deep /= 2)
                if (room(deep) <= size_t(48) << 10 && s.points * tiles >= int64_t(4) * kUnits * t.side * deep) t.deep = deep;
        }
        return t;
    }
    return t;
}
inline Tiling cut(const LayerShape &s, int groups)
{
    const int vec = vec_of(s), cg = s.channels / groups;
    Tiling t = {};
    t.side = t.slices = 1;
    t.threads = kPartThreads;
    t.unit = unit_of(cg, vec);
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
inline int most_groups(const Tiling &t, int groups) { return t.slices > 1 ? 1 : ceil_div(groups, t.tiles); }

// (A piece is of one point: points of few positions whose groups are wide, as 16 384 of one position and 8 192 bf16 channels in one group, leave a row of sums
// each in the gradient, 1.1 GB of them beside 268 MB of activations, and take 1 075 us where the reads and writes that have to be are 161.)
// Points of a pair of launches: as many as a grid takes.  (Fewer, so that what is read twice comes from the last-level cache, cost more at the launches' ends
// than they gain: 64 x 4 096 x 512 bf16, points of 96 MB at a time / of 192 / all: forward 213 / 196 / 176 us, backward 365 / 320 / 279.)
inline int64_t batch_points(const LayerShape &s, const Tiling &t) { return std::max<int64_t>(1, std::min<int64_t>(s.points, (int64_t(1) << 22) / t.pieces)); }

// points of a piece: a workgroup's sums of the parameters' gradients are over so many that they are little beside what it reads
inline int64_t points_of_piece(const LayerShape &s, const Tiling &t)
{
    const int64_t wanted = std::max<int64_t>(1, kUnits * 8 / t.tiles);
    int64_t length = std::max<int64_t>((s.points + wanted - 1) / wanted, std::min<int64_t>(32 / std::min(s.positions, 32), (s.points + kUnits - 1) / kUnits));
    const int at_once = t.side * std::max(t.deep, 1);
    return std::max<int64_t>((length + at_once - 1) / at_once * at_once, 1);
}

struct BackwardPlan {
    RowsPlan rows;
    bool cut;                    // norm_part and norm_join
    Tiling t;
    int64_t units_per_point, length;                     // of the pieces
};
inline BackwardPlan plan_backward(const LayerShape &s, int groups)
{
    BackwardPlan p = {};
    p.units_per_point = 1;
    p.rows = rows_plan(s, groups, true);
    if (p.rows.lanes) {
        p.length = rows_piece(s, groups, p.rows);
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

}  // namespace cr

// Where a row is among a call's points: plain arithmetic, for host and device alike.
#pragma once
#include <cstdint>

namespace cr {

struct RowPlace {
    int64_t point;
    int position;                // 0 .. positions - 1
};
// The place points_on points and positions_on (fewer than `positions`) positions further on.  Positions may be up to 2^31 - 1, so that the sum of two
// numbers of them may not fit an int: compared with what is left of the point, and only then added or subtracted.
constexpr RowPlace row_place_on(RowPlace at, int points_on, int positions_on, int positions)
{
    const int last = positions - positions_on;           // positions from here on step into the next point
    const bool over = at.position >= last;
    return {at.point + points_on + over, over ? at.position - last : at.position + positions_on};
}

}  // namespace cr

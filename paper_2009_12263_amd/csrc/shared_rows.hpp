// Whether two arrays of rows have bytes in common.  Plain integer arithmetic without HIP: a CPU test compiles this header.
#pragma once
#include <stdint.h>

namespace fg {

// `rows` rows of `bytes` each, `step` apart (step >= bytes; not looked at for a single row).
struct RowSpan { uintptr_t at; int64_t rows, step, bytes; };

inline bool share_bytes(const RowSpan &x, const RowSpan &y) {
    typedef __int128 wide;
    if (x.rows <= 0 || y.rows <= 0 || x.bytes <= 0 || y.bytes <= 0) return false;
    const wide x_end = (wide)x.at + (wide)(x.rows - 1) * x.step + x.bytes, y_end = (wide)y.at + (wide)(y.rows - 1) * y.step + y.bytes;
    if (x_end <= (wide)y.at || y_end <= (wide)x.at) return false;
    // Between each other lie, for one, columns of the same matrix.  Row i of the one with fewer rows: of the other's that begin before its end the last one reaches furthest.
    const RowSpan &a = x.rows <= y.rows ? x : y, &b = x.rows <= y.rows ? y : x;
    auto below = [](wide v, wide by) { return v >= 0 ? v / by : -((-v + by - 1) / by); };
    auto row_meets = [&](wide i) {
        const wide begin = (wide)a.at + i * a.step;
        wide j = b.rows == 1 ? 0 : below(begin + a.bytes - 1 - (wide)b.at, b.step);
        if (j >= b.rows) j = b.rows - 1;
        const wide there = (wide)b.at + j * b.step;
        return j >= 0 && there < begin + a.bytes && there + b.bytes > begin;
    };
    if (a.rows == 1) return row_meets(0);
    if (a.step == b.step) {
        // they meet where row k + j of a does row j of b: d - a.bytes < k step < d + b.bytes, with d from a's first byte to b's
        const wide d = (wide)b.at - (wide)a.at, least = below(d - a.bytes, a.step) + 1, most = below(d + b.bytes - 1, a.step);
        return (least > -(b.rows - 1) ? least : (wide)(1 - b.rows)) <= (most < a.rows - 1 ? most : (wide)(a.rows - 1));
    }
    // the rows of a that lie where b does
    wide i = below((wide)b.at - (wide)a.at - a.bytes, a.step) + 1, last = below((wide)(x_end < y_end ? x_end : y_end) - 1 - (wide)a.at, a.step);
    i = i > 0 ? i : 0;
    last = last < a.rows - 1 ? last : (wide)(a.rows - 1);
    for (; i <= last; ++i)
        if (row_meets(i)) return true;
    return false;
}

}  // namespace fg

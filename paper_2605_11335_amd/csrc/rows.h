// Host checks of operands: where the rows of one [n, heads, width] lie, for entry points that write one while others are read, and what fits a launch.
#pragma once
#include <stdint.h>

constexpr int64_t MOST_WGS = (1 << 24) - 1;          // of 256 lanes in one launch

struct Rows {
    const void* p;
    int64_t n, row, heads, head;           // strides in elements
    int64_t width;
    int es;                                // bytes of an element
    const char* lo() const { return (const char*)p; }
    const char* hi() const { return lo() + ((n - 1) * row + (heads - 1) * head + width) * es; }
    // every row has a place of its own: heads inside rows, or rows inside heads
    bool apart() const {
        const bool heads_in = heads == 1 || head >= width, rows_in = n == 1 || row >= width;
        const bool rows_out = n == 1 || row >= (heads - 1) * head + width, heads_out = heads == 1 || head >= (n - 1) * row + width;
        return (heads_in && rows_out) || (rows_in && heads_out);
    }
};
// Whether two operands may share memory.  Columns of one row, as q and k of one projection, are told apart.
inline bool rows_meet(const Rows& a, const Rows& b) {
    if (a.hi() <= b.lo() || b.hi() <= a.lo()) return false;
    if (a.es != b.es || a.row != b.row) return true;
    const int64_t off = (b.lo() - a.lo()) / a.es, wa = (a.heads - 1) * a.head + a.width, wb = (b.heads - 1) * b.head + b.width;
    return !(off >= 0 ? off >= wa && off + wb <= a.row : -off >= wb && -off + wa <= a.row);
}

// Whether the heads of strided matrices lie apart in memory: two writers of one byte would leave what the later one wrote.  Host code only.
#pragma once
#include <stdint.h>

namespace tbe {

// [rows][heads] runs of `len` bytes; rows `row`, heads `head` bytes apart (both >= 0)
struct HeadRuns {
    const void* at;
    int64_t row, head, rows, heads, len;
};

// Whether some r, |r| <= rows - 1, has |t + r row| < len: one of the two next to -t / row, or the nearest there is.
inline bool some_row_meets(const int64_t t, const int64_t row, const int64_t rows, const int64_t len) {
    const auto meets = [&](int64_t r) {
        r = r < 1 - rows ? 1 - rows : (r > rows - 1 ? rows - 1 : r);
        const int64_t d = t + r * row;
        return d < len && d > -len;
    };
    if (row == 0) return meets(0);
    const int64_t r = -t / row;   // (towards zero)
    return meets(r) || meets(t > 0 ? r - 1 : r + 1);
}

// No two runs of m share a byte.  Exact: rows inside heads and heads inside rows are the common cases, others are tried head by head.
inline bool runs_apart(const HeadRuns& m) {
    if (m.rows > 1 && m.row < m.len) return false;
    if (m.heads > 1 && m.head < m.len) return false;
    if (m.rows <= 1 || m.heads <= 1) return true;
    if (m.row >= (m.heads - 1) * m.head + m.len || (__int128)m.head >= (__int128)(m.rows - 1) * m.row + m.len) return true;
    for (int64_t h = 1; h < m.heads; ++h)
        if (some_row_meets(h * m.head, m.row, m.rows, m.len)) return false;
    return true;
}

// A run of a and one of b, of equal length, share a byte.  Exact where they have equal strides, as column blocks of one matrix and shifted views of one
// matrix have; matrices of unlike strides that lie between each other are taken to be apart.
inline bool runs_meet(const HeadRuns& a, const HeadRuns& b) {
    if (a.rows < 1 || b.rows < 1 || a.heads < 1 || b.heads < 1) return false;
    const auto extent = [](const HeadRuns& m) { return (__int128)(m.rows - 1) * m.row + (m.heads - 1) * m.head + m.len; };
    const __int128 from_a = (__int128)reinterpret_cast<uintptr_t>(a.at), from_b = (__int128)reinterpret_cast<uintptr_t>(b.at);
    if (from_a + extent(a) <= from_b || from_b + extent(b) <= from_a) return false;
    const int64_t rows = a.rows > b.rows ? a.rows : b.rows, row = a.rows > 1 ? a.row : b.row, head = a.heads > 1 ? a.head : b.head;
    if ((a.rows > 1 && b.rows > 1 && a.row != b.row) || (a.heads > 1 && b.heads > 1 && a.head != b.head)) return false;
    for (int64_t h = 1 - a.heads; h < b.heads; ++h)
        if (some_row_meets((int64_t)(from_b - from_a) + h * head, row, rows, a.len)) return true;
    return false;
}

}  // namespace tbe

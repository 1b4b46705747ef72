// Whether two matrices of strided rows share memory.
#pragma once

#include <cstdint>

namespace {

// The memory of a matrix: rows of `width` bytes, `pitch` apart.
struct Rows {
    uintptr_t first;
    int64_t rows, width, pitch;
    Rows(const void* p, int64_t rows_, int64_t columns, int64_t ld, int64_t bytes)
        : first(reinterpret_cast<uintptr_t>(p)), rows(columns > 0 ? rows_ : 0), width(columns * bytes), pitch(ld * bytes) {}
    uintptr_t at(int64_t row) const { return first + static_cast<uintptr_t>(row * pitch); }
    uintptr_t end() const { return at(rows - 1) + static_cast<uintptr_t>(width); }
};
// Whether two matrices share a byte.  Columns of one buffer beside each other do not.
inline bool overlap(Rows a, Rows b) {
    if (a.rows == 0 || b.rows == 0 || a.end() <= b.first || b.end() <= a.first) return false;
    if (a.rows == 1) a.pitch = b.pitch;  // a single row's says nothing
    if (b.rows == 1) b.pitch = a.pitch;
    const int64_t p = a.pitch, d = static_cast<int64_t>(b.first - a.first);
    if (p == b.pitch && p > 0) {
        // row j of b lies at d + (j - i) p from row i of a: the least j - i whose row ends behind that row's start
        const int64_t from = -b.width - d;
        int64_t k = from / p - (from % p < 0 ? 1 : 0) + 1;
        if (k < 1 - a.rows) k = 1 - a.rows;
        return k < b.rows && d + k * p < a.width;
    }
    for (int64_t i = 0, j = 0; i < a.rows && j < b.rows;) {
        if (a.at(i) + static_cast<uintptr_t>(a.width) <= b.at(j))
            ++i;
        else if (b.at(j) + static_cast<uintptr_t>(b.width) <= a.at(i))
            ++j;
        else
            return true;
    }
    return false;
}

}  // namespace

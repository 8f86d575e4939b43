// Whether two operands of a call share memory: plain arithmetic on their rows.
#pragma once

#include <stdint.h>

namespace p4q {

// `rows` rows of `width` bytes that begin `stride` >= width bytes apart
struct Rows {
    uint64_t at;                                 // 0: no operand
    uint64_t rows, stride, width;
};

inline Rows rows_at(const void *p, int64_t rows, int64_t stride, int64_t width) {
    const Rows r = {(uint64_t)reinterpret_cast<uintptr_t>(p), (uint64_t)rows, (uint64_t)stride, (uint64_t)width};
    // rows without gaps are one
    if (rows > 1 && stride != width) return r;
    return {r.at, 1, r.rows * r.width, r.rows * r.width};
}

inline uint64_t rows_end(const Rows &r) { return r.at + (r.rows - 1) * r.stride + r.width; }

// Columns of one wider buffer do not share memory.  Exact unless both have gaps of
// different strides: then the first row of the later one decides.
inline bool share_memory(const Rows &a, const Rows &b) {
    if (!a.at || !b.at || a.at >= rows_end(b) || b.at >= rows_end(a)) return false;
    if (a.at > b.at) return share_memory(b, a);
    if (a.rows == 1) return true;
    // b begins in row r of a, or in the gap behind it
    const uint64_t r = (b.at - a.at) / a.stride, column = (b.at - a.at) % a.stride;
    return column < a.width || (r + 1 < a.rows && column + b.width > a.stride);
}

}  // namespace p4q

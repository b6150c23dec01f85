// Whether two arguments of rows share memory.
#pragma once

#include <algorithm>
#include <cstdint>

namespace micro {

// `rows` runs of `width` bytes, `stride` bytes apart (at least width).
struct RowSpan {
    const void* at;
    int64_t rows, stride, width;
    int64_t bytes() const { return rows > 0 && width > 0 ? (rows - 1) * stride + width : 0; }
};

// Exact for equal strides, and where one of the two is one run (so the halves
// of a buffer's columns share nothing); rows of different strides share memory
// where their whole ranges meet.
inline bool rows_share_bytes(RowSpan a, RowSpan b) {
    if (a.bytes() == 0 || b.bytes() == 0) return false;
    for (RowSpan* s : {&a, &b})
        if (s->rows == 1 || s->stride == s->width) *s = {s->at, 1, s->bytes(), s->bytes()};
    const int64_t apart = static_cast<int64_t>(reinterpret_cast<uintptr_t>(b.at) - reinterpret_cast<uintptr_t>(a.at));
    if (apart >= a.bytes() || -apart >= b.bytes()) return false;
    if ((a.rows == 1 && b.rows == 1) || (a.rows > 1 && b.rows > 1 && a.stride != b.stride)) return true;
    // Row i of a and j of b meet where apart - a.width < (i - j) stride < apart + b.width.
    const int64_t stride = a.rows > 1 ? a.stride : b.stride;
    const auto floor_div = [stride](int64_t x) { return x / stride - (x % stride < 0); };
    const int64_t lo = floor_div(apart - a.width) + 1, hi = -floor_div(-(apart + b.width)) - 1;
    return std::max(lo, 1 - b.rows) <= std::min(hi, a.rows - 1);
}

}  // namespace micro

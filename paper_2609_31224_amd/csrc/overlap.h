// Whether rows in memory touch each other (host only): an output over an input that other workgroups
// of the same call still read would be a race.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace a2t {

// `rows` rows of `width` bytes, `stride` bytes apart (width <= stride; rows * stride within 2^62).
struct Rows {
    const void* p;
    int64_t rows, width, stride;
    int64_t first() const { return (int64_t)(uintptr_t)p; }
    int64_t end() const { return first() + (rows - 1) * stride + width; }
};

// Exact: rows that lie between each other's (parts of one projection's output) do not overlap.
inline bool overlap(const Rows& a, const Rows& b) {
    if (!a.p || !b.p || a.rows < 1 || b.rows < 1 || a.width < 1 || b.width < 1) return false;
    if (a.end() <= b.first() || b.end() <= a.first()) return false;
    auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    // the rows of `of` that a run of bytes at `at` touches: those that start after at - of.width, before at + width
    auto touches = [&](const Rows& of, int64_t at, int64_t width, int64_t lo, int64_t hi) {
        const int64_t d = at - of.first();
        return std::max(lo, floor_div(d - of.width, of.stride) + 1) <= std::min(hi, floor_div(d + width - 1, of.stride));
    };
    // of equal strides the rows' distance decides alone: row i of one lies against row i + k of the other
    if (a.stride == b.stride) return touches(a, b.first(), b.width, 1 - b.rows, a.rows - 1);
    const Rows& few = a.rows < b.rows ? a : b;
    const Rows& many = a.rows < b.rows ? b : a;
    for (int64_t i = 0; i < few.rows; ++i)
        if (touches(many, few.first() + i * few.stride, few.width, 0, many.rows - 1)) return true;
    return false;
}

// n contiguous bytes.
inline Rows run_of(const void* p, int64_t n) { return {p, 1, n, n}; }

}  // namespace a2t

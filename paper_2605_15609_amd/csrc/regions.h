// Memory that the calls read and write, and whether two pieces of it overlap (host).
#pragma once
#include <stdint.h>

inline bool misaligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

// Memory of a call, in bytes: `units` times `rows` pieces of `width`
struct Region {
    uintptr_t first;
    int64_t units, unit_stride, rows, row_stride, width;
    int64_t unit_width() const { return (rows - 1) * row_stride + width; }
    int64_t span() const { return units < 1 || rows < 1 || width < 1 ? 0 : (units - 1) * unit_stride + unit_width(); }
};
inline Region dense(const void *p, int64_t bytes) { return {reinterpret_cast<uintptr_t>(p), 1, 0, 1, 0, p ? bytes : 0}; }

// [a, a + wa) and [b, b + wb), each repeated every p bytes, have no byte in common
inline bool apart_modulo(uintptr_t a, int64_t wa, uintptr_t b, int64_t wb, int64_t p) {
    if (p < 1 || wa > p || wb > p) return false;
    const int64_t d = b >= a ? (int64_t)((b - a) % (uintptr_t)p) : (p - (int64_t)((a - b) % (uintptr_t)p)) % p;
    return d >= wa && d + wb <= p;
}

// No byte in common: one lies behind the other, or they are columns of the same rows, or parts of the same units (what alternates in other ways
// is taken to overlap)
inline bool apart(const Region &a, const Region &b) {
    const int64_t na = a.span(), nb = b.span();
    if (na == 0 || nb == 0 || a.first + (uintptr_t)na <= b.first || b.first + (uintptr_t)nb <= a.first) return true;
    auto row_period = [](const Region &r) {   // 0: no period
        if (r.units == 1) return r.rows == 1 ? (int64_t)-1 : r.row_stride;
        if (r.rows == 1) return r.unit_stride;
        return r.row_stride > 0 && r.unit_stride % r.row_stride == 0 ? r.row_stride : 0;
    };
    auto same = [](int64_t x, int64_t y) { return x < 0 ? y : y < 0 || x == y ? x : 0; };   // (-1: a single piece, which fits any period)
    return apart_modulo(a.first, a.width, b.first, b.width, same(row_period(a), row_period(b))) ||
           apart_modulo(a.first, a.unit_width(), b.first, b.unit_width(), same(a.units > 1 ? a.unit_stride : -1, b.units > 1 ? b.unit_stride : -1));
}

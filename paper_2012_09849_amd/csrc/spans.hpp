// Whether two arrays of rows share bytes: host only, so that the C entries and a host test share it.
#pragma once
#include <stdint.h>

namespace hts {

// rows of `bytes` bytes, `ld` bytes apart (0 or more)
struct Span { int64_t p, ld, rows, bytes; };
inline Span span(const void *p, int64_t ld, int64_t rows, int64_t cols, int size) { return Span{(int64_t)(uintptr_t)p, ld * size, p ? rows : 0, cols * size}; }

inline bool meet(Span a, Span b)
{
    if (a.rows == 0 || b.rows == 0) return false;
    if (a.ld == 0) a.rows = 1;
    if (b.ld == 0) b.rows = 1;
    if (a.p + (a.rows - 1) * a.ld + a.bytes <= b.p || b.p + (b.rows - 1) * b.ld + b.bytes <= a.p) return false;
    // the distance of a single row says nothing
    if (a.rows == 1) a.ld = b.rows == 1 ? 1 : b.ld;
    if (b.rows == 1) b.ld = a.ld;
    if (a.ld == b.ld) {
        // some row of b, k = -(a.rows - 1) .. b.rows - 1 distances from where it would be beside a's, begins after 1 - b.bytes and before a.bytes
        const int64_t from = 1 - b.bytes - (b.p - a.p), up = from / a.ld + (from % a.ld > 0), k = up < 1 - a.rows ? 1 - a.rows : up;
        return k < b.rows && b.p - a.p + k * a.ld < a.bytes;
    }
    // distances of their own: row after row (their ends are in order, too)
    for (int64_t i = 0, j = 0; i < a.rows && j < b.rows;) {
        const int64_t s = a.p + i * a.ld, t = b.p + j * b.ld;
        if (s + a.bytes <= t) ++i;
        else if (t + b.bytes <= s) ++j;
        else return true;
    }
    return false;
}
// the same rows of the same array
inline bool same(const Span &a, const Span &b) { return a.p == b.p && (a.ld == b.ld || a.rows == 1) && a.rows == b.rows && a.bytes == b.bytes; }

}  // namespace hts

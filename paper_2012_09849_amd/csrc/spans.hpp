// Whether two arrays of rows, or of steps of sequences, share bytes: host only, so that the C entries and a host test share it.
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

// T x N rows of `bytes` bytes, `st` and `sn` bytes apart (0 or more: the same row again), from the first byte to behind the last one (or the last address; 0: none)
struct Area { int64_t p, end, st, sn, T, N, bytes; };
inline Area area(const void *p, int64_t st, int64_t sn, int64_t T, int64_t N, int64_t cols, int size)
{
    Area a{(int64_t)(uintptr_t)p, 0, st * size, sn * size, st ? T : 1, sn ? N : 1, cols * size};
    if (a.T == 1) a.st = 0;
    if (a.N == 1) a.sn = 0;
    const __int128 end = (__int128)a.p + (__int128)(a.T - 1) * a.st + (__int128)(a.N - 1) * a.sn + a.bytes;
    a.end = !p ? 0 : end < INT64_MAX ? (int64_t)end : INT64_MAX;
    return a;
}
inline Area area(const void *p, int64_t count, int size) { return area(p, 0, 0, 1, 1, count, size); }

inline __int128 floor_div(__int128 a, __int128 b) { return a / b - (a % b < 0); }
// some row of b, u times `large` and w times `small` from where it would be beside a's, begins after -b.bytes and before a.bytes
inline bool meet_shifted(__int128 apart, int64_t large, int64_t u_from, int64_t u_to, int64_t small, int64_t w_from, int64_t w_to, int64_t a_bytes, int64_t b_bytes)
{
    if (small == 0) w_from = w_to = 0;
    if (large == 0) u_from = u_to = 0;
    __int128 u = u_from, last = u_to;
    if (large) {
        const __int128 first = floor_div(-b_bytes - apart - (__int128)w_to * small, large) + 1, most = floor_div(a_bytes - apart - (__int128)w_from * small - 1, large);
        if (first > u) u = first;
        if (most < last) last = most;
    }
    for (; u <= last; ++u) {
        const __int128 x = apart + u * large;
        __int128 w = w_from;
        if (small) {
            const __int128 first = floor_div(-b_bytes - x, small) + 1;
            if (first > w) w = first;
        } else if (x <= -b_bytes) continue;
        if (w <= w_to && x + w * small < a_bytes) return true;
    }
    return false;
}
inline bool meet_within(Area a, Area b)
{
    const auto order = [](Area &x) {
        if (x.sn > x.st) { const Area y = x; x.st = y.sn; x.sn = y.st; x.T = y.N; x.N = y.T; }
    };
    order(a); order(b);
    if (a.st == b.st && a.sn == b.sn) return meet_shifted((__int128)b.p - a.p, a.st, 1 - a.T, b.T - 1, a.sn, 1 - a.N, b.N - 1, a.bytes, b.bytes);
    if (a.T * a.N > b.T * b.N) { const Area c = a; a = b; b = c; }
    for (int64_t i = 0; i < a.T; ++i)
        for (int64_t k = 0; k < a.N; ++k)
            if (meet_shifted((__int128)b.p - (a.p + i * a.st + k * a.sn), b.st, 0, b.T - 1, b.sn, 0, b.N - 1, a.bytes, b.bytes)) return true;
    return false;
}
// Whether two of them share bytes.  Arrays of the same distances (parts of one wider array) are told apart at once, others that lie within each other's reach row by row.
inline bool meet(const Area &a, const Area &b) { return a.end > b.p && b.end > a.p && a.end && b.end && meet_within(a, b); }

}  // namespace hts

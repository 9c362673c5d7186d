// How a matrix product's reduction is cut and where its slices' sums are in the workspace: host only, so that linear.hip and a host test share it.
#pragma once
#include "seq.hpp"

namespace hts {

// dw's reduction over the rows is cut where C has too few tiles for the compute units, into a slice for every 512 rows (8 k-tiles, 16 in binary32) or part of them
// at most, so that one has more than 256 of them: 8192 rows of 2048 x 512 and the slices' sums 28.9 + 3.6 us in four, 27.6 + 8.1 in eight; dw and db of 1024 rows through
// an activation 5 us less with two than with one.
inline int slices_of(int64_t rows, int64_t N, int64_t K)
{
    const int64_t tiles = ceil_div(N, 128) * ceil_div(K, 128), most = ceil_div(rows, 512);
    int64_t z = 256 / tiles;
    if (z > 16) z = 16;
    if (z > most) z = most;
    return (int)(z < 1 ? 1 : z);
}

// C = M x N over K, `parts` times, k-tiles of BK, in at most `slices`.  A slice leaves its sums of C, where they are wanted, and at `rows` A's own (db)
struct Slices { int count, klen; int64_t rows, stride; };             // stride: entries from slice to slice, a multiple of 4
inline Slices cut(int64_t M, int64_t N, int64_t K, int BK, int parts, int slices, bool products)
{
    Slices s;
    const int64_t total = ceil_div(K, BK) * parts;
    s.klen = (int)(ceil_div(total, slices) * BK);
    s.count = (int)ceil_div(total * BK, s.klen);
    s.rows = products ? M * N : 0;
    s.stride = round_up(s.rows + M, 4);
    return s;
}

// The backward call of M rows, N outputs and K inputs; an activation's gradient is `parts_of` arrays of M x N.  Bytes; stride: entries from part to part
struct LinearLayout { int64_t slope, stride, part, total; };
inline int parts_of(int size, int act) { return act != HTS_ACT_NONE && size == 2 ? 3 : 1; }
inline LinearLayout linear_layout(int size, int act, int64_t M, int64_t N, int64_t K)
{
    LinearLayout l;
    l.slope = 0;
    l.stride = act != HTS_ACT_NONE ? round_up(M * N, 128) : 0;
    l.part = l.stride * size * parts_of(size, act);
    const int z = slices_of(M, N, K);
    l.total = l.part + (z > 1 ? 4 * z * round_up(N * K + N, 4) : 0);
    return l;
}
// dw [N,K] and db [N] over the rows; without dw a few columns of any operand, whose products go nowhere
inline int weight_columns(int size, bool dw, int64_t N, int64_t K) { return (int)(dw ? K : N % (16 / size) == 0 ? 16 / size : 1); }
inline Slices weight_slices(int size, int act, int64_t M, int64_t N, int64_t K, bool dw)
{
    return cut(N, weight_columns(size, dw, N, K), M, 128 / size, parts_of(size, act), slices_of(M, N, K), dw);
}

}  // namespace hts

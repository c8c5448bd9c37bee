// Whether two row-strided matrices share memory, in plain C++ (no HIP), so that a CPU test can compare it with the elements.
#pragma once
#include <stdint.h>

namespace reqat {

// Matrices of 2-byte elements, rows x cols with leading dimension ld >= cols.  Exact for column slices of one buffer
// (equal ld; a single row has any); true without a closer look where strides differ and the spans meet.
inline bool rows_overlap(const void *a, int64_t rows_a, int64_t cols_a, int64_t ld_a, const void *b, int64_t rows_b,
                         int64_t cols_b, int64_t ld_b) {
    typedef __int128 wide;
    if (rows_a <= 0 || cols_a <= 0 || rows_b <= 0 || cols_b <= 0) return false;
    const wide at_a = (wide)reinterpret_cast<uintptr_t>(a), at_b = (wide)reinterpret_cast<uintptr_t>(b);
    if (at_a >= at_b + 2 * ((wide)(rows_b - 1) * ld_b + cols_b) || at_b >= at_a + 2 * ((wide)(rows_a - 1) * ld_a + cols_a)) return false;
    if (rows_a == 1) ld_a = ld_b;
    if (rows_b == 1) ld_b = ld_a;
    const wide ld = ld_a, off = at_b - at_a;
    if (ld_a != ld_b || ld < cols_a || ld < cols_b || off % 2) return true;
    // row j of b begins at column c of row j + m of a's grid, 0 <= c < ld
    const wide e = off / 2, m = e >= 0 ? e / ld : -((-e + ld - 1) / ld), c = e - m * ld;
    const auto meet = [&](wide rows) { return rows > -rows_b && rows < rows_a; };   // some row j of b and j + rows of a
    return (c < cols_a && meet(m)) || (c + cols_b > ld && meet(m + 1));
}

}  // namespace reqat

// Whether rows in memory with pitches have a value in common (host side, plain C++).
#pragma once

#include <stdint.h>

namespace pwlq {

// Matrices [matrices, rows, cols] of adjacent values, rows `ld` >= cols and matrices `ldm` values apart.  Two rows meet
// where they begin less than cols values from each other.
inline bool matrices_meet(int64_t matrices, int64_t rows, int64_t cols, int64_t ld, int64_t ldm) {
    if (matrices < 2) return false;
    if (ldm < cols) return true;
    if (rows < 2 || rows - 1 <= (ldm - cols) / ld) return false;                       // each ends before the next begins
    if (ld >= cols && matrices - 1 <= (ld - cols) / ldm) return false;                 // rows between one another's
    for (int64_t i = 1; i < matrices; ++i) {              // the two rows of the first matrix around row 0 of matrix i
        const int64_t at = i * ldm, row = at / ld;
        if ((row < rows && at - row * ld < cols) || (row + 1 < rows && (row + 1) * ld - at < cols)) return true;
    }
    return false;
}

// `rows` rows of `a` values at x and as many of `b` values at y, ldx >= a and ldy >= b values of `size` bytes apart.
inline bool rows_meet(const void* x, int64_t ldx, int64_t a, const void* y, int64_t ldy, int64_t b, int64_t rows, int64_t size) {
    const int64_t from = (int64_t)reinterpret_cast<uintptr_t>(x), to = (int64_t)reinterpret_cast<uintptr_t>(y);
    const int64_t px = ldx * size, py = ldy * size;
    a *= size;
    b *= size;
    if (from + (rows - 1) * px + a <= to || to + (rows - 1) * py + b <= from) return false;
    if (rows == 1) return true;
    if (px == py) {                                       // all rows meet alike, those past an end excepted (above)
        const int64_t off = ((to - from) % px + px) % px;
        return off < a || off + b > px;
    }
    for (int64_t i = 0; i < rows; ++i) {                  // the first row of y that ends behind the beginning of x's row i
        const int64_t before = from + i * px - to - b, j = before < 0 ? 0 : before / py + 1;
        if (j < rows && to + j * py < from + i * px + a) return true;
    }
    return false;
}

}  // namespace pwlq

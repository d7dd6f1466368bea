// Whether outputs in memory with pitches have a value in common (host side, plain C++).
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

}  // namespace pwlq

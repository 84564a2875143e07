// Whether two matrices (or several) in memory whose rows are the same distances apart have anything in common. The spans from
// first to last may cross without it: columns of one buffer next to each other. Checked without a GPU
// (tests/rows_meet_check.cc).
#pragma once
#include <stdint.h>

namespace sage {

// Rows of a_width and b_width, `pitch` apart (at least as wide as either), `rows` of them; those of b begin d behind those of a.
inline bool rows_meet(int64_t d, int64_t pitch, int64_t rows, int64_t a_width, int64_t b_width) {
    // a row has at most two of the others near enough, one on either side
    int64_t q = d / pitch;
    if (q * pitch > d) --q;
    for (int64_t k = q; k <= q + 1; ++k) {
        const int64_t left = d - k * pitch;
        if (k > -rows && k < rows && -b_width < left && left < a_width) return true;
    }
    return false;
}

// The same for `groups` of such rows, `apart` from each other, which is at least what a group spans.
inline bool groups_meet(int64_t d, int64_t apart, int64_t groups, int64_t pitch, int64_t rows, int64_t a_width, int64_t b_width) {
    int64_t q = d / apart;
    if (q * apart > d) --q;
    for (int64_t k = q; k <= q + 1; ++k)
        if (k > -groups && k < groups && rows_meet(d - k * apart, pitch, rows, a_width, b_width)) return true;
    return false;
}

}  // namespace sage

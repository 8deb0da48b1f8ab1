// Arithmetic of the calls on the caller's own memory on numbers alone, for the host and the kernels (and for a plain C++ compiler).
#pragma once
#include "nfd_attn_plan.h"

// Rows start .. end - 1 of a buffer of n_rows, whatever device memory says: both ends are clamped into 0 .. n_rows before anything is formed of
// them, so that first and first + n lie in 0 .. n_rows and no difference leaves an int.
struct RowSpan {
    int first, n;
};
NFD_HD int clamp_row(int row, int n_rows) { return row < 0 ? 0 : row > n_rows ? n_rows : row; }
NFD_HD RowSpan rows_between(int start, int end, int n_rows) {
    const int a = clamp_row(start, n_rows), b = clamp_row(end, n_rows);
    return {a, b > a ? b - a : 0};
}

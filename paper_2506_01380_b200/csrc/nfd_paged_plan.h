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

// Probabilities of states are formed 2^-bits of their size: with a reference m of a row that may be short of its largest score, n of them of up to
// 2^growth have a sum of 1 at most then, so that O, a sum of values times them, is no larger than the largest value and leaves fp32 for no
// finite one; the quotient of O and the sum does not know of it.  (What it costs is at the other end: small values
// lose bits in O, which ends at 2^-149 whatever the scale.)
NFD_HD int sum_bits(int growth, int n) {
    if (n <= 1) return growth;
#ifdef __CUDA_ARCH__
    return growth + 32 - __clz(n - 1);
#else
    return growth + 32 - __builtin_clz((unsigned int)n - 1);
#endif
}

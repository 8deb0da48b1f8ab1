"""Arithmetic of the calls on the caller's own memory (csrc/nfd_paged_plan.h), on the CPU."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "nfd_paged_plan.h"
extern "C" void span(int start, int end, int n_rows, int *out) {
    const RowSpan r = rows_between(start, end, n_rows);
    out[0] = r.first, out[1] = r.n;
}
extern "C" int bits(int growth, int n) { return sum_bits(growth, n); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2506_01380_b200", "csrc"), "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    return C.CDLL(str(d / "plan.so"))


def test_row_starts_of_any_value_stay_in_the_buffer(lib):
    """Ends below 0 too: formed before it is clamped, 8 rows from 4 on with an end of -2^31 would be 2^31 - 4 rows."""
    low, high = -(1 << 31), (1 << 31) - 1
    values = [low, low + 1, low + 8, -(1 << 30), -7, -1, 0, 1, 4, 7, 8, 9, 200, 1 << 30, high - 1, high]
    out = (C.c_int * 2)()
    for n_rows in (0, 1, 8, 200, 1 << 30):
        for a in values:
            for b in values:
                lib.span(a, b, n_rows, out)
                first, n = out
                assert 0 <= first <= n_rows and 0 <= n <= n_rows - first, (a, b, n_rows)
                inside = [min(max(x, 0), n_rows) for x in (a, b)]
                assert (first, n) == (inside[0], max(0, inside[1] - inside[0]))


def test_probabilities_of_all_keys_add_up_to_one_at_most(lib):
    """n probabilities of 2^growth, scaled: the next power of two of n, and no bit more."""
    for n in list(range(1, 5000)) + [(1 << b) + d for b in range(13, 30) for d in (-1, 0, 1)] + [1 << 30]:
        for growth in (1, 8, 24):
            b = lib.bits(growth, n) - growth
            assert n <= 1 << b and (b == 0 or n > 1 << b - 1), n
    assert lib.bits(8, 0) == 8

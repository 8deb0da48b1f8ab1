"""Arithmetic of the calls on the caller's own memory (csrc/nfd_paged_plan.h), on the CPU."""
import ctypes as C
import os
import shutil
import subprocess
from fractions import Fraction

import numpy as np
import pytest

from oracle import paged_oracle as P

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "nfd_paged_plan.h"
extern "C" void span(int start, int end, int n_rows, int *out) {
    const RowSpan r = rows_between(start, end, n_rows);
    out[0] = r.first, out[1] = r.n;
}
extern "C" float step(float lo, float hi) { return kv4_step(kv4_range(lo, hi)); }
extern "C" float range(float lo, float hi) { return kv4_range(lo, hi); }
extern "C" int bits(int growth, int n) { return sum_bits(growth, n); }
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("paged")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2506_01380_b200", "csrc"), "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    lib = C.CDLL(str(d / "plan.so"))
    for f in (lib.step, lib.range):
        f.restype, f.argtypes = C.c_float, [C.c_float, C.c_float]
    return lib


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


def _step(lo, hi):
    """The smallest number of 4 significant bits, at least 2^-100, with 15 of it at least hi - lo, in fractions."""
    r = Fraction(float(hi)) - Fraction(float(lo))
    e = max(-100, int(np.floor(np.log2(max(float(r), 1e-40) / 15))) - 1)
    while True:
        for m in range(8, 16):
            if Fraction(2) ** e * m / 8 * 15 >= r:
                return Fraction(2) ** e * m / 8
        e += 1


def test_steps_of_4_bit_numbers_by_their_definition(lib):
    """Ranges of all sizes; those next to 15 steps from either side by any amount, of which fp32 loses some when it forms hi - lo.  The
    oracle has the same steps."""
    rng = np.random.default_rng(0)
    f = np.float32
    pairs = [(-1e-8, 15), (-1e-30, 15), (-15, 1e-9), (-15, 15), (0, 0), (0, 15), (-2.0 ** -19, 30 - 2.0 ** -19), (-1e-45, 1e-45), (0, 1.9e-29),
             (-1.7e38, 1.7e38), (0, np.finfo(f).max), (-2.0 ** 102, np.finfo(f).max - 2.0 ** 104)]
    for _ in range(4000):
        lo, hi = -abs(rng.standard_normal()) * 10.0 ** rng.uniform(-34, 36), abs(rng.standard_normal()) * 10.0 ** rng.uniform(-34, 36)
        pairs += [(lo, hi), (lo, -lo * rng.uniform(0, 2))]
        edge = 15 * 2.0 ** int(rng.integers(-100, 120)) * int(rng.integers(8, 16)) / 8
        part = f(edge * rng.choice([2.0 ** -int(rng.integers(1, 60)), rng.uniform(0, 1)]))
        near = f(edge - float(part))
        for big in (near, np.nextafter(near, f(0)), np.nextafter(near, f(np.inf)), f(edge)):
            pairs += [(-part, big), (-big, part)]
    for lo, hi in pairs:
        lo, hi = float(f(lo)), float(f(hi))
        want = _step(lo, hi)
        assert Fraction(lib.step(lo, hi)) == want, (lo, hi)
        x = np.zeros(32, f)
        x[3], x[4] = lo, hi
        n, z, step = P.kv4_quantise(x[None])
        assert Fraction(float(step[0, 0])) == want and int(z[0, 0]) == round(Fraction(-lo) / want), (lo, hi)
    top = float(np.finfo(f).max)
    for lo, hi in ((-1.0, top), (-top, top), (-2e38, 2e38), (-2.0 ** 102, top)):
        x = np.zeros(32, f)
        x[3], x[4] = lo, hi
        assert lib.range(lo, hi) == np.inf and np.isnan(P.kv4_quantise(x[None])[2]).all()

"""The polynomial exponential of the attention of many rows (csrc/nfd_attn_block.cuh), its own lines compiled for the CPU."""
import ctypes as C
import os
import re
import shutil
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2506_01380_b200", "csrc")
# what the GPU has and a C++ compiler has not; products and sums of pairs are rounded once each, flush2 takes subnormal numbers to 0
SHIM = r"""
#include <math.h>
#include <string.h>
#define __device__
#define __forceinline__ inline
struct float2 { float x, y; };
static float2 make_float2(float x, float y) { return {x, y}; }
static float2 fadd2(float2 a, float2 b) { return {a.x + b.x, a.y + b.y}; }
static float2 ffma2(float2 a, float2 b, float2 c) { return {fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y)}; }
static int __float_as_int(float x) { int b; memcpy(&b, &x, 4); return b; }
static float __int_as_float(int b) { float x; memcpy(&x, &b, 4); return x; }
static float __saturatef(float x) { return x > 0.f ? x < 1.f ? x : 1.f : 0.f; }
static float flush(float x) { return fpclassify(x) == FP_SUBNORMAL ? 0.f : x; }
static float2 flush2(float2 a) { return {flush(a.x), flush(a.y)}; }
"""
CALL = r"""
extern "C" void run(const float *x, float *y, int n) {
    for (int i = 0; i < n; ++i) {
        const float2 p = block_exp2_poly(make_float2(x[i], 0.f), 1.f, 0.f), q = block_exp2_poly(make_float2(0.f, x[i] + 3.f), 1.f, 3.f);
        y[2 * i] = p.x, y[2 * i + 1] = q.y;
    }
}
extern "C" void scores(const float *s, float c, float mc, float *y, float *x, int n) {
    for (int i = 0; i < n; ++i) y[i] = block_exp2_poly(make_float2(s[i], s[i]), c, mc).x, x[i] = fmaf(s[i], c, -mc);
}
"""
# Relative: the polynomial's own 1.0e-4; an argument that may be formed in steps of 2^-24 of a range of 2^8 and of constants rounded to that: off by three
# half steps, 3 x 2^-17 ln 2; three roundings of 2^-24, and one of x + 3.
ERROR = 1.0e-4 + 3 * 2.0 ** -17 * 0.7 + 3 * 2.0 ** -24 + 127 * 2.0 ** -24


@pytest.fixture(scope="module")
def exp2(tmp_path_factory):
    text = open(os.path.join(CSRC, "nfd_attn_block.cuh")).read()
    body = re.search(r"^__device__ __forceinline__ float2 block_exp2_poly\(.*?^}\n", text, re.S | re.M).group(0)
    d = tmp_path_factory.mktemp("exp2")
    (d / "exp2.cpp").write_text(SHIM + body + CALL)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-fwrapv", "-ffp-contract=off", "-shared", "-fPIC", "-o", str(d / "exp2.so"),
                    str(d / "exp2.cpp")], check=True)
    lib = C.CDLL(str(d / "exp2.so"))

    def run(x):
        """[n, 2]: 2^x as the first and as the second of a pair, the second as 2^((x + 3) - 3)."""
        x = np.ascontiguousarray(x, np.float32)
        y = np.zeros((len(x), 2), np.float32)
        lib.run(x.ctypes.data_as(C.c_void_p), y.ctypes.data_as(C.c_void_p), len(x))
        return y

    def scores(s, c, mc):
        """2^(s c - mc), and the argument as the other columns form it."""
        s = np.ascontiguousarray(s, np.float32)
        y, x = np.zeros_like(s), np.zeros_like(s)
        lib.scores(s.ctypes.data_as(C.c_void_p), C.c_float(c), C.c_float(mc), y.ctypes.data_as(C.c_void_p), x.ctypes.data_as(C.c_void_p), len(s))
        return y, x
    run.scores = scores
    return run


def test_within_its_range(exp2):
    x = np.concatenate([np.linspace(-125.9, 126.9, 400001), np.arange(-125, 127), np.arange(-125, 127) + 0.5]).astype(np.float32)
    want = np.exp2(x.astype(np.float64))
    assert (np.abs(exp2(x) - want[:, None]) <= ERROR * want[:, None]).all()


def test_above_its_range_a_sum_cannot_pass_for_a_small_one(exp2):
    """A part's sum is looked at for what outgrows the reference: it has to be large, or NaN, wherever one of its scores is, and where one is NaN."""
    x = np.concatenate([np.linspace(126.9, 600, 100001), [128, 129, 129.5, 130, 150, 178, 255.5, 256, 300, 383, 384, 390, 512, 1e5, 4194304, 1.3e7, 1e30, 3e38,
                                                        np.inf, np.nan]])
    y = exp2(x)
    assert not (y < 2.0 ** 126).any(), x[(y < 2.0 ** 126).any(1)]


def test_below_its_range_it_is_nothing(exp2):
    """Not a number that sends the warp to its keys again, nor one that counts beside large values."""
    x = np.concatenate([np.linspace(-600, -126, 100001), [-126.4, -126.5, -127, -127.4, -127.5, -128, -129, -150, -253, -256, -383, -500, -1e5, -4194304, -1.3e7, -1e30,
                                                          -3e38, -np.inf]])
    y = exp2(x)
    assert ((y >= 0) & (y <= 2.0 ** -126)).all() and (y[x < -126.1] == 0).all()


@pytest.mark.parametrize("dh", [32, 64, 128])
def test_its_argument_is_that_of_the_other_columns_whatever_the_scores(exp2, dh):
    """Scores that all have a large part in common, which their reference takes away: what is left is rounded once, as in the columns beside."""
    c = float(np.float32(np.log2(np.e) / np.sqrt(dh)))
    for common in (0.0, 1e3, -1e4, 1e5, -3e6):
        s = (common + np.linspace(-200, 0, 4001)).astype(np.float32)
        y, x = exp2.scores(s, c, float(np.float32(common * c + 57)))
        inside = x > -125.9
        want = np.exp2(x.astype(np.float64))
        assert inside.any() and (np.abs(y - want)[inside] <= ERROR * want[inside]).all() and (y[x < -126.1] == 0).all(), common

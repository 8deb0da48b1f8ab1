"""Arithmetic of the calls around a block's projections (csrc/nfd_paged_plan.h), on the CPU."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = r"""
#include "nfd_paged_plan.h"
extern "C" long long seen(long long held, int frame_tokens, int window, int rows) { return keys_seen(held, frame_tokens, window, rows); }
extern "C" long long prompt(int n_rows, int frame_tokens, int window, int rows) { return prompt_keys_seen(n_rows, frame_tokens, window, rows); }
extern "C" int parts(long long keys, int part) { return parts_touched(keys, part); }
extern "C" void norm(int regs, int threads, int row_bytes, int own, int *out) {
    const NormPlan p = norm_plan(regs, threads, row_bytes, own);
    out[0] = p.ctas, out[1] = p.stages;
}
"""
LAST = (1 << 31) - 1


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    d = tmp_path_factory.mktemp("block")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run([shutil.which("g++") or "g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-fsanitize=undefined", "-fno-sanitize-recover", "-I",
                    os.path.join(ROOT, "paper_2506_01380_b200", "csrc"), "-o", str(d / "plan.so"), str(d / "plan.cpp")], check=True)
    lib = C.CDLL(str(d / "plan.so"))
    lib.seen.restype, lib.seen.argtypes = C.c_longlong, [C.c_longlong] + 3 * [C.c_int]
    lib.prompt.restype, lib.prompt.argtypes = C.c_longlong, 4 * [C.c_int]
    lib.parts.argtypes = [C.c_longlong, C.c_int]
    return lib


def _span(first, rows, frame, window, length):
    """Keys from the first that token `first` sees to the last that token first + rows - 1 of a sequence of `length` sees."""
    last = first + rows - 1
    return min(length, (last // frame + 1) * frame) - max(0, first // frame - window) * frame


def test_keys_that_a_chunk_sees(lib):
    """The most over all places of the chunk: no less, or a plan would be for fewer keys than there are, and no more than are held."""
    for frame in (1, 2, 3, 7, 50, 77):
        for window in (0, 1, 2, 9):
            for rows in (1, 2, 3, 8, 50, 51, 76, 77, 78, 79, 200):
                span = max(_span(p, rows, frame, window, 10 ** 6) for p in range(20 * frame, 21 * frame))
                assert lib.seen(10 ** 6, frame, window, rows) == span, (frame, window, rows)
                assert lib.seen(span - 1, frame, window, rows) == span - 1
    assert lib.seen(1 << 30, 1 << 20, LAST, 1 << 30) == 1 << 30 and lib.seen(1 << 60, 1 << 20, LAST, 1) == 1 << 51


def test_keys_that_a_prompt_sees(lib):
    """Of one prompt, however many there are in the batch; of one whose first rows only are computed, to the end of their frame."""
    for frame in (1, 2, 7, 77, 500):
        for window in (0, 1, 5, LAST):
            for length in (1, 2, 6, 7, 8, 153, 154, 155, 400):
                for rows in {1, 2, length // 2 or 1, length}:
                    if rows > length:
                        continue
                    most = max(_span(p, 1, frame, window, length) for p in range(rows))
                    for others in (0, 1, 100000):
                        got = lib.prompt(length + others, frame, window, rows)
                        assert most <= _span(0, rows, frame, window, length) <= got <= length + others
                        assert got <= -(-rows // frame) * frame and got <= (window + (rows + frame - 2) // frame + 1) * frame
    assert lib.prompt(1353, 1, LAST, 200) == 200 and lib.prompt(1 << 30, 1 << 20, LAST, 1 << 30) == 1 << 30


def test_parts_that_keys_touch(lib):
    for part in (1, 2, 64, 96):
        for keys in (0, 1, 2, 3, 63, 64, 65, 66, 96, 97, 98, 500):
            most = max(len({(a + i) // part for i in range(keys)}) for a in range(part))
            assert lib.parts(keys, part) == most, (keys, part)
    assert lib.parts(1 << 30, 64) == (1 << 24) + 1


def test_a_wave_of_norms_is_what_the_device_holds(lib):
    """All widths that go through shared memory, of two rows of 2 or 4 bytes a number: an SM has 64 K registers, 2048 threads and 228 KB, of which a CTA takes 1 KB and whole
    units of 128 bytes beside its own.  No CTA is counted that has to wait for another one to leave, and no room for two more is left over."""
    out = (C.c_int * 2)()
    for size in (4, 6, 8):
        for width in range(264, 16385, 8):
            row, pieces = width * size, width // 8
            if 2 * row > 196608:
                continue
            v = 1 if pieces <= 512 else 2 if pieces <= 1024 else 4
            threads = (-(-pieces // v) + 31) // 32 * 32
            for regs in (40, 64, 80, 128):
                for own in (0, 176, 1000):
                    lib.norm(regs, threads, row, own, out)
                    ctas, stages = out
                    assert 2 <= stages <= 6 and stages * row <= 196608
                    taken = -(-(stages * row + own) // 128) * 128 + 1024
                    held = min(65536 // (regs * threads), 2048 // threads, 233472 // taken)
                    assert 1 <= ctas <= max(held, 1) and held - ctas <= 1, (size, width, regs, ctas, held)
    lib.norm(32, 128, 0, 0, out)
    assert tuple(out) == (16, 0)

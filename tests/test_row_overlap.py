"""CPU: csrc/row_overlap.h, built with the host compiler, against the sets of elements of two row-strided matrices."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2606_15682_amd import build as libbuild

SOURCE = """
#include "row_overlap.h"
extern "C" int overlap_(int64_t a, int64_t ra, int64_t ca, int64_t la, int64_t b, int64_t rb, int64_t cb, int64_t lb) {
    return reqat::rows_overlap((const void *)a, ra, ca, la, (const void *)b, rb, cb, lb);
}
"""


@pytest.fixture(scope="module")
def overlap(tmp_path_factory):
    d = tmp_path_factory.mktemp("overlap")
    (d / "o.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", libbuild.CSRC,
                    str(d / "o.cpp"), "-o", str(d / "o.so")], check=True)
    lib = ctypes.CDLL(os.path.join(str(d), "o.so"))
    lib.overlap_.argtypes = [ctypes.c_int64] * 8
    return lambda *a: bool(lib.overlap_(*a))


def elements(at, rows, cols, ld):
    return {at + 2 * (i * ld + j) for i in range(rows) for j in range(cols)}


def test_against_the_elements(overlap):
    rng = random.Random(1)
    exact = loose = 0
    for _ in range(40000):
        la = rng.randint(1, 24)
        lb = la if rng.random() < 0.7 else rng.randint(1, 24)
        ca, cb = rng.randint(0, la), rng.randint(0, lb)
        ra, rb = rng.randint(0, 5), rng.randint(0, 5)
        a, b = 1 << 20, (1 << 20) + 2 * rng.randint(-130, 130)
        shared = bool(elements(a, ra, ca, la) & elements(b, rb, cb, lb))
        got = overlap(a, ra, ca, la, b, rb, cb, lb)
        assert got == overlap(b, rb, cb, lb, a, ra, ca, la)
        if la == lb:
            assert got == shared, (ra, ca, la, b - a, rb, cb, lb)
            exact += 1
        else:
            assert got or not shared, (ra, ca, la, b - a, rb, cb, lb)
            loose += 1
    assert exact > 1000 and loose > 1000


def test_slices_of_the_fused_product(overlap):
    """q, k and v side by side in rows of 7168 elements; far strides do not overflow."""
    for rows in (1, 2, 8192):
        q, k, v = 1 << 30, (1 << 30) + 2 * 5120, (1 << 30) + 2 * 6144
        assert not overlap(q, rows, 5120, 7168, k, rows, 1024, 7168) and not overlap(k, rows, 1024, 7168, v, rows, 1024, 7168)
        assert overlap(q, rows, 5128, 7168, k, rows, 1024, 7168) and overlap(k, rows, 1024, 7168, k + 16, rows, 1024, 7168)
    assert overlap(1 << 40, 1 << 31, 128, 1 << 61, (1 << 40) + (1 << 62), 2, 128, 1 << 61)
    assert not overlap(1 << 40, 1 << 31, 128, 1 << 61, (1 << 40) + 256, 1 << 31, 128, 1 << 61)

"""The training side's kernels are those that its rules choose, no others: norm_plan's forms (csrc/norm_plan.h, built with the host
compiler) for every row length, the policy loss's numbers of vectors, and the kernels in the built library."""
import ctypes
import os
import re
import subprocess

import pytest

from paper_2606_15682_amd import build as libbuild
from paper_2606_15682_amd import reqat

SOURCE = """
#include "norm_plan.h"
using namespace reqat;
extern "C" void plan_(int64_t M, int64_t K, int bf16, int *out) {
    const NormPlan p = norm_plan(M, K, bf16 != 0);
    out[0] = p.threads; out[1] = p.vpt; out[2] = norm_least_vectors(p.threads); out[3] = norm_most_vectors(p.threads);
}
"""


@pytest.fixture(scope="module")
def forms(tmp_path_factory):
    """(bf16, threads, vectors, whole) of every length."""
    d = tmp_path_factory.mktemp("norm")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", libbuild.CSRC,
                    str(d / "plan.cpp"), "-o", str(d / "plan.so")], check=True)
    lib = ctypes.CDLL(str(d / "plan.so"))
    lib.plan_.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    out, seen = (ctypes.c_int * 4)(), set()
    for bf16, n in ((1, 8), (0, 4)):
        for K in range(1, 32769):
            lib.plan_(100, K, bf16, out)
            threads, vpt, least, most = out
            assert least <= vpt <= most and threads * vpt * n >= K > threads * (vpt - 1) * n
            assert threads <= (512 if bf16 else 1024) and (K >= n or (threads, vpt) == (64, 1))
            seen.add((bool(bf16), threads, vpt, K >= n))
    return seen


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(reqat.LIB_PATH):
        pytest.skip("libreqat.so not built")
    names = subprocess.run(["nm", "-C", reqat.LIB_PATH], capture_output=True, text=True, check=True).stdout
    return lambda name: {tuple(m.split(", ")) for m in re.findall(r" d void reqat::.*%s<([^>]*)>" % name, names)}


@pytest.mark.parametrize("name", ["norm_forward_kernel", "norm_backward_kernel"])
def test_norm(forms, kernels, name):
    want = {("unsigned short" if bf16 else "float", str(threads), str(vpt), "true" if whole else "false")
            for bf16, threads, vpt, whole in forms}
    assert kernels(name) == want


def test_policy(kernels):
    want = set()
    for t, n in (("unsigned short", 8), ("float", 4)):
        for full in list(range(0, 1025, 64)) + list(range(1, 30000, 97)) + [1025]:     # whole vectors of a row
            threads = 256 if full <= 1024 else 1024
            want.add((t, str(threads), str(min(-(-full // threads), 4 if threads == 256 else 18))))
    assert kernels("policy_grad_kernel") == want

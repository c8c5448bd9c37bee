"""CPU: one workspace of a serving loop's largest sizes serves all its calls.  The size that the library names never
falls as a size grows, and covers the partial rows of the plan (csrc/kv4_plan.h, built with the host compiler)."""
import ctypes
import os
import random
import subprocess

import pytest

from paper_2606_15682_amd import build as libbuild
from paper_2606_15682_amd import reqat

pytestmark = pytest.mark.skipif(not os.path.exists(reqat.LIB_PATH), reason="libreqat.so not built")

SOURCE = """
#include "kv4_plan.h"
extern "C" int64_t pieces_(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads) {
    return reqat::kv4_plan(B, max_q, max_kv, q_heads, kv_heads).splits;
}
"""
HEADS = [(40, 8), (28, 4), (7, 1), (12, 2), (6, 1), (1, 1), (64, 64), (40, 1), (65, 1), (96, 3)]
KV = [0, 1, 255, 256, 257, 511, 512, 513, 1024, 1536, 2047, 2048, 2049, 4001, 8192, 9001, 16383, 16384, 16385, 20000,
      32768, 65536, 131072, 1 << 20, 1 << 30]


def size(B, q, kv, heads, D=128):
    return reqat.reqat_kv4_attention_workspace_bytes(B, B * q, q, kv, heads[0], heads[1], D)


@pytest.fixture(scope="module")
def pieces(tmp_path_factory):
    d = tmp_path_factory.mktemp("pieces")
    (d / "pieces.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", libbuild.CSRC,
                    str(d / "pieces.cpp"), "-o", str(d / "pieces.so")], check=True)
    lib = ctypes.CDLL(os.path.join(str(d), "pieces.so"))
    lib.pieces_.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2
    lib.pieces_.restype = ctypes.c_int64
    return lib.pieces_


@pytest.mark.parametrize("heads", HEADS)
def test_size_never_falls(heads):
    for q in (1, 2, 5, 6, 7, 16, 33, 64, 777, 8192):
        for B in (1, 2, 3, 5, 16, 63, 64, 65, 512, 2000, 65535):
            sizes = [size(B, q, kv, heads) for kv in KV]
            assert sizes == sorted(sizes), (B, q, sizes)
    for kv in KV:
        for q in (1, 5, 7, 70, 1024):
            sizes = [size(B, q, kv, heads) for B in (1, 2, 3, 7, 31, 32, 63, 64, 65, 128, 511, 512, 1000, 65535)]
            assert sizes == sorted(sizes), (kv, q, sizes)
        for B in (1, 2, 16, 64, 1000):
            sizes = [size(B, q, kv, heads) for q in (1, 2, 4, 5, 6, 7, 8, 16, 32, 33, 64, 255, 256, 1024, 8192, 100000)]
            assert sizes == sorted(sizes), (kv, B, sizes)
            sizes = [reqat.reqat_kv4_attention_workspace_bytes(B, T, 64, kv, *heads, 128) for T in range(0, 200, 7)]
            assert sizes == sorted(sizes), (kv, B, sizes)


@pytest.mark.parametrize("heads", HEADS)
def test_size_covers_the_plan(pieces, heads):
    rng = random.Random(5)
    shapes = [(B, q, kv) for B in (1, 2, 7, 64, 1000) for q in (1, 5, 7, 64, 1024) for kv in KV]
    shapes += [(rng.randint(1, 300), int(2 ** rng.uniform(0, 13)), int(2 ** rng.uniform(0, 20))) for _ in range(4000)]
    for B, q, kv in shapes:
        n = pieces(B, q, kv, *heads)
        for D in (64, 128):
            need = n * B * q * heads[0] * (4 * D + 16) if n > 1 else 0   # FP32 rows, each with its reference and sum
            assert size(B, q, kv, heads, D) >= need, (B, q, kv, n)


def test_size_is_bounded():
    """8192 pieces of 32 rows, or 510 of 256, whatever the sizes."""
    for heads in HEADS:
        for B, q, kv in ((1, 1, 1 << 30), (64, 6, 1 << 30), (65535, 8192, 1 << 30), (1, 1 << 30, 1 << 30)):
            assert size(B, q if B * q < 2 ** 31 else 2 ** 31 // B - 1, kv, heads) <= 8192 * 32 * (4 * 128 + 16)
    assert size(1, 1, 256, (40, 8)) == 0

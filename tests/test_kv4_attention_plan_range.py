"""CPU: how a call of the KV4 attention is cut at the largest sizes that its arguments can hold (csrc/kv4_plan.h, built
with the host compiler, with traps on signed overflow): no count wraps, and what no launch can hold is said not to fit."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_15682_amd import build as libbuild

SOURCE = """
#include "kv4_plan.h"
using namespace reqat;
extern "C" void plan_(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads, int64_t *out) {
    const Kv4Plan p = kv4_plan(B, max_q, max_kv, q_heads, kv_heads);
    out[0] = p.tiles; out[1] = p.qtiles; out[2] = p.splits; out[3] = p.chunk;
    out[4] = kv4_plan_fits(p, B, kv_heads);
    out[5] = kv4_piece_rows(B, max_q, max_kv, q_heads, kv_heads);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-ftrapv", "-Wall", "-Werror", "-shared", "-fPIC", "-I", libbuild.CSRC,
                    str(d / "plan.cpp"), "-o", str(d / "plan.so")], check=True)
    lib = ctypes.CDLL(os.path.join(str(d), "plan.so"))
    lib.plan_.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.POINTER(ctypes.c_int64)]

    def ask(*a):
        out = (ctypes.c_int64 * 6)()
        lib.plan_(*a, out)
        return dict(zip(("tiles", "qtiles", "splits", "chunk", "fits", "rows"), out))
    return ask


def test_the_largest_sizes(plan):
    for B in (1, 2, 4097, 65535):
        for q in (1, 33, 1 << 20, 2 ** 31 - 1):
            for heads, kv_heads in ((1, 1), (40, 8), (65535, 1), (65535, 65535), (65535, 3)):
                for kv in (0, 1, 300, 1 << 30):
                    p = plan(B, q, kv, heads, kv_heads)
                    rows = q * (heads // kv_heads)
                    assert p["qtiles"] == -(-rows // (16 * p["tiles"])), (B, q, heads, kv_heads)
                    groups = B * kv_heads * p["qtiles"] * p["splits"]
                    assert p["fits"] == (groups < 1 << 23), (B, q, heads, kv_heads, kv)
                    assert p["splits"] >= 1 and p["splits"] * p["chunk"] >= kv
                    need = p["splits"] * B * q * heads if p["splits"] > 1 else 0
                    assert need <= p["rows"] <= 8192 * 32, (B, q, heads, kv_heads, kv)

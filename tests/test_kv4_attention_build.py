"""CPU checks of the attention over the paged KV4 cache: the wait states in front of its direct-to-LDS loads, in the
assembly that hipcc makes; and the rule that cuts a call (csrc/kv4_plan.h, built with the host compiler)."""
import ctypes
import os
import subprocess

import pytest

from paper_2606_15682_amd import build as libbuild
from tests.test_direct_to_lds_hazards import _assembly, hazards

SOURCE = """
#include "kv4_plan.h"
using namespace reqat;
extern "C" void plan_(int64_t B, int64_t max_q, int64_t max_kv, int q_heads, int kv_heads, int *out) {
    const Kv4Plan p = kv4_plan(B, max_q, max_kv, q_heads, kv_heads);
    out[0] = p.tiles; out[1] = p.qtiles; out[2] = p.waves; out[3] = p.splits; out[4] = p.chunk;
    out[5] = kv4_plan_fits(p, B, kv_heads);
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I", libbuild.CSRC,
                    str(d / "plan.cpp"), "-o", str(d / "plan.so")], check=True)
    lib = ctypes.CDLL(os.path.join(str(d), "plan.so"))
    lib.plan_.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2 + [ctypes.POINTER(ctypes.c_int)]

    def ask(*a):
        out = (ctypes.c_int * 6)()
        lib.plan_(*a, out)
        return dict(zip(("tiles", "qtiles", "waves", "splits", "chunk", "fits"), out))
    return ask


def test_wait_states(tmp_path):
    loads, bad = hazards(_assembly("kv4_attention.hip", str(tmp_path / "out.s")))
    assert loads >= 8 * 2 * 6                        # two places of every instance of the kernel
    assert not bad, "%d of %d loads:\n%s" % (len(bad), loads, "\n".join(bad[:20]))


@pytest.mark.parametrize("args,want", [
    ((1, 1, 256, 12, 2), (1, 4, 1)), ((1, 1, 257, 12, 2), (1, 8, 1)), ((1, 1, 512, 12, 2), (1, 8, 1)),
    ((33, 1, 512, 40, 8), (1, 4, 2)), ((1, 1, 513, 12, 2), (1, 4, 3)), ((1, 1, 131072, 40, 8), (1, 4, 64)),
    ((1, 1, 131072, 7, 1), (1, 4, 256)), ((64, 1, 16384, 40, 8), (1, 4, 11)), ((128, 1, 2000, 40, 8), (1, 4, 1)),
    ((2000, 1, 131072, 40, 8), (1, 4, 1)), ((16, 5, 4001, 40, 8), (2, 4, 4)), ((16, 7, 4001, 40, 8), (16, 4, 2)),
    ((1, 8192, 8192, 40, 8), (16, 4, 1)), ((1, 65, 40000, 40, 8), (16, 4, 16))])
def test_how_a_call_is_cut(plan, args, want):
    p = plan(*args)
    assert (p["tiles"], p["waves"], p["splits"]) == want and p["fits"]


def test_pieces_cover_every_length(plan):
    for B in (0, 1, 2, 7, 64, 1000, 65535):
        for heads, group in ((1, 1), (1, 40), (2, 6), (8, 5), (64, 1)):
            for q in (1, 3, 9, 64, 4096):
                for kv in (0, 1, 16, 255, 256, 257, 511, 513, 2048, 2049, 5000, 131072, 1000003, 1 << 30):
                    p = plan(B, q, kv, heads * group, heads)
                    assert 1 <= p["splits"] <= 256 and p["chunk"] % 128 == 0 and p["chunk"] > 0
                    assert p["splits"] * p["chunk"] >= kv and (p["splits"] - 1) * p["chunk"] < max(kv, 1)
                    assert p["qtiles"] * 16 * p["tiles"] >= q * group
                    assert p["tiles"] == 16 or p["qtiles"] == 1          # the decode kernel takes all rows at once
                    assert p["splits"] == 1 or B * heads * p["splits"] <= max(8192, 2 * 512 + B * heads)


def test_what_does_not_fit_a_launch(plan):
    assert not plan(65535, 1, 100, 256, 256)["fits"]
    assert plan(65535, 1, 100, 64, 64)["fits"]
    assert not plan(65535, 2 ** 31 - 1, 100, 40, 8)["fits"]

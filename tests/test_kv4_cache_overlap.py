"""CPU: outputs of the KV4 cache's calls over memory that the call still reads or writes elsewhere are refused, before a
launch."""
import os

import pytest

from paper_2606_15682_amd import reqat
from tests.test_kv4_cache_abi import E_UNSUP, P, append, gather

pytestmark = pytest.mark.skipif(not os.path.exists(reqat.LIB_PATH), reason="libreqat.so not built")


@pytest.mark.parametrize("name,ld", [("k", "ldk"), ("v", "ldv")])
def test_rotated_queries_over_the_keys_or_values(name, ld):
    far = 64 * P
    other = {"k": "v", "v": "k"}[name]
    for where in (far, far + 16, far + 2 * 3 * 1024, far + 2 * 4 * 1024 - 16, far - 2 * 240):
        assert append(**{name: where, other: 32 * P, "q_out": far}) == E_UNSUP, where - far
    # one buffer: the queries' columns 0 .. 1023, keys or values from the last of them
    assert append(**{"q": far, "ldq": 1536, "q_out": far, "ldqo": 1536, name: far + 2 * 1016, ld: 1536}) == E_UNSUP


def test_values_read_back_over_the_keys():
    for where in (P, P + 16, P + 2 * 4 * 256 - 16):
        assert gather(v=where) == E_UNSUP and gather(k=where, v=P) == E_UNSUP
    assert gather(ldk=512, ldv=512, v=P + 2 * 248) == E_UNSUP
    assert gather(ldk=264, ldv=512, v=P + 2 * 600) == E_UNSUP

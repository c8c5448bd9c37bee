"""CPU build of the paged KV4 cache's host code under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU; device code
is never instrumented): every rejection path and the workspace query, at the ends of the sizes' ranges.  Only the sources that
these calls reach are built; the library's other launches stay unresolved, and nothing calls them."""
import os
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2606_15682_amd import build as libbuild
from tests.test_sanitizers import HERE, SAN_ENV, _run


def test_kv4_cache_validation_under_asan_ubsan(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    clang = "/opt/rocm/llvm/bin/clang"
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("ROCm compilers not found")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = [f for f in libbuild.HIPCC_FLAGS if f not in ("-shared", "-O3")] + ["-O1", "-g"] + san
    sources = ["api.hip", "kv4_cache.hip", "kv4_attention.hip"]
    objs = [str(tmp_path / (s[:-4] + ".o")) for s in sources]
    with ThreadPoolExecutor(len(sources)) as ex:
        list(ex.map(_run, [[hipcc, *flags, "-c", os.path.join(libbuild.CSRC, s), "-o", o] for s, o in zip(sources, objs)]))
    lib = str(tmp_path / "libreqat_san.so")
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *san, "-Wl,-z,lazy", "-o", lib, *objs])
    exe = str(tmp_path / "kv4_cache_driver")
    _run([clang, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
          os.path.join(HERE, "kv4_cache_driver.c"), lib, "-Wl,--allow-shlib-undefined", "-Wl,-z,lazy",
          "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    r = _run([exe], env=SAN_ENV)
    assert "kv4 cache driver ok" in r.stdout, r.stdout
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr[-3000:]

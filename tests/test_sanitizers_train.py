"""CPU build of the training side's host code under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU; device code is
never instrumented): every entry point with sizes and strides at the ends of their ranges, refused or taken, before launches
that do nothing."""
import os

import pytest

from paper_2606_15682_amd import build as libbuild
from tests.test_sanitizers import HERE, SAN_ENV, _run


def test_training_calls_under_asan_ubsan(tmp_path):
    hipcc = "/opt/rocm/bin/hipcc"
    clang = "/opt/rocm/llvm/bin/clang"
    if not (os.path.exists(hipcc) and os.path.exists(clang)):
        pytest.skip("ROCm compilers not found")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-omit-frame-pointer"]
    flags = [f for f in libbuild.HIPCC_FLAGS if f not in ("-shared", "-O3")] + ["-O1", "-g", "-I", libbuild.CSRC] + san
    sources = [os.path.join(libbuild.CSRC, "api_train.hip"), os.path.join(HERE, "train_launches.hip")]
    objs = [str(tmp_path / ("%d.o" % i)) for i in range(2)]
    for s, o in zip(sources, objs):
        _run([hipcc, *flags, "-c", s, "-o", o])
    lib = str(tmp_path / "libreqat_san.so")
    _run([hipcc, "--offload-arch=gfx950", "-shared", "-fPIC", *san, "-o", lib, *objs])
    exe = str(tmp_path / "train_driver")
    _run([clang, "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
          os.path.join(HERE, "train_driver.c"), lib, "-lm", "-Wl,--allow-shlib-undefined",
          "-Wl,-rpath," + str(tmp_path), "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
    r = _run([exe], env=SAN_ENV)
    assert "train driver ok" in r.stdout, r.stdout
    assert "runtime error" not in r.stderr and "ERROR: AddressSanitizer" not in r.stderr, r.stderr[-3000:]

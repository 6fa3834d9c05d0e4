"""Host code of the norm, cache and cached-attention entry points under AddressSanitizer and UndefinedBehaviorSanitizer: all checks
and plans over sizes and strides of every kind (CPU only, no GPU work)."""

import os
import tempfile

import pytest

from paper_2508_10774_amd import build
from tests.test_sanitizers import ENV, ROOT, _run


def test_host_code_around_the_attention_call_is_clean():
    clangxx = "/opt/rocm/llvm/bin/clang++"
    if not os.path.exists(clangxx):
        pytest.skip("no ROCm clang++ for the driver")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=undefined", "-Xarch_host", "-fno-omit-frame-pointer", "-g"]
    with tempfile.TemporaryDirectory() as tmp:
        lib = build.build_lib(extra=san, lib_path=os.path.join(tmp, "libasa_san.so"), objdir=tmp,
                              link_extra=["-fsanitize=address", "-fsanitize=undefined", "-fno-gpu-sanitize"])
        exe = os.path.join(tmp, "san_cache")
        _run([clangxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
              "-I" + os.path.join(ROOT, "include"), os.path.join(ROOT, "tests", "sanitize_cache_driver.cpp"), lib,
              "-Wl,-rpath," + tmp, "-Wl,-rpath,/opt/rocm/lib", "-o", exe])
        out = _run([exe], env=dict(ENV, ASAN_OPTIONS="detect_leaks=0"))
        assert out.strip().endswith("ok"), out

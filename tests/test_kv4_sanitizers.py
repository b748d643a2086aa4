"""Address and undefined-behaviour sanitizers over the host code of the 4-bit cache's and of eviction's entry points."""
import os
import subprocess
import sys

from tests.test_sanitizers import OUT, ROOT, _run


def test_kv4_and_eviction_host_code_under_address_and_ub_sanitizers():
    sys.path.insert(0, ROOT)
    from paper_2603_12201_amd import build as lib_build
    os.makedirs(OUT, exist_ok=True)
    exe = os.path.join(OUT, "kv4_san")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-g"]
    objs = lib_build.compile_objects(extra=san, tag=".san")
    subprocess.check_call(["hipcc", "--offload-arch=gfx950", "-std=c++17", "-I" + os.path.join(ROOT, "include")] + san +
                          ["-x", "c++", os.path.join(ROOT, "tests", "sanitize", "kv4_driver.cpp"), "-x", "none"] + objs + ["-o", exe])
    assert "kv4 sanitizer run ok" in _run(exe)

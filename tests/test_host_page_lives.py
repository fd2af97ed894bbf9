"""Pools, caches, pages and lists whose lives end in an unusual order, in a native program built with AddressSanitizer + UndefinedBehaviorSanitizer over the
host code (no GPU, no HIP library: tests/native/page_lives.cpp)."""
import os
import shutil
import subprocess

import pytest

from test_host_library import ROOT


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path_factory.mktemp("lives") / "page_lives")
    csrc = os.path.join(ROOT, "paper_2603_16104_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", os.path.join(ROOT, "tests", "native", "page_lives.cpp"),
                           *(os.path.join(csrc, f) for f in ("api.cpp", "operators.cpp", "pages.cpp", "cache.cpp")), "-o", exe])
    return exe


@pytest.mark.timeout(600)
@pytest.mark.parametrize("name", ["caches_after_their_pool", "evictions_beside_forks", "forks_that_end_cached_sequences", "copies_between_pools_that_overlap",
                                  "lists_that_fail_on_their_way"])
def test_lives(program, name):
    r = subprocess.run([program, name], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "1 programs, 0 failed checks" in out, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]

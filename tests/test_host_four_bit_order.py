"""The order of a 4-bit plan's workgroups, in a native program built with AddressSanitizer + UndefinedBehaviorSanitizer over the host code (no GPU, no HIP
library: tests/native/four_bit_order.cpp)."""
import os
import shutil
import subprocess

import pytest

from test_host_library import ROOT


@pytest.mark.timeout(600)
def test_every_set_goes_out_once(tmp_path):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "four_bit_order")
    csrc = os.path.join(ROOT, "paper_2603_16104_amd", "csrc")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", os.path.join(ROOT, "tests", "native", "four_bit_order.cpp"),
                           *(os.path.join(csrc, f) for f in ("api.cpp", "operators.cpp", "pages.cpp", "cache.cpp")), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    out = r.stdout + r.stderr
    assert r.returncode == 0 and " 0 failed checks" in out, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]

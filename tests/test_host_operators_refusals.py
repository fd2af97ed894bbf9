"""What the calls around a step's attention refuse in the middle of a plan's life, in a native program built with AddressSanitizer +
UndefinedBehaviorSanitizer over the host code (no GPU, no HIP library: tests/native/operators_refusals.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path_factory.mktemp("refusals") / "operators_refusals")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", os.path.join(ROOT, "tests", "native", "operators_refusals.cpp"), "-o", exe])
    return exe


@pytest.mark.parametrize("name", ["appends_to_one_block", "prompts_into_shared_pages", "appends_under_capture"])
def test_refusals_after_other_calls(program, name):
    r = subprocess.run([program, name], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "1 programs, 0 failed checks" in out, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]

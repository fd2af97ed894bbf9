"""What the calls around a step's attention refuse in the middle of a plan's life, in a native program built with AddressSanitizer +
UndefinedBehaviorSanitizer over the host code (no GPU, no HIP library: tests/native/operators_refusals.cpp); and of rows that do not belong together."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import fake_pool

A = 0x100000
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


# ---- rows of the stores (addresses are never dereferenced here)
def store_code(x):
    pool = fake_pool()
    plan = hkv.hkv_prefill_plan_create(pool, [0, 5, 9], [[0, 1], [2, 3]], [20, 9], 8, hkv.PLAN_HOST_ONLY)
    try:
        with pytest.raises(hkv.HkvError) as e:
            hkv.hkv_prefill_plan_store(plan, x, 0)
        return e.value.code, hkv.last_error()
    finally:
        hkv.hkv_prefill_plan_destroy(plan)
        hkv.kv_pool_destroy(pool)


def test_several_axes_need_a_stride():
    x = hkv.qkv_rows(A, A, A, 2 * A, rotary_dim=128, inv_freq=A, positions=A, n_axes=3, axis=[0, 1, 2, 1] * 16)
    for stride, text in ((0, "position_stride"), (-9, "position_stride"), (9, "host-only")):
        x.position_stride = stride
        code, error = store_code(x)
        assert code == hkv.EINVAL and text in error
    x.n_axes, x.axis, x.position_stride = 1, None, 0     # (one axis: there is nothing to step over)
    assert "host-only" in store_code(x)[1]


def test_places_expanded_over_the_axes_are_one_axis():
    import torch
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    how = dict(q=q, k=q[:, :2].contiguous(), v=q[:, :2].contiguous(), q_out=q, rotary_dim=128, inv_freq=torch.zeros(64, dtype=torch.float64), axis=np.arange(64) % 3)
    line = torch.arange(4, dtype=torch.int32)
    x = hkv.qkv_rows(positions=line.expand(3, 4), **how)
    assert x.n_axes == 1 and x.axis is None and x.positions == line.data_ptr()
    assert "host-only" in store_code(x)[1]
    x = hkv.qkv_rows(positions=line.repeat(3, 1), **how)
    assert x.n_axes == 3 and x.axis is not None and x.position_stride == 4
    for bad in (dict(axis=np.arange(64) % 4), dict(axis=None)):   # what is wrong without them stays wrong
        assert store_code(hkv.qkv_rows(positions=line.expand(3, 4), **{**how, **bad}))[0] == hkv.EINVAL


def test_rows_that_are_fewer_than_the_queries_are_refused():
    import torch
    q, k = torch.zeros(6, 8, 128, dtype=torch.bfloat16), torch.zeros(9, 2, 128, dtype=torch.bfloat16)
    how = dict(q=q, k=k, v=k, q_out=q, rotary_dim=128, inv_freq=torch.zeros(64, dtype=torch.float64))
    grid = torch.zeros(3, 6, dtype=torch.int32)
    three = dict(positions=grid, axis=np.arange(64) % 3)
    for ok in (dict(), dict(k=k[:6]), dict(positions=grid[0]), three, dict(positions=torch.zeros(3, 7, dtype=torch.int32), axis=np.arange(64) % 2, n_axes=2),
               dict(positions=torch.zeros(3, 2, 3, dtype=torch.int32), axis=np.arange(64) % 3), dict(k=A, v=A, positions=A)):
        hkv.qkv_rows(**{**how, **ok})
    for bad in (dict(k=k[:5]), dict(v=k[:5]), dict(k=k[:0]), dict(positions=grid[0, :5]), dict(positions=grid[:, :5], axis=np.arange(64) % 3),
                {**three, "n_axes": 4}, dict(positions=grid[0], axis=np.arange(64) % 3, n_axes=3), dict(positions=grid[:, :5].expand(3, 5), n_axes=1),
                dict(positions=grid[0, 0]), dict(positions=torch.zeros(12, dtype=torch.int32)[::2])):
        with pytest.raises(ValueError):
            hkv.qkv_rows(**{**how, **bad})


def test_frequencies_are_float64():
    import torch
    q = torch.zeros(6, 8, 128, dtype=torch.bfloat16)
    how = dict(q=q, k=q, v=q, q_out=q, rotary_dim=128)
    hkv.qkv_rows(inv_freq=torch.zeros(64, dtype=torch.float64), **how)
    for wide in (torch.int64, torch.complex64):
        with pytest.raises(ValueError):
            hkv.qkv_rows(inv_freq=torch.zeros(64, dtype=wide), **how)

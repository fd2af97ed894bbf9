"""The calls that move pages (copies between pools, forks, compaction) on the host: refusals and bookkeeping (addresses are never dereferenced
here), and in a native program built with AddressSanitizer + UndefinedBehaviorSanitizer (no GPU, no HIP library: tests/native/pages_check.cpp)."""
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import FAKE_K, FAKE_V, ROOT, fake_pool


def code(f, *args, **kw):
    with pytest.raises(hkv.HkvError) as e:
        f(*args, **kw)
    return e.value.code


def counts(pool, n):
    return [hkv.kv_pool_refcount(pool, i) for i in range(n)]


@pytest.mark.timeout(600)
def test_under_asan_and_ubsan(tmp_path):
    if shutil.which("g++") is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("needs g++ and the HIP headers")
    exe = str(tmp_path / "pages_check")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-D__HIP_PLATFORM_AMD__",
                           "-I/opt/rocm/include", os.path.join(ROOT, "tests", "native", "pages_check.cpp"),
                           os.path.join(ROOT, "paper_2603_16104_amd", "csrc", "cache.cpp"), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0"))
    out = r.stdout + r.stderr
    assert r.returncode == 0 and " 0 failed checks" in out, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out and "LeakSanitizer" not in out, out[-4000:]


def test_copies_between_unlike_pools():
    a, wide, large = fake_pool(), fake_pool(page_size=32), fake_pool(num_kv_heads=4)
    for other in (wide, large):
        assert code(hkv.kv_pool_copy_pages, other, [0], a, [1], stream=0) == hkv.ESHAPE
        assert code(hkv.kv_pool_copy_pages, a, [0], other, [1], stream=0) == hkv.ESHAPE
    small = hkv.kv_pool_create(8, 2, hkv.FP32, 0x50000, 0x60000)
    assert code(hkv.kv_pool_copy_pages, small, [8], a, [9], stream=0) == hkv.ERANGE
    assert code(hkv.kv_pool_copy_pages, small, [7], a, [64], stream=0) == hkv.ERANGE
    assert code(hkv.kv_pool_copy_pages, small, [7], a, [-1], stream=0) == hkv.ERANGE
    assert code(hkv.kv_pool_copy_pages, small, [7], a, [5], [17], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, small, [7], a, [5], [-1], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, small, [7, 6], a, [5], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, small, [7], a, [5], [16, 16], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, small, [7, 7], a, [5, 6], stream=0) == hkv.EINVAL
    shared = hkv.kv_pool_alloc(small, 1)
    hkv.kv_pool_retain(small, shared)
    assert code(hkv.kv_pool_copy_pages, small, shared, a, [5], stream=0) == hkv.EINVAL
    hkv.kv_pool_copy_pages(small, [], a, [], stream=0)
    twin = fake_pool()  # another handle over the same buffers
    assert code(hkv.kv_pool_copy_pages, a, [3], twin, [3], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, a, [3, 4], a, [5, 3], stream=0) == hkv.EINVAL
    assert code(hkv.kv_pool_copy_pages, None, [3], a, [5], stream=0) == hkv.EINVAL
    for p in (a, wide, large, small, twin):
        hkv.kv_pool_destroy(p)


@pytest.mark.parametrize("page", [16, 128])
@pytest.mark.parametrize("release", [False, True])
def test_forks_of_full_pages_share_them(page, release):
    n = 12
    pool = hkv.kv_pool_create(n, 2, hkv.BF16, FAKE_K, FAKE_V, page_size=page)
    ids = hkv.kv_pool_alloc(pool, 6)  # 3, 0 and 2 pages, and one of somebody else
    out = hkv.kv_pool_fork(pool, ids[:5], [3 * page, 0, 2 * page], [2, 0, 1, 2], release, stream=0)
    assert list(out) == [*ids[3:5], *ids[:3], *ids[3:5]]
    base = 0 if release else 1
    assert counts(pool, 6) == [base + 1] * 3 + [base + 2] * 2 + [1]
    assert hkv.kv_pool_num_free(pool) == 6
    hkv.kv_pool_release(pool, out)
    if release:
        assert hkv.kv_pool_num_free(pool) == 11
        # a sequence that nobody goes on with
        rest = hkv.kv_pool_alloc(pool, 4)
        assert len(hkv.kv_pool_fork(pool, rest, [4 * page], [], True, stream=0)) == 0
        assert hkv.kv_pool_num_free(pool) == 11
    hkv.kv_pool_destroy(pool)


def test_a_fork_takes_the_last_page_over():
    """One fork a sequence that ends: nothing is copied, nothing is queued, whatever the last page holds."""
    pool = fake_pool(8)
    ids = hkv.kv_pool_alloc(pool, 5)
    out = hkv.kv_pool_fork(pool, ids, [20, 40], [1, 0], True, stream=0)
    assert list(out) == [*ids[2:], *ids[:2]] and counts(pool, 8) == [1] * 5 + [0] * 3
    hkv.kv_pool_destroy(pool)


def test_forks_refused():
    pool = fake_pool(8)
    ids = list(hkv.kv_pool_alloc(pool, 4))
    before = counts(pool, 8)
    for bad, want in [((ids[:2], [20], [1], False), hkv.ERANGE), ((ids[:2], [20], [-1], False), hkv.ERANGE), (([0, 9], [20], [0], False), hkv.ERANGE),
                      (([0, -1], [20], [0], False), hkv.ERANGE), (([0, 7], [20], [0], False), hkv.EINVAL), ((ids[:3], [20], [0], False), hkv.EINVAL),
                      ((ids[:2], [-20], [0], False), hkv.EINVAL), (([0, 0], [20], [0], True), hkv.EINVAL), (([0, 1, 0, 2], [32, 20], [0], True), hkv.EINVAL),
                      ((ids[:2], [20], [0] * 5, False), hkv.ENOMEM), ((ids, [20, 20], [0, 0, 0, 1, 1, 1, 1], True), hkv.ENOMEM)]:
        assert code(hkv.kv_pool_fork, pool, *bad, stream=0) == want, bad
        assert counts(pool, 8) == before and hkv.kv_pool_num_free(pool) == 4
    assert code(hkv.kv_pool_fork, None, [], [], [], stream=0) == hkv.EINVAL
    assert len(hkv.kv_pool_fork(pool, [], [], [], stream=0)) == 0
    hkv.kv_pool_destroy(pool)


def test_compaction_without_moves():
    pool = fake_pool(8)
    assert list(hkv.kv_pool_compact(pool, stream=0)) == [-1] * 8
    ids = hkv.kv_pool_alloc(pool, 8)
    hkv.kv_pool_retain(pool, ids[2:4])
    assert list(hkv.kv_pool_compact(pool, stream=0)) == list(range(8)) and counts(pool, 8) == [1, 1, 2, 2, 1, 1, 1, 1]
    hkv.kv_pool_release(pool, ids[[7, 5, 6]])  # the free list's order was 7, 5, 6
    assert list(hkv.kv_pool_compact(pool, stream=0)) == [0, 1, 2, 3, 4, -1, -1, -1]
    assert list(hkv.kv_pool_alloc(pool, 3)) == [5, 6, 7]
    L = hkv.lib()
    assert L.kv_pool_compact(pool, None, None) == hkv.EINVAL and L.kv_pool_compact(None, ids.ctypes.data, None) == hkv.EINVAL
    hkv.kv_pool_destroy(pool)

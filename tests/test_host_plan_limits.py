"""Decode plans of more partial results than their 32-bit numbers can name (addresses are never dereferenced here)."""
import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import FAKE_K, FAKE_V


@pytest.mark.parametrize("dtype,chunk,step", [(hkv.FP4_E2M1, 64, 64), (hkv.BF16, 16, 16), (hkv.FP8_E4M3, 16, 16)])
def test_partials_are_counted(dtype, chunk, step):
    """A long sequence in short items, beside many short ones: every row has as many places as the longest sequence has items."""
    tokens, hq, hk = 1 << 18, 16, 1
    parts = tokens // step
    fits = (2 ** 31 - 1) // (parts * hq)
    scales = () if dtype == hkv.BF16 else (0x30000, 0x40000)
    pool = hkv.kv_pool_create(tokens // 16 + 1, hk, dtype, FAKE_K, FAKE_V, *scales)
    pages = np.append(np.arange(tokens // 16), tokens // 16).astype(np.int32)
    nodes = [(-1, 0, tokens // 16, tokens), (-1, tokens // 16, 1, 1)]
    make = lambda n: hkv.hkv_decode_plan_create_ex(pool, nodes, pages, [0] + [1] * (n - 1), hq, hkv.PLAN_HOST_ONLY, leaf_chunk=chunk, max_rows=16, shared_chunk=2048)
    plan = make(fits)
    n_parts = fits * hq * parts
    assert hkv.hkv_decode_plan_workspace_bytes(plan) >= n_parts * 264
    hkv.hkv_decode_plan_destroy(plan)
    with pytest.raises(hkv.HkvError) as e:
        make(fits + 1)
    assert e.value.code == hkv.EINVAL and "partial results" in str(e.value)
    hkv.kv_pool_destroy(pool)

"""4-bit pools: items are as long as the caller's leaf_chunk and shared_chunk say, as over the other pools (addresses are never dereferenced here)."""
import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import FAKE_K, FAKE_V


@pytest.mark.parametrize("tokens", [640, 650, 2000])
@pytest.mark.parametrize("rows", ["few", "many"])
@pytest.mark.parametrize("chunk", [16, 48, 64, 80, 144, 640])
def test_chunks_are_the_callers(tokens, rows, chunk):
    n = 2 if rows == "few" else 20
    count = -(-tokens // 16)
    nodes = [(-1, 0, count, tokens)] + [(0, count + i, 1, 5) for i in range(n)]
    name = "leaf_chunk" if rows == "few" else "shared_chunk"
    found = {}
    for dtype, scales in ((hkv.FP4_E2M1, (0x30000, 0x40000)), (hkv.BF16, ())):
        pool = hkv.kv_pool_create(count + n, 2, dtype, FAKE_K, FAKE_V, *scales)
        plan = hkv.hkv_decode_plan_create_ex(pool, nodes, np.arange(count + n), list(range(1, n + 1)), 16, hkv.PLAN_HOST_ONLY, pack=1, **{name: chunk})
        items = hkv.hkv_decode_plan_items(plan)
        root = items[items[:, 7] == 0]
        found[dtype] = sorted({(int(i[6]), int(i[1])) for i in root})
        hkv.hkv_decode_plan_destroy(plan)
        hkv.kv_pool_destroy(pool)
    for items in found.values():
        assert max(n_tok for _, n_tok in items) <= chunk
        at = 0
        for begin, n_tok in items:
            assert begin == at
            at += n_tok
        assert at == tokens
    assert len(found[hkv.FP4_E2M1]) == len(found[hkv.BF16]) == -(-count // (chunk // 16))

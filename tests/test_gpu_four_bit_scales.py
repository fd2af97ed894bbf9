"""4-bit pools: softmax scales that are zero, next to it, or no number, in every form of decode."""
import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool
from test_gpu_four_bit import Forest, check_decode, decode, poison_unused_slots, queries
from test_gpu_four_bit_sums import KINDS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("scale", [0.0, -0.0, 2.0 ** -120, -2.0 ** -120, 2.0 ** -149, float("nan")])
def test_small_scales(kind, scale):
    """Queries of 2^95: scores that only a scale of nothing brings to nothing."""
    settings, rows = KINDS[kind]
    n = rows // 8
    f = Forest([(-1, 150)] + [(0, 5 + 3 * i) for i in range(n)], list(range(1, n + 1)), 16, seed=n)
    pool = Pool(f.n_pages, 1, seed=n)
    poison_unused_slots(pool, f)
    q = queries(n, 8) * 2.0 ** 95
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 8, shared_chunk=0 if kind == "paths" else 2048, **settings)
    assert (hkv.hkv_decode_plan_num_paths(plan) > 0) == (kind == "paths")
    out, lse = decode(plan, q, scale=scale)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    if scale != scale:
        assert np.isnan(out).all() and np.isnan(lse).all()
    else:
        check_decode(f, pool, q, out, lse, scale=scale)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()

"""4-bit pools: items of many steps (the operands of two steps on their way, page ids three ahead), and plans whose workgroups go out in an order of their own."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool
from test_gpu_four_bit import Forest, check_decode, decode, poison_unused_slots, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,rows,setting", [(n, 8, dict(pack=1, leaf_chunk=4096)) for n in (769, 1000, 1280, 2049)] +
                         [(n, 8, dict(pack=3, leaf_chunk=4096)) for n in (129, 192, 193, 257, 320, 1000)] +
                         [(n, 24, dict(max_rows=32, shared_chunk=2048)) for n in (513, 1025, 2000)] +
                         [(n, 48, dict(max_rows=64, shared_chunk=2048)) for n in (1025, 2000)] +
                         [(n, 96, dict(max_rows=128, shared_chunk=2048)) for n in (1025, 2000)])
def test_items_of_many_steps(tokens, rows, setting):
    n = rows // 8
    f = Forest([(-1, tokens)] + [(0, 3 + i) for i in range(n)], list(range(1, n + 1)) if n > 1 else [0], 16, seed=tokens)
    pool = Pool(f.n_pages, 2, seed=tokens)
    poison_unused_slots(pool, f)
    q = queries(n, 16)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 16, **setting)
    items = hkv.hkv_decode_plan_items(plan)
    root = items[items[:, 7] == 0]
    assert root[:, 1].max() == tokens and 8 * root[0, 4] == rows
    out, lse = decode(plan, q)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, out, lse)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("hq,hk,max_rows", [(64, 8, 32), (64, 8, 128), (15, 5, 48)])
def test_more_sets_than_places(hq, hk, max_rows):
    """Items of many rows and packed ones, several times what starts at once: the order of the plan, of which every item is part, against the plain one and 64 bits."""
    roots, each = 8, 38
    f = Forest([(-1, 512 + 16 * i) for i in range(roots)] + [(i % roots, 40 + i % 90) for i in range(roots * each)], list(range(roots, roots + roots * each)), 16, seed=hq)
    pool = Pool(f.n_pages, hk, seed=hq)
    poison_unused_slots(pool, f)
    q = queries(len(f.leaves), hq)
    results = []
    for interleave in (0, -1):
        plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, pack=3, max_rows=max_rows, shared_chunk=64, leaf_chunk=64, interleave=interleave)
        items = hkv.hkv_decode_plan_items(plan)
        many = items[:, 4] * (hq // hk) > 16
        assert many.sum() / 8 + (~many).sum() / 32 > 64 and many.any() and not many.all()
        results.append(decode(plan, q))
        hkv.hkv_decode_plan_destroy(plan)
    np.testing.assert_array_equal(results[0][0], results[1][0])
    np.testing.assert_array_equal(results[0][1], results[1][1])
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    some = np.arange(0, len(f.leaves), 41)
    f.leaves = [f.leaves[i] for i in some]
    check_decode(f, pool, q[torch.from_numpy(some).cuda()], results[0][0][some], results[0][1][some])
    pool.close()

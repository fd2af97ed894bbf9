"""4-bit pools: items that end inside a step of 64 tokens, in every form of items, below rows that see all of a node, part of it or single drafted tokens."""
import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool
from test_gpu_four_bit import Forest, check_decode, decode, poison_unused_slots, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("setting", [dict(max_rows=16, pack=1), dict(max_rows=16, pack=3), dict(max_rows=32), dict(max_rows=64), dict(max_rows=128)])
@pytest.mark.parametrize("chunk", [16, 48, 80, 144])
def test_shared_and_own_tokens(setting, chunk):
    f = Forest([(-1, 500)] + [(0, 30 + 21 * i) for i in range(16)], list(range(1, 17)) + [0] * 4, 16, seed=chunk)
    pool = Pool(f.n_pages, 2, seed=1)
    poison_unused_slots(pool, f)
    q = queries(20, 16)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 16, leaf_chunk=chunk, shared_chunk=chunk, **setting)
    assert hkv.hkv_decode_plan_items(plan)[:, 1].max() <= chunk
    out, lse = decode(plan, q)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, out, lse)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("setting", [dict(max_rows=16, pack=1), dict(max_rows=16, pack=3), dict(max_rows=32), dict(max_rows=64), dict(max_rows=128)])
@pytest.mark.parametrize("chunk", [16, 48, 80])
@pytest.mark.parametrize("hq,T,tree", [(16, 8, True), (16, 8, False), (2, 21, True), (1, 64, True), (4, 5, False)])
def test_drafted_tokens(setting, chunk, hq, T, tree):
    """A request's drafts are the end of its own node, and reach over the border of two of its items."""
    f = Forest([(-1, 70)] + [(0, T + n) for n in (0, 9, 16, 40, 61)], [1, 2, 3, 4, 5], 16, seed=T)
    pool = Pool(f.n_pages, 1, seed=2)
    poison_unused_slots(pool, f)
    q = queries(5 * T, hq)
    visible = None
    if tree:
        rng = np.random.default_rng(T)
        masks = []
        for t in range(T):
            masks.append((masks[rng.integers(0, t)] if t and rng.random() < 0.8 else 0) | 1 << t)
        visible = np.asarray(masks * 5, dtype=np.uint64)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, tokens_per_req=T, visible=visible, leaf_chunk=chunk, shared_chunk=chunk, **setting)
    out, lse = decode(plan, q)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, out, lse, T, visible)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


def test_a_growing_plan():
    """The last item of a leaf grows over the chunk's end; the ones in front of it end inside a step."""
    f = Forest([(-1, 100), (0, 75), (0, 90)], [1, 2], 16, extra=6)
    pool = Pool(f.n_pages, 2, poison=False)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 8, reserve_tokens=40, leaf_chunk=48, shared_chunk=48)
    fresh = list(f.unused)
    for step in range(40):
        new = np.full(2, -1, dtype=np.int32)
        for r in range(2):
            if f.n_tokens[r + 1] % 16 == 0:
                new[r] = fresh.pop()
                f.pages[r + 1] = np.append(f.pages[r + 1], new[r])
            f.n_tokens[r + 1] += 1
        hkv.hkv_decode_plan_append(plan, new)
        if step % 13 == 0 or step == 39:
            q = queries(2, 8, seed=step)
            check_decode(f, pool, q, *decode(plan, q))
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()

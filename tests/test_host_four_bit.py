"""4-bit pools on the host: what their calls refuse before anything is queued, and how decode plans cut a forest (addresses are never
dereferenced here)."""
import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import FAKE_K, FAKE_V

A = 0x100000


def pool_of(num_pages=64, heads=2, page=16):
    return hkv.kv_pool_create(num_pages, heads, hkv.FP4_E2M1, FAKE_K, FAKE_V, 0x30000, 0x40000, page_size=page)


def code(f, *args, **kw):
    with pytest.raises(hkv.HkvError) as e:
        f(*args, **kw)
    return e.value.code


def test_create():
    assert code(hkv.kv_pool_create, 8, 2, hkv.FP4_E2M1, FAKE_K, FAKE_V) == hkv.ESHAPE
    assert code(hkv.kv_pool_create, 8, 2, hkv.FP4_E2M1, FAKE_K, FAKE_V, 0x30000, None) == hkv.ESHAPE
    assert code(hkv.kv_pool_create, 8, 2, hkv.FP4_E2M1, FAKE_K, FAKE_V, 0x30008, 0x40000) == hkv.EINVAL
    assert code(hkv.kv_pool_create, 8, 2, hkv.FP4_E2M1, FAKE_K, FAKE_V, 0x30000, 0x40004) == hkv.EINVAL
    assert code(hkv.kv_pool_create, 8, 2, hkv.FP4_E2M1, FAKE_K + 8, FAKE_V, 0x30000, 0x40000) == hkv.EINVAL
    for page in (16, 32, 64, 128):
        pool = pool_of(page=page)
        assert hkv.kv_pool_page_size(pool) == page and hkv.lib().kv_pool_num_pages(pool) == 64
        hkv.kv_pool_destroy(pool)
    assert hkv.lib().kv_pool_num_pages(None) == hkv.EINVAL


def test_stores():
    pool = pool_of(page=32)
    assert code(hkv.kv_pool_write, pool, [64], 0, 32, A, A, 0) == hkv.ERANGE
    assert code(hkv.kv_pool_write, pool, [1], 32, 1, A, A, 0) == hkv.EINVAL
    assert code(hkv.kv_pool_write, pool, [1], 0, 1, None, A, 0) == hkv.EINVAL
    assert code(hkv.kv_pool_append, pool, [1], [32], A, A, 0) in (hkv.EINVAL, hkv.ERANGE)
    assert code(hkv.kv_pool_append, pool, [1, 1], [3, 5], A, A, 0) == hkv.EINVAL     # one block twice
    assert code(hkv.kv_pool_append, pool, [-1], [3], A, A, 0) == hkv.ERANGE
    hkv.kv_pool_destroy(pool)


def test_plans():
    pool = pool_of()
    nodes, pages = [(-1, 0, 2, 32), (0, 2, 1, 9), (0, 3, 1, 16)], [0, 1, 2, 3]
    assert code(hkv.hkv_decode_plan_create, pool, nodes, pages, [1, 2], 8, hkv.PLAN_HOST_ONLY | hkv.PLAN_FP8_MATRIX) == hkv.ESHAPE
    assert code(hkv.hkv_decode_plan_create, pool, nodes, pages, [1, 2], 34, hkv.PLAN_HOST_ONLY) == hkv.ESHAPE
    for bad in (15, 129):
        assert code(hkv.hkv_decode_plan_create_ex, pool, nodes, pages, [1, 2], 8, hkv.PLAN_HOST_ONLY, max_rows=bad) == hkv.EINVAL
    assert code(hkv.hkv_decode_plan_create, pool, nodes, pages, [1, 2], 3, hkv.PLAN_HOST_ONLY) == hkv.ESHAPE
    assert code(hkv.hkv_decode_plan_create, pool, nodes, [0, 1, 2, 64], [1, 2], 8, hkv.PLAN_HOST_ONLY) == hkv.ERANGE
    plan = hkv.hkv_decode_plan_create(pool, nodes, pages, [1, 2], 8, hkv.PLAN_HOST_ONLY)
    assert hkv.hkv_decode_plan_num_paths(plan) == 2 and hkv.hkv_decode_plan_num_tile_items(plan) == 0 and not hkv.hkv_decode_plan_is_fused(plan)
    for other in (hkv.hkv_decode_plan_create_ex(pool, nodes, pages, [1, 2], 8, hkv.PLAN_HOST_ONLY, pack=1),        # a setting of the items, a plan that grows
                  hkv.hkv_decode_plan_create_growing(pool, nodes, pages, [1, 2], 8, 5, hkv.PLAN_HOST_ONLY)):
        assert hkv.hkv_decode_plan_num_paths(other) == 0
        hkv.hkv_decode_plan_destroy(other)
    assert code(hkv.hkv_decode_plan_track_weights, plan) == hkv.ESHAPE
    assert code(hkv.hkv_decode_plan_store, plan, hkv.qkv_rows(q=A, k=A, v=A, q_out=2 * A, rotary_dim=128, inv_freq=A), 0) == hkv.ESHAPE
    assert code(hkv.attn_decode_plan_run, plan, A, 0.1, A, A, A, 1 << 20, 0) == hkv.EINVAL  # a host-only plan
    hkv.hkv_decode_plan_destroy(plan)
    plan = hkv.hkv_prefill_plan_create(pool, [0, 5], [[0, 1]], [20], 8, hkv.PLAN_HOST_ONLY)
    assert hkv.hkv_prefill_plan_workspace_bytes(plan) >= 2 * 2 * 2 * 16 * 128 * 2
    assert code(hkv.hkv_prefill_plan_store, plan, hkv.qkv_rows(q=A, k=A, v=A, q_out=2 * A, rotary_dim=128, inv_freq=A), 0) == hkv.ESHAPE
    hkv.hkv_prefill_plan_destroy(plan)
    assert code(hkv.kv_pool_evict, pool, [0, 1], [32], [2], [16], 4, 4, A, None, stream=0) == hkv.ESHAPE
    hkv.kv_pool_destroy(pool)


def random_forest(rng, page):
    """Nodes of 0 to some hundred tokens, any of them inside a page, requests anywhere below."""
    parent, tokens = [], []
    for v in range(rng.integers(1, 12)):
        parent.append(int(rng.integers(-1, v)) if v else -1)
        tokens.append(int(rng.choice([0, 1, 15, 16, 17, 64, 100, int(rng.integers(1, 3000))])))
    leaves = [int(x) for x in rng.integers(0, len(parent), size=rng.choice([1, 3, 40, 130]))]
    for v in set(leaves):
        depth_tokens, u = 0, v
        while u >= 0:
            depth_tokens, u = depth_tokens + tokens[u], parent[u]
        if depth_tokens == 0:
            tokens[v] = 1
    nodes, at = [], 0
    for p, n in zip(parent, tokens):
        count = (n + page - 1) // page
        nodes.append((p, at, count, n))
        at += count
    return nodes, at, leaves


SETTINGS = [{}, dict(max_rows=16), dict(max_rows=64, leaf_chunk=64), dict(shared_chunk=128), dict(pack=1), dict(pack=3), dict(leaf_chunk=16, shared_chunk=2048, pack=3),
            dict(max_rows=32, shared_chunk=1024), dict(max_rows=128)]


@pytest.mark.parametrize("hq,hk,T", [(8, 2, 1), (32, 8, 1), (16, 1, 1), (5, 1, 1), (40, 8, 8), (4, 4, 16)])
@pytest.mark.parametrize("page", [16, 64])
def test_every_row_reads_every_token_once(hq, hk, T, page):
    """Items cover each (request, KV head, token) once; a request's partials take the slots from 0 on without a gap, one a chunk."""
    G = hq // hk  # (rows are those of the drafted tokens, one after the other)
    for seed in range(2 * len(SETTINGS)):
        rng = np.random.default_rng([seed, hq, page, T])
        nodes, n_pages, leaves = random_forest(rng, page)
        if T > 1:  # every request a leaf of its own that holds its drafts
            parents = {n[0] for n in nodes}
            ends = [v for v in range(len(nodes)) if v not in parents]
            leaves = [v for v in ends]
            fixed, at = [], 0
            for v, (p, _, _, n) in enumerate(nodes):
                n = max(n, T) if v in ends else n
                fixed.append((p, at, (n + page - 1) // page, n))
                at += (n + page - 1) // page
            nodes, n_pages = fixed, at
        pool = pool_of(max(n_pages, 1), hk, page)
        setting = SETTINGS[seed % len(SETTINGS)]
        kw = dict(tokens_per_req=T) if T > 1 else {}
        plan = hkv.hkv_decode_plan_create_ex(pool, nodes, np.arange(n_pages), leaves, hq, hkv.PLAN_HOST_ONLY, **setting, **kw)
        block, start = np.cumsum([0] + [-(-n[3] // 16) for n in nodes]), []
        for p, _, _, n in nodes:
            start.append(0 if p < 0 else start[p] + nodes[p][3])
        under = [[] for _ in nodes]
        leaves = np.repeat(leaves, T).tolist()
        for r, v in enumerate(leaves):
            while v >= 0:
                under[v].append(r)
                v = nodes[v][0]
        base = np.cumsum([0] + [len(u) for u in under])
        total = [start[v] + nodes[v][3] for v in leaves]
        seen = [np.zeros((hk, n), dtype=np.int32) for n in total]
        slots = [set() for _ in leaves]
        items = hkv.hkv_decode_plan_items(plan)
        limit = max(setting.get("max_rows", 128), G)
        for off, n_tok, head, req_off, n_req, slot, tok_begin, node in items:
            assert n_tok >= 1 and tok_begin % 16 == 0 and tok_begin + n_tok <= nodes[node][3]
            assert tok_begin + n_tok == nodes[node][3] or n_tok % 64 == 0 or "leaf_chunk" in setting
            assert off == block[node] + tok_begin // 16
            assert n_req >= 1 and n_req * G <= limit
            few = len(under[node]) * G <= 16
            chunk = setting.get("leaf_chunk" if few else "shared_chunk")
            assert chunk is None or n_tok <= max(64, chunk)
            order = under[node]
            at = req_off - base[node]
            assert 0 <= at and at + n_req <= len(order)
            for r in order[at: at + n_req]:
                seen[r][head, start[node] + tok_begin: start[node] + tok_begin + n_tok] += 1
                assert (head, slot) not in slots[r]
                slots[r].add((head, slot))
        for r in range(len(leaves)):
            assert (seen[r] == 1).all()
            for h in range(hk):
                mine = sorted(s for x, s in slots[r] if x == h)
                assert mine == list(range(len(mine)))
        hkv.hkv_decode_plan_destroy(plan)
        hkv.kv_pool_destroy(pool)


def test_the_same_forest_is_cut_the_same_way():
    rng = np.random.default_rng(4)
    nodes, n_pages, leaves = random_forest(rng, 16)
    pool = pool_of(max(n_pages, 1))
    plans = [hkv.hkv_decode_plan_create(pool, nodes, np.arange(n_pages), leaves, 8, hkv.PLAN_HOST_ONLY) for _ in range(2)]
    assert np.array_equal(*(hkv.hkv_decode_plan_items(p) for p in plans))
    for p in plans:
        hkv.hkv_decode_plan_destroy(p)
    hkv.kv_pool_destroy(pool)


@pytest.mark.parametrize("heads", [3, 11, 513, 700])
@pytest.mark.parametrize("setting", [dict(pack=1), dict(pack=3), dict(interleave=-1, pack=1)])
def test_any_number_of_heads(heads, setting):
    """Sets of items are whole sets of KV heads, however many those are; every item is listed once."""
    nodes = [(-1, 0, 4, 64)] + [(0, 4 + i, 1, 9) for i in range(20)]
    pool = pool_of(24, heads)
    plan = hkv.hkv_decode_plan_create_ex(pool, nodes, np.arange(24), list(range(1, 21)), heads, hkv.PLAN_HOST_ONLY, **setting)
    items = hkv.hkv_decode_plan_items(plan)
    key = items[:, [7, 6, 2, 3]]
    assert len(np.unique(key, axis=0)) == len(items) and (np.bincount(items[:, 2], minlength=heads) == len(items) // heads).all()
    hkv.hkv_decode_plan_destroy(plan)
    hkv.kv_pool_destroy(pool)

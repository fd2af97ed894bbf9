"""4-bit pools: stores against the format's definition, bit for bit; decode and prefill attention against 64-bit attention over the same values."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool, attention, blocks_of, check_rows, of_sequence, quantised

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))


def rows_of(n, heads, seed, spread=True):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(n, heads, 128, device="cuda", generator=g)
    if spread:  # groups of very different size, some of them all zeros
        x *= torch.exp2(torch.randint(-30, 30, (n, heads, 4, 1), device="cuda", generator=g).float()).expand(-1, -1, -1, 32).reshape(n, heads, 128)
        x *= (torch.rand(n, heads, 4, 1, device="cuda", generator=g) > 0.1).expand(-1, -1, -1, 32).reshape(n, heads, 128)
    return x.to(torch.bfloat16)


def f64(t):
    return t.float().double().cpu().numpy()


def check_stored(pool, before, places, k, v):
    """Places (block, slot) hold what rows k, v [n][heads][128] are in 4 bits, everything else what it held."""
    kc, ks, vc, vs = before
    for i, (b, t) in enumerate(places):
        kc[b, :, t], ks[b, :, t], _ = quantised(k[i])
        vc[b, :, t], vs[b, :, t], _ = quantised(v[i])
    for got, want in zip(pool.read(), (kc, ks, vc, vs)):
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("heads,page,first,n", [(8, 16, 0, 1), (2, 16, 3, 1), (2, 16, 5, 40), (8, 16, 0, 64), (1, 32, 31, 2), (3, 64, 17, 100), (8, 128, 127, 130), (2, 16, 0, 17000)])
def test_write(heads, page, first, n):
    n_pages = -(-(first + n) // page)
    pool = Pool(n_pages + 3, heads, page, seed=n)
    pages = np.random.default_rng(n).permutation(n_pages + 3)[:n_pages].astype(np.int32)
    k, v = rows_of(n, heads, 1), rows_of(n, heads, 2)
    before = pool.read()
    hkv.kv_pool_write(pool.handle, pages, first, n, k, v)
    b = blocks_of(pages, page)
    at = first + np.arange(n)
    check_stored(pool, before, list(zip(b[at // 16], at % 16)), f64(k), f64(v))
    pool.close()


@pytest.mark.parametrize("heads,page,n", [(8, 16, 1), (2, 16, 7), (3, 32, 16), (8, 64, 256), (2, 128, 257), (1, 16, 1000)])
def test_append(heads, page, n):
    pool = Pool(n + 5, heads, page, seed=n)
    rng = np.random.default_rng(n)
    pages, slots = rng.permutation(n + 5)[:n].astype(np.int32), rng.integers(0, page, n).astype(np.int32)
    k, v = rows_of(n, heads, 3), rows_of(n, heads, 4)
    before = pool.read()
    hkv.kv_pool_append(pool.handle, pages, slots, k, v)
    check_stored(pool, before, [(p * (page // 16) + s // 16, s % 16) for p, s in zip(pages, slots)], f64(k), f64(v))
    pool.close()


def test_write_borders():
    """Ties, numbers beyond 6, the smallest and largest scales, signed zeros, infinities and NaN."""
    x = np.zeros((6, 1, 128), dtype=np.float32)
    x[0, 0, :32] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -0.25, -0.75, -1.25, -1.75, -2.5, -3.5, -5, 6, 7, 7.96875, -7.96875, 0.0, -0.0, 0.251953125, 0.2490234375, 1, 2, 3, 1.5, -6, -1, 4.96875, 5.03125, 0.5]
    x[1, 0] = x[0, 0, np.arange(128) % 32] * 2.0 ** -124
    x[2, 0] = x[0, 0, np.arange(128) % 32] * 2.0 ** 125
    x[3, 0] = 2.0 ** -133  # bf16's smallest
    x[4, 0, 5], x[4, 0, 6], x[4, 0, 7] = np.inf, -np.inf, 3e38
    x[5, 0, :32] = 3
    x[5, 0, 9] = np.nan
    k = torch.from_numpy(x).to(torch.bfloat16).cuda()
    finite = f64(k)
    finite[4] = 0
    finite[5, 0, 9] = 0
    pool = Pool(1, 1, seed=1)
    hkv.kv_pool_write(pool.handle, [0], 0, 6, k, k)
    kc, ks, vc, vs = pool.read()
    want, want_s, _ = quantised(finite)
    for c, s in ((kc, ks), (vc, vs)):
        c, s = c[0, 0, :6].copy(), s[0, 0, :6]
        np.testing.assert_array_equal(s[[0, 1, 2, 3, 5]], want_s[[0, 1, 2, 3, 5], 0])
        assert s[4, 0] == 252 and list(c[4, 5:8]) == [7, 15, 7] and not (c[4, 8:32] & 7).any()  # 3e38 is held as 6 * 2^125
        assert c[5, 9] & 7 == 7
        c[5, 9] = 0
        np.testing.assert_array_equal(c[[0, 1, 2, 3, 5]], want[[0, 1, 2, 3, 5], 0])
    pool.close()


class Forest:
    """nodes [(parent, tokens)], requests [node]; pages drawn at random."""

    def __init__(self, nodes, leaves, page, seed=0, extra=2):
        self.n_tokens, self.parent, self.leaves, self.page = [n for _, n in nodes], [p for p, _ in nodes], leaves, page
        count = [-(-n // page) for n in self.n_tokens]
        self.n_pages = sum(count) + extra
        order = np.random.default_rng(seed).permutation(self.n_pages).astype(np.int32)
        self.pages, self.nodes, at = [], [], 0
        for (p, n), c in zip(nodes, count):
            self.pages.append(order[at: at + c])
            self.nodes.append((p, at, c, n))
            at += c
        self.node_pages = order[:at]
        self.unused = order[at:]

    def path(self, v):
        out = []
        while v >= 0:
            out.append(v)
            v = self.parent[v]
        return out[::-1]

    def keys(self, values, leaf):
        return np.concatenate([of_sequence(values, self.pages[v], self.page, self.n_tokens[v]) for v in self.path(leaf)])


def poison_unused_slots(pool, forest):
    """Scale bytes of 255 behind every node's last token and in pages that no node has."""
    dead = np.ones((pool.blocks, 16), dtype=bool)
    for v in range(len(forest.nodes)):
        b, t = blocks_of(forest.pages[v], forest.page), np.arange(forest.n_tokens[v])
        dead[b[t // 16], t % 16] = False
    mask = torch.from_numpy(dead).cuda()[:, None, None, :].expand(-1, pool.heads, 4, -1)
    pool.k_scale.view(pool.blocks, pool.heads, 4, 16)[mask] = 255
    pool.v_scale.view(pool.blocks, pool.heads, 4, 16)[mask] = 255


def decode(plan, q, static=False, scale=SCALE):
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:2], float("nan"), device="cuda")
    need = hkv.hkv_decode_plan_workspace_bytes(plan)
    if static:
        hkv.attn_decode_plan_run_static(plan, q, scale, out, lse)
    else:
        ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
        hkv.attn_decode_plan_run(plan, q, scale, out, lse, ws, need)
        assert (ws[need:] == 255).all()
    torch.cuda.synchronize()
    return f64(out), lse.double().cpu().numpy()


def check_decode(forest, pool, q, out, lse, T=1, visible=None, scale=SCALE):
    k, v = pool.values()
    refs = []
    for r, leaf in enumerate(forest.leaves):
        kk, vv = forest.keys(k, leaf), forest.keys(v, leaf)
        n = len(kk)
        for t in range(T):
            seen = np.ones(n, dtype=bool)
            if T > 1 or visible is not None:
                mask = int(visible[r * T + t]) if visible is not None else (1 << (t + 1)) - 1
                seen[n - T:] = [mask >> j & 1 for j in range(T)]
            refs.append(attention(f64(q)[r * T + t], kk, vv, scale, seen))
    check_rows(out, lse, tuple(np.stack([x[i] for x in refs]) for i in range(4)))


def queries(n, hq, seed=9):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(n, hq, 128, device="cuda", generator=g) * 2).to(torch.bfloat16)


FORESTS = [
    # (query heads, KV heads, page, nodes, leaves)
    (1, 1, 16, [(-1, 1)], [0]),
    (8, 2, 16, [(-1, 256), (0, 17), (0, 49), (0, 33), (0, 1)], [1, 2, 3, 4]),
    (32, 8, 16, [(-1, 63), (-1, 64), (-1, 65), (-1, 129), (-1, 1000)], [0, 1, 2, 3, 4]),
    (16, 1, 32, [(-1, 300), (0, 70), (0, 40)], [1, 1, 2, 0]),                 # several requests on a node, one that ends above
    (40, 8, 64, [(-1, 130), (0, 20), (1, 7), (1, 90), (2, 64)], [3, 4]),        # nodes that end inside a page, with children
    (5, 1, 16, [(-1, 0), (0, 30), (0, 0)], [1, 2, 0]),                         # requests that see nothing
    (48, 3, 128, [(-1, 500), (0, 129)], [1, 1]),
    (32, 8, 16, [(-1, 700)] + [(0, 30 + i) for i in range(21)], list(range(1, 22))),   # 84 rows a head: more than an item's
    (12, 4, 16, [(-1, 2048), (-1, 17)] + [(i % 2, 5 * i + 1) for i in range(12)], list(range(2, 14))),
]


@pytest.mark.parametrize("case", range(len(FORESTS)))
def test_decode(case):
    hq, hk, page, nodes, leaves = FORESTS[case]
    f = Forest(nodes, leaves, page, seed=case)
    pool = Pool(f.n_pages, hk, page, seed=case)
    poison_unused_slots(pool, f)
    q = queries(len(leaves), hq)
    plans = [hkv.hkv_decode_plan_create(pool.handle, f.nodes, f.node_pages, leaves, hq),
             hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, leaves, hq, leaf_chunk=64, shared_chunk=128, max_rows=16)]
    results = [decode(plan, q, static) for plan in plans for static in (False, True)]
    pool.k_scale[pool.k_scale == 255] = 127  # (for the reference: those slots count for nothing)
    pool.v_scale[pool.v_scale == 255] = 127
    for out, lse in results:
        check_decode(f, pool, q, out, lse)
    for i in (0, 2):
        np.testing.assert_array_equal(results[i][0], results[i + 1][0])
    for plan in plans:
        hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("hq,hk,T,prefix,own,tree", [(8, 2, 2, 100, 5, False), (32, 8, 16, 64, 70, False), (40, 8, 8, 500, 33, False), (4, 4, 64, 130, 64, True), (32, 8, 21, 77, 90, True), (16, 1, 5, 0, 5, True)])
def test_decode_drafts(hq, hk, T, prefix, own, tree):
    f = Forest([(-1, prefix)] + [(0, own + 3 * i) for i in range(3)], [1, 2, 3], 16, seed=T)
    pool = Pool(f.n_pages, hk, seed=T)
    q = queries(3 * T, hq)
    visible = None
    if tree:
        rng = np.random.default_rng(T)
        visible = []
        for _ in range(3):
            masks = []
            for t in range(T):  # a random ancestor's mask, and itself
                masks.append((masks[rng.integers(0, t)] if t and rng.random() < 0.8 else 0) | 1 << t)
            visible += masks
        visible = np.asarray(visible, dtype=np.uint64)
        plan = hkv.hkv_decode_plan_create_tree(pool.handle, f.nodes, f.node_pages, f.leaves, T, visible, hq)
    else:
        plan = hkv.hkv_decode_plan_create_multi(pool.handle, f.nodes, f.node_pages, f.leaves, T, hq)
    out, lse = decode(plan, q)
    check_decode(f, pool, q, out, lse, T, visible)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("setting", [{}, dict(max_rows=16), dict(max_rows=128, pack=3)])
def test_decode_rows_of_q(setting):
    """q_rows: the plan's rows lie among others."""
    f = Forest([(-1, 90), (0, 40), (0, 17)], [1, 2], 16)
    pool = Pool(f.n_pages, 2)
    q = queries(7, 8)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 8, q_rows=np.asarray([5, 2], dtype=np.int32), **setting)
    out, lse = decode(plan, q)
    others = [0, 1, 3, 4, 6]
    assert np.isnan(out[others]).all() and np.isnan(lse[others]).all()
    check_decode(f, pool, q[[5, 2]], out[[5, 2]], lse[[5, 2]])
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("hq,hk,page,prefix,own,n_req,T", [(8, 2, 16, 256, 49, 4, 1), (1, 1, 16, 0, 1, 1, 1), (32, 8, 32, 33, 20, 40, 1), (8, 2, 16, 736, 30, 2, 1), (64, 8, 16, 1200, 30, 16, 1), (40, 8, 64, 65, 100, 3, 2), (4, 2, 16, 129, 16, 5, 16), (16, 1, 128, 200, 3, 2, 3)])
def test_whole_paths(hq, hk, page, prefix, own, n_req, T):
    """Small steps: a workgroup a leaf and KV head, with 8 wavefronts or (many leaves) 4; nodes that end anywhere, a leaf of two requests, one above others."""
    f = Forest([(-1, prefix), (0, 7)] + [(i % 2, own + i) for i in range(n_req)], list(range(2, 2 + n_req)) + ([2, 1] if T == 1 else []), page, seed=3)
    pool = Pool(f.n_pages, hk, page, seed=5)
    poison_unused_slots(pool, f)
    q = queries(len(f.leaves) * T, hq)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, tokens_per_req=T)
    assert hkv.hkv_decode_plan_num_paths(plan) > 0
    results = [decode(plan, q, static) for static in (False, True)]
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, *results[0], T)
    for a, b in zip(*results):
        np.testing.assert_array_equal(a, b)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


ITEM_ROWS = [(32, 17), (32, 32), (64, 33), (64, 56), (64, 64), (128, 65), (128, 96), (128, 100), (128, 128)]


@pytest.mark.parametrize("max_rows,rows", ITEM_ROWS)
@pytest.mark.parametrize("tokens", [1, 16, 63, 64, 65, 200, 256, 500])
def test_items_of_many_rows(max_rows, rows, tokens):
    """A node of so many tokens under items of each kind; requests of one token of their own, some of none."""
    group = next(g for g in (16, 8, 5, 4, 3, 1) if rows % g == 0)
    n = rows // group
    f = Forest([(-1, tokens)] + [(0, 1 if i % 3 else 0) for i in range(n)], list(range(1, n + 1)), 16, seed=tokens)
    pool = Pool(f.n_pages, 2, seed=rows)
    poison_unused_slots(pool, f)
    q = queries(n, 2 * group)
    q[0] *= 4  # (scores that leave the first step's reference)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 2 * group, max_rows=max_rows, shared_chunk=2048)
    items = hkv.hkv_decode_plan_items(plan)
    assert group * items[items[:, 7] == 0][0, 4] == rows and items[items[:, 7] == 0][0, 1] == tokens
    out, lse = decode(plan, q)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, out, lse)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("max_rows", [16, 32, 64, 128])
@pytest.mark.parametrize("hq,hk,T,tree", [(16, 1, 8, True), (32, 2, 5, False), (8, 1, 16, False)])
def test_masks_in_items_of_many_rows(max_rows, hq, hk, T, tree):
    """Drafted tokens in the only node: its items have all of a request's rows, some of which see nothing of an item."""
    f = Forest([(-1, T + 60), (-1, 130), (-1, T)], [0, 1, 2], 16, seed=2)
    pool = Pool(f.n_pages, hk, seed=4)
    poison_unused_slots(pool, f)
    q = queries(3 * T, hq)
    visible = None
    if tree:
        rng = np.random.default_rng(0)
        parent = [-1] + [int(rng.integers(0, j)) for j in range(1, T)]
        one = []
        for j in range(T):
            m, u = 0, j
            while u >= 0:
                m, u = m | 1 << u, parent[u]
            one.append(m)
        visible = np.array(one * 3, dtype=np.uint64)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, tokens_per_req=T, visible=visible, max_rows=max_rows, shared_chunk=64)
    out, lse = decode(plan, q)
    pool.k_scale[pool.k_scale == 255] = 127
    pool.v_scale[pool.v_scale == 255] = 127
    check_decode(f, pool, q, out, lse, T, visible)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("max_rows,rows", [(16, 16), (32, 32), (64, 64), (128, 128)])
def test_references_that_move(max_rows, rows):
    """Scores that grow from step to step by more than a reference's slack, and a first step of the lowest: weights of the last one count alone."""
    f = Forest([(-1, 512)], [0] * (rows // 16), 16)
    pool = Pool(f.n_pages, 1, seed=6)
    b = f.pages[0]
    step = np.repeat(np.arange(8), 4)  # K's values grow by 4 a step
    for i, page in enumerate(b):
        pool.k_scale.view(pool.blocks, 1, 64)[int(page)] = int(121 + step[i])
    pool.k.fill_(0x22)  # ones
    q = torch.ones(rows // 16, 16, 128, dtype=torch.bfloat16, device="cuda")
    q[:, 1::2] = -1
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 16, max_rows=max_rows, shared_chunk=512)
    out, lse = decode(plan, q, scale=4.0)
    check_decode(f, pool, q, out, lse, scale=4.0)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("scale", [0.0, -0.05, 3.0])
def test_decode_scales(scale):
    f = Forest([(-1, 200), (0, 40), (0, 90)], [1, 2], 16)
    pool = Pool(f.n_pages, 2)
    q = queries(2, 8)
    plan = hkv.hkv_decode_plan_create(pool.handle, f.nodes, f.node_pages, f.leaves, 8)
    out, lse = decode(plan, q, scale=scale)
    check_decode(f, pool, q, out, lse, scale=scale)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


def test_decode_row_with_nan():
    """A NaN in a query: that row and head alone."""
    f = Forest([(-1, 200), (0, 40), (0, 90)], [1, 2], 16)
    pool = Pool(f.n_pages, 2)
    q = queries(2, 8)
    plan = hkv.hkv_decode_plan_create(pool.handle, f.nodes, f.node_pages, f.leaves, 8)
    clean = decode(plan, q)
    q[1, 3, 77] = float("nan")
    out, lse = decode(plan, q)
    assert np.isnan(out[1, 3]).all() and np.isnan(lse[1, 3])
    out[1, 3], lse[1, 3] = clean[0][1, 3], clean[1][1, 3]
    np.testing.assert_array_equal(out, clean[0])
    np.testing.assert_array_equal(lse, clean[1])
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("max_rows", [16, 32, 64, 128])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_rows_that_are_not_finite(value, max_rows):
    """That row and head alone have no result, in items of every kind; an infinity times a key of both signs is no number either."""
    n = max_rows // 4
    f = Forest([(-1, 200)] + [(0, 5)] * n, list(range(1, n + 1)), 16)
    pool = Pool(f.n_pages, 2)
    q = queries(n, 8)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 8, max_rows=max_rows, shared_chunk=256)
    clean = decode(plan, q)
    q[1, 3, 77] = value
    out, lse = decode(plan, q)
    assert np.isnan(out[1, 3]).all() and np.isnan(lse[1, 3])
    out[1, 3], lse[1, 3] = clean[0][1, 3], clean[1][1, 3]
    np.testing.assert_array_equal(out, clean[0])
    np.testing.assert_array_equal(lse, clean[1])
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("n_req,page,large", [(3, 16, 0), (3, 32, 1), (260, 16, 0)])
def test_growing_plan(n_req, page, large):
    """Tokens are stored and decoded step by step, over the border of pages."""
    hq, hk, steps = 8, 2, 20
    f = Forest([(-1, 48)] + [(0, 1 + i % 31) for i in range(n_req)], list(range(1, n_req + 1)), page, extra=2 * n_req)
    pool = Pool(f.n_pages, hk, page, poison=False)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, reserve_tokens=steps, large_batch_updates=large)
    fresh = list(f.unused)
    for step in range(steps):
        new = np.full(n_req, -1, dtype=np.int32)
        for r in range(n_req):
            if f.n_tokens[r + 1] % page == 0:
                new[r] = fresh.pop()
                f.pages[r + 1] = np.append(f.pages[r + 1], new[r])
            f.n_tokens[r + 1] += 1
        k, v = rows_of(n_req, hk, 100 + step, spread=False), rows_of(n_req, hk, 200 + step, spread=False)
        hkv.hkv_decode_plan_append_tokens(plan, new, k, v)
        if step in (0, 7, steps - 1):
            q = queries(n_req, hq, seed=step)
            out, lse = decode(plan, q)
            if n_req > 16:  # (the reference takes long: some rows)
                some = np.arange(0, n_req, 37)
                leaves, f.leaves = f.leaves, [f.leaves[i] for i in some]
                check_decode(f, pool, q[torch.from_numpy(some).cuda()], out[some], lse[some])
                f.leaves = leaves
            else:
                check_decode(f, pool, q, out, lse)
    kv, vv = pool.values()
    last = of_sequence(kv, f.pages[2], page, f.n_tokens[2])[-1]
    np.testing.assert_array_equal(last, quantised(f64(k)[1])[2])
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("hq,hk,page,lens", [(8, 2, 16, [(0, 1)]), (32, 8, 16, [(64, 70), (0, 33), (100, 1)]), (40, 8, 64, [(300, 100), (128, 64)]), (16, 1, 128, [(1000, 40)])])
def test_prefill(hq, hk, page, lens):
    """(prefix, new) tokens of each request; the plan's and the one-shot form."""
    total = [a + b for a, b in lens]
    count = [-(-n // page) for n in total]
    order = np.random.default_rng(1).permutation(sum(count) + 1).astype(np.int32)
    table = np.full((len(lens), max(count)), -1, dtype=np.int32)
    at = 0
    for i, c in enumerate(count):
        table[i, :c] = order[at: at + c]
        at += c
    pool = Pool(len(order), hk, page, seed=7)
    cu = np.concatenate([[0], np.cumsum([b for _, b in lens])]).astype(np.int32)
    q = queries(int(cu[-1]), hq)
    plan = hkv.hkv_prefill_plan_create(pool.handle, cu, table, total, hq)
    need = hkv.hkv_prefill_plan_workspace_bytes(plan)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    with pytest.raises(hkv.HkvError):
        hkv.attn_prefill_plan_run(plan, q, SCALE, torch.empty_like(q), None)
    results = []
    for one_shot in (False, True):
        out, lse = torch.full_like(q, float("nan")), torch.full(q.shape[:2], float("nan"), device="cuda")
        if one_shot:
            hkv.attn_prefill_with_prefix(pool.handle, q, cu, table, total, hq, SCALE, out, lse, ws, need)
        else:
            hkv.attn_prefill_plan_run(plan, q, SCALE, out, lse, None, ws, need)
        results.append((f64(out), lse.double().cpu().numpy()))
    np.testing.assert_array_equal(results[0][0], results[1][0])
    k, v = pool.values()
    refs = []
    for i, (prefix, new) in enumerate(lens):
        kk, vv = (of_sequence(x, table[i, : count[i]], page, total[i]) for x in (k, v))
        for j in range(new):
            refs.append(attention(f64(q)[cu[i] + j], kk, vv, SCALE, np.arange(total[i]) <= prefix + j))
    check_rows(*results[0], tuple(np.stack([x[i] for x in refs]) for i in range(4)))
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


def test_prefill_rows_anywhere():
    """The new tokens' rows lie where the caller says; rows between them stay as they are."""
    pool = Pool(30, 2, seed=7)
    order = np.random.default_rng(1).permutation(30).astype(np.int32)
    table = np.full((2, 19), -1, dtype=np.int32)
    table[0, :6], table[1] = order[:6], order[6:25]
    q = queries(100, 8)
    results = []
    for plan, rows in ((hkv.hkv_prefill_plan_create(pool.handle, [0, 40, 60], table, [90, 300], 8), torch.cat([q[5:45], q[70:90]])),
                       (hkv.hkv_prefill_plan_create_rows(pool.handle, [5, 70], [40, 20], table, [90, 300], 8), q)):
        out, lse = torch.full_like(rows, float("nan")), torch.full((len(rows), 8), float("nan"), device="cuda")
        need = hkv.hkv_prefill_plan_workspace_bytes(plan)
        hkv.attn_prefill_plan_run(plan, rows, SCALE, out, lse, None, torch.empty(need, dtype=torch.uint8, device="cuda"), need)
        results.append((f64(out), lse.double().cpu().numpy()))
        hkv.hkv_prefill_plan_destroy(plan)
    mine = np.r_[5:45, 70:90]
    for a, b in zip(*results):
        np.testing.assert_array_equal(a, b[mine])
        assert np.isnan(np.delete(b, mine, axis=0)).all()
    pool.close()


def test_copy_on_write():
    pool = Pool(6, 3, 32, seed=2)
    ids = hkv.kv_pool_alloc(pool.handle, 3)
    hkv.kv_pool_retain(pool.handle, ids[:2])
    before = pool.read()
    new = hkv.kv_pool_copy_on_write(pool.handle, ids)
    assert list(new[2:]) == [ids[2]] and not set(new[:2]) & set(ids)
    for got, was in zip(pool.read(), before):
        for a, b in zip(ids[:2], new[:2]):
            was[2 * b: 2 * b + 2] = was[2 * a: 2 * a + 2]
        np.testing.assert_array_equal(got, was)
    pool.close()

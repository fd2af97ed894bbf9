"""4-bit pools as programs use them: attention in graphs that outlive the lengths they were captured at, two streams at once, pools beyond
4 GiB, page copies, forks and compaction in between; each against a twin that does the same in another way, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool
from test_gpu_four_bit import SCALE, Forest, queries, rows_of

pytestmark = pytest.mark.gpu


def same(a, b):
    return all(torch.equal(x, y) for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale)))


def same_bits(a, b):
    """(rows of any magnitude give infinities and NaN, which are compared, too)"""
    bits = {2: torch.int16, 4: torch.int32, 1: torch.uint8}[a.element_size()]
    return torch.equal(a.contiguous().view(bits), b.contiguous().view(bits))


def workspace(n):
    return torch.empty(n + 256, dtype=torch.uint8, device="cuda")


def results_of(n, hq):
    return torch.zeros(n, hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, hq, device="cuda")


def capture(call):
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(torch.cuda.current_stream())
    return graph


@pytest.mark.parametrize("n_req,prefix,page", [(3, 48, 16), (40, 640, 32), (300, 96, 16)])
def test_captured_attention_follows_a_growing_plan(n_req, prefix, page):
    """Tokens are appended by calls; attention is captured once (two graphs share its workspace) and replayed, beside a call of a twin."""
    hq, hk, steps = 16, 4, 24
    f = Forest([(-1, prefix)] + [(0, 1 + i % 33) for i in range(n_req)], list(range(1, n_req + 1)), page, extra=2 * n_req)
    twins = [Pool(f.n_pages, hk, page, seed=3) for _ in range(2)]
    plans = [hkv.hkv_decode_plan_create_growing(p.handle, f.nodes, f.node_pages, f.leaves, hq, steps) for p in twins]
    ws = [workspace(hkv.hkv_decode_plan_workspace_bytes(p)) for p in plans]
    q = [queries(n_req, hq, seed=1) for _ in range(3)]
    out, lse = zip(*(results_of(n_req, hq) for _ in range(3)))

    def run(i, stream=None, of=None):
        of = i if of is None else of
        hkv.attn_decode_plan_run(plans[of], q[i], SCALE, out[i], lse[i], ws[of], ws[of].numel() - 256, stream)

    length, fresh, graphs = np.asarray(f.n_tokens[1:]), list(f.unused), None
    for step in range(steps):
        new = np.full(n_req, -1, dtype=np.int32)
        for r in np.flatnonzero(length % page == 0):
            new[r] = fresh.pop()
        length = length + 1
        k, v = rows_of(n_req, hk, 100 + step), rows_of(n_req, hk, 200 + step)
        for p in plans:
            hkv.hkv_decode_plan_append_tokens(p, new, k, v)
        q[1].copy_(queries(n_req, hq, seed=300 + step))
        q[0].copy_(q[1])
        q[2].copy_(-q[1])
        if graphs is None:
            graphs = [capture(lambda s: run(0, s)), capture(lambda s: run(2, s, of=0))]
        graphs[1].replay()
        graphs[0].replay()
        run(1)
        torch.cuda.synchronize()
        assert torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]) and torch.isfinite(lse[0]).all(), step
        q[1].copy_(q[2])
        run(1)
        torch.cuda.synchronize()
        assert torch.equal(out[2], out[1]) and torch.equal(lse[2], lse[1]), step
    assert same(*twins)
    del graphs
    for p in plans:
        hkv.hkv_decode_plan_destroy(p)
    for p in twins:
        p.close()


def test_captured_prefill():
    """Prefill captured once; pages and queries change between its replays."""
    hq, hk, total = 8, 2, [90, 300]
    table = np.full((2, 19), -1, dtype=np.int32)
    order = np.random.default_rng(1).permutation(30).astype(np.int32)
    table[0, :6], table[1] = order[:6], order[6:25]
    pool = Pool(30, hk, seed=7)
    plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 40, 90], table, total, hq)
    ws = workspace(hkv.hkv_prefill_plan_workspace_bytes(plan))
    q = queries(90, hq)
    out, lse = zip(*(results_of(90, hq) for _ in range(2)))
    graph = capture(lambda s: hkv.attn_prefill_plan_run(plan, q, SCALE, out[0], lse[0], s, ws, ws.numel() - 256))
    for i in range(5):
        k, v = rows_of(200, hk, i), rows_of(200, hk, 50 + i)
        hkv.kv_pool_write(pool.handle, table[1, :13], 3, 200, k, v)
        q.copy_(queries(90, hq, seed=i))
        graph.replay()
        hkv.attn_prefill_plan_run(plan, q, SCALE, out[1], lse[1], None, ws, ws.numel() - 256)
        torch.cuda.synchronize()
        assert same_bits(out[0], out[1]) and same_bits(lse[0], lse[1]) and torch.isfinite(lse[0][:40]).all()
    del graph
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


def test_two_streams_at_once():
    """Steps of two forests of one pool, a stream each, and one plan on both streams with workspaces of their own."""
    hq, hk, steps = 32, 8, 12
    f = Forest([(-1, 640), (0, 40), (0, 33), (-1, 3200)] + [(3, 7 + 40 * i) for i in range(30)], [], 16, extra=64)
    leaves = [[1, 2], list(range(4, 34))]
    results = []
    pools = [Pool(f.n_pages, hk, seed=1) for _ in range(2)]
    for twin, pool in enumerate(pools):
        plans = [hkv.hkv_decode_plan_create_growing(pool.handle, f.nodes, f.node_pages, x, hq, steps) for x in leaves]
        ws = [workspace(hkv.hkv_decode_plan_workspace_bytes(p)) for p in plans]
        q = [queries(len(x), hq, seed=i) for i, x in enumerate(leaves)]
        res = [results_of(len(x), hq) for x in leaves]
        rows = [(rows_of(len(x), hk, 5, spread=False), rows_of(len(x), hk, 6, spread=False)) for x in leaves]
        here = torch.cuda.current_stream()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if twin else [here, here]
        for s in streams:
            s.wait_stream(here)
        fresh = list(f.unused)
        for step in range(steps):
            for i, s in enumerate(streams):
                length = np.asarray([f.n_tokens[v] for v in leaves[i]]) + step
                new = np.array([fresh.pop() if n % 16 == 0 else -1 for n in length], dtype=np.int32)
                hkv.hkv_decode_plan_append_tokens(plans[i], new, *rows[i], s)
                hkv.attn_decode_plan_run(plans[i], q[i], SCALE, *res[i], ws[i], ws[i].numel() - 256, s)
        torch.cuda.synchronize()
        again = [results_of(30, hq) for _ in range(2)]
        more = workspace(ws[1].numel())
        for i, s in enumerate(streams):
            hkv.attn_decode_plan_run(plans[1], q[1], SCALE, *again[i], (ws[1], more)[i], ws[1].numel() - 256, s)
        torch.cuda.synchronize()
        results.append([*res[0], *res[1], *again[0], *again[1]])
        for p in plans:
            hkv.hkv_decode_plan_destroy(p)
    for a, b in zip(*results):
        assert torch.equal(a, b) and torch.isfinite(a).all()
    for i in (0, 1):  # the plan's last step, and the same on both streams
        assert torch.equal(results[0][2 + i], results[0][4 + i]) and torch.equal(results[0][4 + i], results[0][6 + i])
    assert same(*pools)
    for p in pools:
        p.close()


def test_the_one_shot_form():
    hq, hk = 32, 8
    f = Forest([(-1, 100), (0, 5), (0, 0), (0, 64), (3, 1)], [1, 2, 4, 4], 16)
    pool = Pool(f.n_pages, hk)
    q = queries(4, hq)
    plan = hkv.hkv_decode_plan_create(pool.handle, f.nodes, f.node_pages, f.leaves, hq)
    need = hkv.attn_decode_workspace_bytes(pool.handle, f.nodes, f.node_pages, f.leaves, hq)
    assert need == hkv.hkv_decode_plan_workspace_bytes(plan)
    ws, res = workspace(need), [results_of(4, hq) for _ in range(2)]
    hkv.attn_decode_plan_run(plan, q, SCALE, *res[0], ws, need)
    hkv.attn_decode_prefix_tree(pool.handle, q, f.nodes, f.node_pages, f.leaves, hq, SCALE, *res[1], ws, need)
    torch.cuda.synchronize()
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1]) and torch.isfinite(res[0][1]).all()
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


class PlacedPool(Pool):
    """Zeros, large or small."""

    def __init__(self, pages, heads, dtype):
        self.heads, self.page_size, self.blocks, self.dtype = heads, 16, pages, dtype
        n = pages * heads
        if dtype == hkv.FP4_E2M1:
            self.k, self.v = (torch.zeros(n * 1024, dtype=torch.uint8, device="cuda") for _ in range(2))
            self.k_scale, self.v_scale = (torch.full((n * 64,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        else:
            self.k, self.v = (torch.zeros(n * 2048, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.k_scale = self.v_scale = None
        self.handle = hkv.kv_pool_create(pages, heads, dtype, self.k, self.v, self.k_scale, self.v_scale)


def test_blocks_beyond_4_gib():
    """A prompt, a step and its attention, copies to a bf16 pool and back, a fork and a compaction in a pool's last pages: as in a small one."""
    hq, hk, prompt = 32, 8, 700
    far_pages = (1 << 32) // (hk * 1024) + 200  # (scales: 512 bytes a page)
    wide_pages = (1 << 32) // (hk * 4096) + 200
    results = []
    order = np.random.default_rng(1).permutation(100).astype(np.int32)
    for pages, other_pages in ((200, 200), (far_pages, wide_pages)):
        pool, wide = PlacedPool(pages, hk, hkv.FP4_E2M1), PlacedPool(other_pages, hk, hkv.BF16)
        hkv.kv_pool_alloc(pool.handle, pages)
        hkv.kv_pool_release(pool.handle, np.arange(pages - 60, pages, dtype=np.int32))
        ids, there = order + pages - 200, order + other_pages - 200
        k, v = rows_of(prompt, hk, 1, spread=False), rows_of(prompt, hk, 2, spread=False)
        hkv.kv_pool_write(pool.handle, ids[:44], 0, prompt, k, v)
        hkv.kv_pool_append(pool.handle, ids[44:46], [5, 9], k[:2], v[:2])
        hkv.kv_pool_copy_pages(wide.handle, there[:46], pool.handle, ids[:46])
        hkv.kv_pool_copy_pages(pool.handle, ids[46:92], wide.handle, there[:46])
        base, own = ids[46:90], ids[90:92]
        plan = hkv.hkv_decode_plan_create(pool.handle, [(-1, 0, 44, 700), (0, 44, 1, 6), (0, 45, 1, 10)], [*base, *own], [1, 2] * 20, hq)
        q = queries(40, hq, seed=4)
        ws, res = workspace(hkv.hkv_decode_plan_workspace_bytes(plan)), results_of(40, hq)
        hkv.attn_decode_plan_run(plan, q, SCALE, *res, ws, ws.numel() - 256)
        hkv.hkv_decode_plan_destroy(plan)
        plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 40], [list(base)], [700], hq)
        wp, pre = workspace(hkv.hkv_prefill_plan_workspace_bytes(plan)), results_of(40, hq)
        hkv.attn_prefill_plan_run(plan, q, SCALE, *pre, None, wp, wp.numel() - 256)
        hkv.hkv_prefill_plan_destroy(plan)
        seq = hkv.kv_pool_alloc(pool.handle, 3)
        hkv.kv_pool_copy_pages(pool.handle, seq, wide.handle, there[:3])
        fork = hkv.kv_pool_fork(pool.handle, seq, [40], [0, 0])
        at = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int64)).cuda()
        content = [t.view(pages, -1)[at(fork)] for t in (pool.k, pool.v, pool.k_scale, pool.v_scale)]
        held = [t.view(pages, -1)[at(ids)] for t in (pool.k, pool.v, pool.k_scale, pool.v_scale)]
        # everything but the forks goes, and those move to the pool's front (in the small pool onto some of ids)
        hkv.kv_pool_release(pool.handle, np.arange(pages - 60, dtype=np.int32))
        hkv.kv_pool_release(pool.handle, seq)
        new = hkv.kv_pool_compact(pool.handle)
        moved = [t.view(pages, -1)[at(new[fork])] for t in (pool.k, pool.v, pool.k_scale, pool.v_scale)]
        torch.cuda.synchronize()
        assert sorted(set(new[fork])) == [0, 1, 2, 3] and all(torch.equal(a, b) for a, b in zip(content, moved))
        results.append([*res, *pre, *content, wide.k.view(other_pages, -1)[at(there[:46])].view(torch.int16), *held])
        assert torch.isfinite(res[1]).all() and torch.isfinite(pre[1]).all() and held[0][:44].any()
        used = pool.k.view(pages, -1)[4: pages - 200].any()
        assert not used, "pages of nobody"
        pool.close()
        wide.close()
    for a, b in zip(*results):
        assert torch.equal(a, b)

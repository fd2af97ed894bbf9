"""The calls around a step's attention as programs make them: in graphs that outlive the lengths they were captured at, on two streams at
once, and over pools beyond 4 GiB; each against a twin that does the same in another way, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from operators_plain import TORCH, Pool
from test_gpu_operators import SCALE, Rows, forest

pytestmark = pytest.mark.gpu


def same_pools(a, b, blocks=None, others=None):
    """Equal bytes (of those blocks of a and the others of b)."""
    for x, y, kind in ((a.k, b.k, 0), (a.v, b.v, 0), (a.k_scale, b.k_scale, 1), (a.v_scale, b.v_scale, 1)):
        if x is None:
            continue
        x, y = x.view(a.blocks, -1), y.view(b.blocks, -1)
        if blocks is not None:
            x, y = x[blocks], y[others]
        bits = torch.int32 if kind else torch.uint8
        if not torch.equal(x.contiguous().view(bits), y.contiguous().view(bits)):
            return False
    return True


@pytest.mark.parametrize("dtype, page", [(hkv.BF16, 16), (hkv.FP8_E4M3, 32)])
def test_a_captured_step_follows_a_growing_plan(dtype, page):
    """Store, attention and weights captured once and replayed after every append, beside the same calls made anew."""
    hq, heads, steps, n = 8, 2, 40, 3
    parent, tokens = [-1, 0, 0, 0], [48, 1, 15, 40]
    nodes, pages, _, spare = forest(parent, tokens, page, 2, spare=n * 4)
    twins = [Pool(len(pages) + len(spare), heads, dtype, page, seed=6) for _ in range(2)]
    plans = [hkv.hkv_decode_plan_create_growing(p.handle, nodes, pages, [1, 2, 3], hq, steps) for p in twins]
    x = [Rows(n, hq, heads, dtype, 1) for _ in range(2)]
    ws = [torch.empty(hkv.hkv_decode_plan_workspace_bytes(p) + 256, dtype=torch.uint8, device="cuda") for p in plans]
    out, lse = [torch.zeros_like(r.q_out) for r in x], [torch.zeros(n, hq, device="cuda") for _ in x]
    w = [torch.zeros(p.blocks, heads, 16, device="cuda") for p in twins]
    for p in plans:
        hkv.hkv_decode_plan_track_weights(p)

    def step(i, stream=None):
        hkv.hkv_decode_plan_store(plans[i], x[i].arg, stream)
        hkv.attn_decode_plan_run(plans[i], x[i].q_out, SCALE, out[i], lse[i], ws[i], ws[i].numel(), stream)
        hkv.attn_decode_plan_weights(plans[i], x[i].q_out, SCALE, lse[i], 0.9, 1, w[i], stream)

    length, taken, graph = np.asarray(tokens[1:]), 0, None
    for k in range(steps):
        ids = np.full(n, -1, dtype=np.int32)
        for r in np.flatnonzero(length % page == 0):
            ids[r], taken = spare[taken], taken + 1
        length = length + 1
        fresh = torch.randn_like(x[0].all, dtype=torch.float32)
        for i in range(2):
            x[i].all.copy_(fresh)
            hkv.hkv_decode_plan_append(plans[i], ids)
        step(1)
        if graph is None:  # (nothing runs while it is captured: the replay is this step's, too)
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                step(0, torch.cuda.current_stream())
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(x[0].q_out, x[1].q_out) and torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]) and torch.equal(w[0], w[1]), k
        assert torch.isfinite(lse[0]).all() and same_pools(*twins), k
    for p in plans:
        hkv.hkv_decode_plan_destroy(p)
    for p in twins:
        p.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3, hkv.FP32])
def test_a_captured_store_of_prompts(dtype):
    """Several launches' worth of requests, replayed with other rows in the same buffers."""
    n, hq, heads = 200, 4, 2
    rng = np.random.default_rng(3)
    new, prefix = rng.integers(0, 30, n), rng.integers(0, 30, n)
    cu = np.concatenate([[0], np.cumsum(new)])
    table = rng.permutation(4 * n).astype(np.int32).reshape(n, 4)
    twins = [Pool(4 * n, heads, dtype, seed=8) for _ in range(2)]
    plans = [hkv.hkv_prefill_plan_create(p.handle, cu, table, prefix + new, hq) for p in twins]
    x = [Rows(int(cu[-1]), hq, heads, dtype, 2) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        hkv.hkv_prefill_plan_store(plans[0], x[0].arg, torch.cuda.current_stream())
    for k in range(3):
        fresh = torch.randn_like(x[0].all, dtype=torch.float32) * (k + 1)
        for r in x:
            r.all.copy_(fresh)
            r.q_out.fill_(float("nan"))
        graph.replay()
        hkv.hkv_prefill_plan_store(plans[1], x[1].arg)
        torch.cuda.synchronize()
        assert torch.equal(x[0].q_out, x[1].q_out) and not torch.isnan(x[0].q_out).any() and same_pools(*twins), k
    for p in plans:
        hkv.hkv_prefill_plan_destroy(p)
    for p in twins:
        p.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3, hkv.FP32])
def test_two_streams_at_once(dtype):
    """Two forests of one pool, a stream each, and one plan's weights on both streams: as one after the other."""
    hq, heads = 8, 2
    parent, tokens = [-1, 0, 0, -1, 3, 3], [640, 40, 33, 320, 70, 7]
    nodes, pages, _, _ = forest(parent, tokens, 16, 5)
    twins = [Pool(len(pages), heads, dtype, seed=1) for _ in range(2)]
    results = []
    for twin, p in enumerate(twins):
        plans = [hkv.hkv_decode_plan_create(p.handle, nodes, pages, leaves, hq) for leaves in ([1, 2], [4, 5])]
        x = [Rows(2, hq, heads, dtype, 10 + i) for i in range(2)]
        ws = [torch.empty(hkv.hkv_decode_plan_workspace_bytes(q) + 256, dtype=torch.uint8, device="cuda") for q in plans]
        out, lse = [torch.zeros_like(r.q_out) for r in x], [torch.zeros(2, hq, device="cuda") for _ in x]
        w = [torch.zeros(p.blocks, heads, 16, device="cuda") for _ in range(4)]
        for q in plans:
            hkv.hkv_decode_plan_track_weights(q)
        here = torch.cuda.current_stream()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()] if twin else [here, here]
        for s in streams:
            s.wait_stream(here)
        for _ in range(10):
            for i, s in enumerate(streams):
                hkv.hkv_decode_plan_store(plans[i], x[i].arg, s)
                hkv.attn_decode_plan_run(plans[i], x[i].q_out, SCALE, out[i], lse[i], ws[i], ws[i].numel(), s)
                hkv.attn_decode_plan_weights(plans[i], x[i].q_out, SCALE, lse[i], 0.5, 1, w[i], s)
        torch.cuda.synchronize()
        for i, s in enumerate(streams):  # the same plan's, on both
            hkv.attn_decode_plan_weights(plans[0], x[0].q_out, SCALE, lse[0], 0.0, 0, w[2 + i], s)
        torch.cuda.synchronize()
        results.append([*(r.q_out for r in x), *out, *lse, *w])
        assert torch.equal(w[2], w[3])
        for q in plans:
            hkv.hkv_decode_plan_destroy(q)
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert same_pools(*twins)
    for p in twins:
        p.close()


class FarPool(Pool):
    """A pool of more than 4 GiB a buffer, of zeros."""

    def __init__(self, pages, heads, dtype):
        self.heads, self.dtype, self.page_size, self.blocks = heads, dtype, 16, pages
        self.k, self.v = (torch.zeros(pages * 16 * heads * 128, dtype=TORCH[dtype], device="cuda") for _ in range(2))
        self.k_scale, self.v_scale = (torch.ones(pages * heads, device="cuda") if dtype == hkv.FP8_E4M3 else None for _ in range(2))
        self.handle = hkv.kv_pool_create(pages, heads, dtype, self.k, self.v, self.k_scale, self.v_scale, page_size=16)


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3, hkv.FP32])
def test_blocks_beyond_4_gib(dtype):
    """A prompt stored, a step stored and weighed, and the prompt shrunk, in a pool's last pages: as in a small one."""
    hq, heads, prompt = 8, 8, 700
    size = {hkv.BF16: 2, hkv.FP8_E4M3: 1, hkv.FP32: 4}[dtype]
    far = FarPool((1 << 32) // (16 * heads * 128 * size) + 200, heads, dtype)
    near = FarPool(200, heads, dtype)
    order = np.random.default_rng(1).permutation(200).astype(np.int32)
    results = []
    for p, base in ((near, 0), (far, far.blocks - 200)):
        ids = order + base
        mine, own, kept_pages = ids[:44], ids[44:46], ids[46:66]
        plan = hkv.hkv_prefill_plan_create(p.handle, [0, prompt], [list(mine)], [prompt], hq)
        x = Rows(prompt, hq, heads, dtype, 4)
        hkv.hkv_prefill_plan_store(plan, x.arg)
        hkv.hkv_prefill_plan_destroy(plan)
        # (the forest's root is whole blocks of it: plans over fp32 pools ask for those)
        plan = hkv.hkv_decode_plan_create(p.handle, [(-1, 0, 43, 688), (0, 43, 1, 9), (0, 44, 1, 5)], [*mine[:43], *own], [1, 2], hq)
        y = Rows(2, hq, heads, dtype, 5)
        hkv.hkv_decode_plan_store(plan, y.arg)
        ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
        out, lse, w = torch.zeros_like(y.q_out), torch.zeros(2, hq, device="cuda"), torch.zeros(p.blocks, heads, 16, device="cuda")
        hkv.attn_decode_plan_run(plan, y.q_out, SCALE, out, lse, ws, ws.numel())
        hkv.hkv_decode_plan_track_weights(plan)
        hkv.attn_decode_plan_weights(plan, y.q_out, SCALE, lse, 1.0, 1, w)
        kept = torch.zeros(heads, 300, dtype=torch.int32, device="cuda")
        hkv.kv_pool_evict(p.handle, mine, [prompt], kept_pages[:19], [300], 4, 20, w, kept)
        torch.cuda.synchronize()
        results.append([x.q_out, y.q_out, out, lse, kept, w[torch.from_numpy(ids).long().cuda()]])
        hkv.hkv_decode_plan_destroy(plan)
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert torch.isfinite(results[0][3]).all() and (results[0][5] > 0).any()
    at = torch.from_numpy(order).long().cuda()
    assert same_pools(near, far, at, at + far.blocks - 200)
    assert not far.k.view(far.blocks, -1)[: far.blocks - 200].view(torch.uint8).any(), "blocks of nobody"
    near.close()
    far.close()

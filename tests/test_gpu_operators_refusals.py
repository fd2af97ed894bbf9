"""What the calls around a step's attention refuse beside work on the GPU, and that the work goes on."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from operators_plain import Pool
from test_gpu_operators import Rows, forest
from test_gpu_operators_use import same_pools

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_req", [3, 300])
def test_an_append_is_refused_while_a_graph_is_captured(n_req):
    """... and neither the capture nor the plan suffers: replays and later appends as on a twin that was never asked."""
    hq, heads = 4, 2
    tokens = [32] + [15, 16, 3] * (n_req // 3)
    nodes, pages, _, spare = forest([-1] + [0] * n_req, tokens, 16, 7, spare=2 * n_req)
    twins = [Pool(len(pages) + len(spare), heads, hkv.BF16, seed=5) for _ in range(2)]
    plans = [hkv.hkv_decode_plan_create_growing(p.handle, nodes, pages, np.arange(1, n_req + 1), hq, 8) for p in twins]
    x = [Rows(n_req, hq, heads, hkv.BF16, 1) for _ in range(2)]
    count = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(hkv.HkvError) as e:
            hkv.hkv_decode_plan_append_qkv(plans[0], spare[:n_req], x[0].arg)
        count += 1
    assert e.value.code == hkv.EINVAL and "captur" in hkv.last_error()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert (count == 3).all() and torch.isnan(x[0].q_out).all() and same_pools(*twins)
    for step in range(3):
        for i in range(2):
            hkv.hkv_decode_plan_append_qkv(plans[i], spare[n_req * (step % 2):][:n_req], x[i].arg)
        torch.cuda.synchronize()
        assert torch.equal(x[0].q_out, x[1].q_out) and not torch.isnan(x[0].q_out).any() and same_pools(*twins), step
    for p in plans:
        hkv.hkv_decode_plan_destroy(p)
    for p in twins:
        p.close()


def test_places_expanded_over_the_axes_turn_as_when_written_out():
    pool = Pool(2, 2, hkv.BF16)
    plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 20], [[1, 0]], [20], 4)
    line, axis = torch.arange(100, 120, dtype=torch.int32, device="cuda"), np.arange(64) % 3
    x, results = Rows(20, 4, 2, hkv.BF16, 3, norm=False), []
    for places in (line.expand(3, 20), line.repeat(3, 1)):
        hkv.hkv_prefill_plan_store(plan, hkv.qkv_rows(x.q, x.k, x.v, x.q_out, rotary_dim=128, inv_freq=x.inv_freq, positions=places, axis=axis))
        torch.cuda.synchronize()
        results.append((x.q_out.clone(), pool.k.clone()))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and not torch.isnan(results[0][0]).any()
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()

"""The README's lines for what stands around a step's attention, run as they are written there and held against 64 bits: a call
that generates, weighs its keys, is shrunk and goes on."""
import os
import textwrap

import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from operators_plain import Pool, check_rows, evicted, key_weights
from test_gpu_operators import SCALE, WEIGHT_TOL, Rows, weight_nodes

pytestmark = pytest.mark.gpu
README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")
N, KEPT = 301, 301 // 4                                  # tokens, the first step's among them, and how many stay


class Program:
    """What the README's lines find around them: the binding, with fresh rows and pages for every step and a note of what came out."""

    def __init__(self, dtype):
        self.pool = Pool(60, 2, dtype, seed=2)
        order = np.random.default_rng(3).permutation(60).astype(np.int32)
        self.pages, self.fresh, self.spare = order[:19], order[19:24], list(order[24:])
        self.x = Rows(1, 8, 2, dtype, 5)
        self.x.eps = 1e-6                                # (the README leaves it at the binding's)
        self.first = self.x.all.clone()
        self.lse = torch.zeros(1, 8, device="cuda")
        self.weights = 50 * torch.rand(60, 2, 16, device="cuda")     # what earlier users of the pages left
        self.kept = torch.full((2, KEPT), -1, dtype=torch.int32, device="cuda")
        self.new_page_ids = np.full(1, -1, dtype=np.int32)
        self.plan = hkv.hkv_decode_plan_create_growing(self.pool.handle, [(-1, 0, 19, N - 1)], self.pages, [0], 8, 8)
        self.at, self.plans, self.steps = list(self.fresh), [], []
        self.weighed = None

    def rows(self, step):
        self.x.all.copy_(self.first * (1 + step % 5))
        self.x.q_in = self.x.q.clone()

    def hkv_decode_plan_append_qkv(self, plan, *rest):
        step = len(self.plans)
        self.rows(step)
        if step and (KEPT + step - 1) % 16 == 0:
            self.at.append(self.spare.pop())
            self.new_page_ids[0] = self.at[-1]
        self.plans.append(plan)
        hkv.hkv_decode_plan_append_qkv(plan, *rest)

    def attn_decode_plan_run(self, plan, q, *rest):
        hkv.attn_decode_plan_run(plan, q, *rest)
        self.steps.append((q.float().cpu().double().numpy(), self.lse.cpu().double().numpy(), self.pool.values()[0] if len(self.steps) % 50 < 3 else None))

    def attn_decode_plan_weights(self, *rest):
        hkv.attn_decode_plan_weights(*rest)
        if self.weighed is None:
            self.weighed = self.weights.cpu().numpy().copy()

    def __getattr__(self, name):                         # everything else is the binding's
        return getattr(hkv, name)


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3])
def test_a_call_that_is_shrunk_goes_on_as_the_readme_has_it(dtype):
    with open(README) as f:
        text = f.read()
    lines = textwrap.dedent(text[text.index("    # with the projections' raw rows"): text.index("    # several tokens per call")])
    p = Program(dtype)
    x = p.x
    exec(lines, dict(hkv=p, torch=torch, pool=p.pool.handle, plan=p.plan, q_rows=x.q, k_rows=x.k, v_rows=x.v, q_rot=x.q_out, wq=x.qw, wk=x.kw, inv_freq=x.inv_freq,
                     scale=SCALE, out=torch.zeros_like(x.q_out), lse=p.lse, ws=torch.empty(1 << 22, dtype=torch.uint8, device="cuda"), key_weights=p.weights, kept=p.kept,
                     pages=p.pages, fresh_pages=p.fresh, n=N, num_q_heads=8, new_page_ids=p.new_page_ids))
    torch.cuda.synchronize()
    # the first step's weights, over pages that others had used, and what they say
    q, lse, keys = p.steps[0]
    blocks, t = p.pages.astype(np.int64), np.arange(N)
    want = key_weights(keys, weight_nodes([-1], [N], [blocks], [0], 1), q, lse, SCALE, 2, np.zeros(p.weights.shape), 0.99, 1, 1)[blocks[t // 16], :, t % 16]
    assert (np.abs(p.weighed[blocks[t // 16], :, t % 16] - want) <= WEIGHT_TOL * want).all()
    for h in range(2):
        assert np.array_equal(p.kept.cpu().numpy()[h], evicted(p.weighed[:, h], blocks, N, KEPT, 4, 64))
    # every step's token is at its own place, the first at N - 1 and the others behind it, wherever its key lies
    assert len(p.steps) == len(p.plans) > 3
    for i, (q, _, keys) in enumerate(p.steps):
        p.rows(i)
        exact, size, k, k_size = x.exact([N - 1 + i])
        check_rows(q, exact, size, hkv.BF16, f"queries of step {i}")
        if keys is not None:
            j = KEPT + i - 1
            got = keys[p.at[j // 16], :, j % 16] if i else keys[blocks[-1], :, (N - 1) % 16]
            step = 2.0 ** -8 if dtype == hkv.BF16 else 2.0 ** -3     # (8 bits: half a step of the block's largest, twice rounded at most)
            assert (np.abs(got - k[0]) <= step * np.abs(keys[p.at[j // 16] if i else blocks[-1]]).max() + 2.0 ** -18 * k_size[0]).all(), f"key of step {i}"
    for plan in (p.plan, p.plans[-1]):
        hkv.hkv_decode_plan_destroy(plan)
    p.pool.close()

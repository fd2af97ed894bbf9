"""4-bit pools: how exact decode's scores are where a row's products differ much in size (queries with outlier dimensions, keys with outlier groups of
32, products that cancel), in every kind of item and in whole paths, against 64-bit attention."""
import math

import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from four_bit_plain import Pool, check_rows
from test_gpu_four_bit import Forest, decode, f64, queries

pytestmark = pytest.mark.gpu

# (settings, rows under the root): whole paths, items whose tokens four wavefronts share, one wavefront each, two row tiles, 16 rows a wavefront, 32 rows a wavefront
KINDS = {"paths": ({}, 16), "shared tokens": (dict(max_rows=16, pack=1), 16), "wavefronts": (dict(max_rows=16, pack=3), 16), "two tiles": (dict(max_rows=32), 32),
         "rows": (dict(max_rows=64), 64), "tall": (dict(max_rows=128), 128)}


def reference(q, k, v, scale):
    """Rows of one request, as four_bit_plain.attention gives them, but for what a score may be off by: a row of q is four terms of e2m3, exact for elements down to 2^-12
    of the largest of their 32 dimensions and 2^-20 of that below, and a score is the sum of 4 x 16 sums of eight products, which lose less than a step of 2^-23 each."""
    hq, hk = q.shape[0], k.shape[1]
    out, weight, lse, size = np.zeros((hq, 128)), np.zeros((hq, 128)), np.zeros(hq), np.zeros(hq)
    for h in range(hq):
        kk, vv = k[:, h // (hq // hk)], v[:, h // (hq // hk)]
        top = np.repeat(np.abs(q[h]).reshape(4, 32).max(1), 32)
        lost = np.where(np.abs(q[h]) < 2.0 ** -12 * top, 2.0 ** -20 * top, 0)
        size[h] = (np.abs(kk) @ (np.abs(q[h]) * 130 * 2.0 ** -24 + lost)).max() * abs(scale)
        x = kk @ q[h] * scale
        lse[h] = x.max() + math.log(np.exp(x - x.max()).sum())
        p = np.exp(x - lse[h])
        out[h], weight[h] = p @ vv, p @ np.abs(vv)
    return out, lse, weight, size


def outliers(kind, n, hq):
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x = queries(n, hq).float()
    if kind == "one":            # a dimension 2^8 of the others
        x.scatter_(2, torch.randint(0, 128, (n, hq, 1), device="cuda", generator=g), 500.0)
    elif kind == "each eight":   # a dimension of every eight
        at = torch.randint(0, 8, (n, hq, 16, 1), device="cuda", generator=g)
        y = x.view(n, hq, 16, 8)
        y.scatter_(3, at, y.gather(3, at) * 300)
    elif kind == "wide":         # sizes from 1 to 2^-20
        x *= torch.exp2(-20 * torch.rand(x.shape, device="cuda", generator=g))
    elif kind == "small":        # a row near the smallest numbers that the terms' scales reach, another of zeros
        x *= 2.0 ** -100
        x[:, 0] = 0
    return x.to(torch.bfloat16)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("query", ["one", "each eight", "wide", "small", "cancel"])
@pytest.mark.parametrize("sign", [1, -1])
def test_sums_of_unlike_products(kind, query, sign):
    settings, rows = KINDS[kind]
    hq, hk = 8, 1
    n = rows // hq
    f = Forest([(-1, 150)] + [(0, 5 + 3 * i) for i in range(n)], list(range(1, n + 1)), 16, seed=n)
    pool = Pool(f.n_pages, hk, seed=n)
    q = outliers(query, n, hq)
    if query == "cancel":  # in one group of 32 K is 2^12 of the others; two of its products are each other's negatives, the others of it nothing
        pool.k_scale.view(pool.blocks, hk, 4, 16)[:, :, 1] += 12
        q[:, :, 32:64] = 0
        q[:, :, 35] = q[:, :, 57] = 1.75
        codes = pool.k.view(pool.blocks, hk, 4, 4, 64)  # [t % 4][t / 4][d / 2]: dims 56, 57 beside 34, 35
        codes[..., 57 // 2] = (codes[..., 35 // 2] & 0xF0) ^ 0x80
    k, v = pool.values()
    raw = np.abs(f64(q) @ k.reshape(-1, 128).T).max()
    scale = sign * float(np.float32(12 / raw))
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, hq, shared_chunk=0 if kind == "paths" else 2048, **settings)
    assert (hkv.hkv_decode_plan_num_paths(plan) > 0) == (kind == "paths")
    out, lse = decode(plan, q, scale=scale)
    refs = [reference(f64(q)[r], f.keys(k, leaf), f.keys(v, leaf), scale) for r, leaf in enumerate(f.leaves)]
    check_rows(out, lse, tuple(np.stack([x[i] for x in refs]) for i in range(4)))
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("q_by,k_by", [(-106, 110), (110, -115), (-60, -50), (60, 50)])
def test_far_scales(kind, q_by, k_by):
    """Queries and keys near the ends of their scales, whose scores are ordinary numbers of 32 bits."""
    settings, rows = KINDS[kind]
    n = rows // 8
    f = Forest([(-1, 150)] + [(0, 5 + 3 * i) for i in range(n)], list(range(1, n + 1)), 16, seed=n)
    pool = Pool(f.n_pages, 1, seed=n)
    pool.k_scale += k_by % 256
    q = queries(n, 8) * 2.0 ** q_by
    k, v = pool.values()
    scale = float(np.float32(12 / np.abs(f64(q) @ k.reshape(-1, 128).T).max()))
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, f.nodes, f.node_pages, f.leaves, 8, shared_chunk=0 if kind == "paths" else 2048, **settings)
    out, lse = decode(plan, q, scale=scale)
    refs = [reference(f64(q)[r], f.keys(k, leaf), f.keys(v, leaf), scale) for r, leaf in enumerate(f.leaves)]
    check_rows(out, lse, tuple(np.stack([x[i] for x in refs]) for i in range(4)))
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()

"""Calls that move pages: copies between pools of every pair of types, forks, compaction, against plain forms on the host."""
import os
import textwrap

import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

import four_bit_plain as four
import operators_plain as plain

pytestmark = pytest.mark.gpu
TYPES = [hkv.BF16, hkv.FP8_E4M3, hkv.FP32, hkv.FP4_E2M1]
NAMES = ["bf16", "fp8", "fp32", "fp4"]


def make(pages, heads, dtype, page, seed):
    return four.Pool(pages, heads, page, seed) if dtype == hkv.FP4_E2M1 else plain.Pool(pages, heads, dtype, page, seed)


def raw(pool):
    """Everything the pool's buffers hold, as arrays of bytes by block."""
    return [t.view(torch.uint8).cpu().numpy().reshape(pool.blocks, -1).copy() for t in (pool.k, pool.v, pool.k_scale, pool.v_scale) if t is not None]


def converted(x, dtype):
    """Values [heads][tokens][128] of a block as a pool of a type holds them: taken in fp32 first (an fp8 code of 4 significant bits times a scale of
    24 has up to 28)."""
    x = x.astype(np.float32).astype(np.float64)
    if dtype == hkv.FP32:
        return x
    if dtype == hkv.BF16:
        return torch.from_numpy(x).float().to(torch.bfloat16).double().numpy()
    if dtype == hkv.FP4_E2M1:
        return four.quantised(x)[2]
    x = torch.from_numpy(x).float()
    top = x.abs().amax((1, 2), keepdim=True)
    scale = torch.where(top > 0, top / torch.full_like(top, 448.0), torch.ones_like(top))
    return (x / scale).clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy() * scale.double().numpy()


@pytest.mark.parametrize("src_type", TYPES, ids=NAMES)
@pytest.mark.parametrize("dst_type", TYPES, ids=NAMES)
@pytest.mark.parametrize("heads,page,n", [(2, 16, 5), (8, 64, 3), (3, 32, 400), (1, 128, 2)])
def test_copy(src_type, dst_type, heads, page, n):
    rng = np.random.default_rng(n)
    a, b = make(n + 2, heads, src_type, page, 1), make(n + 3, heads, dst_type, page, 2)
    src, dst = rng.integers(0, n + 2, n), rng.permutation(n + 3)[:n]  # a source may be copied several times
    tokens = rng.integers(0, page + 1, n)
    tokens[:2] = [page, 1]
    values, before, bytes_before, src_bytes = a.values(), b.values(), raw(b), raw(a)
    hkv.kv_pool_copy_pages(b.handle, dst, a.handle, src, tokens)
    torch.cuda.synchronize()
    S = page // 16
    if src_type == dst_type:
        want = [x.copy() for x in bytes_before]
        for s, d, m in zip(src, dst, tokens):
            k = -(-int(m) // 16)
            for w, x in zip(want, src_bytes):
                w[d * S: d * S + k] = x[s * S: s * S + k]
        for got, w in zip(raw(b), want):
            np.testing.assert_array_equal(got, w)
    else:
        after = b.values()
        for is_v in (0, 1):
            want = before[is_v].copy()
            keep = np.ones(want.shape[:1] + (16,), dtype=bool)
            for s, d, m in zip(src, dst, tokens):
                for j in range(-(-int(m) // 16)):
                    k = min(16, int(m) - 16 * j)
                    want[d * S + j, :, :k] = converted(values[is_v][s * S + j, :, :k], dst_type)
                    keep[d * S + j] = np.arange(16) < k if dst_type == hkv.FP8_E4M3 else True  # (fp8: the block's scale is another, codes behind stay)
            mask = np.broadcast_to(keep[:, None, :, None], want.shape)
            np.testing.assert_array_equal(after[is_v][mask], want[mask])
    for got, was in zip(raw(a), src_bytes):
        np.testing.assert_array_equal(got, was)
    a.close()
    b.close()


def test_copy_leaves_what_is_behind_the_tokens():
    """Codes behind the last token of an fp8 block stay as bytes; garbage there, NaN among it, counts for no scale."""
    a, b = make(1, 2, hkv.BF16, 16, 1), make(1, 2, hkv.FP8_E4M3, 16, 2)
    a.k.view(2, 4, 16, 32)[:, :, 5:] = float("nan")
    a.v.view(2, 128, 16)[:, :, 5:] = float("inf")
    before = b.codes(b.k, True), b.codes(b.v, False)
    hkv.kv_pool_copy_pages(b.handle, [0], a.handle, [0], [5])
    after = b.codes(b.k, True), b.codes(b.v, False)
    for x, y in zip(before, after):
        np.testing.assert_array_equal(x[:, :, 5:], y[:, :, 5:])
        assert np.isfinite(y[:, :, :5]).all() and np.abs(y[:, :, :5]).max() == 448
    assert np.isfinite(b.scales()[0]).all()
    a.close()
    b.close()


def test_copy_within_a_pool():
    a = make(5, 2, hkv.FP4_E2M1, 32, 3)
    before = raw(a)
    hkv.kv_pool_copy_pages(a.handle, [0, 3], a.handle, [4, 4])
    for got, w in zip(raw(a), before):
        w[0:2] = w[6:8] = w[8:10]
        np.testing.assert_array_equal(got, w)
    a.close()


def refcounts(pool, n):
    return [hkv.kv_pool_refcount(pool.handle, i) for i in range(n)]


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("release", [False, True])
@pytest.mark.parametrize("page,lens,parent", [(16, [40, 32, 17, 0], [0, 2, 0, 1, 1, 3]), (64, [130, 63, 64], [2, 1, 1, 1, 0]), (16, [5] * 200, list(range(0, 200, 2)) * 2), (128, [100], [])])
def test_fork(dtype, release, page, lens, parent):
    heads, count = 2, [-(-n // page) for n in lens]
    total = sum(count) + 2 * len(parent) + 1
    pool = make(total, heads, dtype, page, 5)
    ids = hkv.kv_pool_alloc(pool.handle, sum(count))
    before, refs, free = raw(pool), refcounts(pool, total), hkv.kv_pool_num_free(pool.handle)
    begin = np.concatenate([[0], np.cumsum(count)])
    out = hkv.kv_pool_fork(pool.handle, ids, lens, parent, release)
    torch.cuda.synchronize()
    after, S, at = raw(pool), page // 16, 0
    want = [x.copy() for x in before]
    want_refs, seen, fresh = list(refs), set(), sum(count)
    for i in parent:
        mine, theirs = out[at: at + count[i]], ids[begin[i]: begin[i + 1]]
        at += count[i]
        whole = lens[i] // page
        assert list(mine[:whole]) == list(theirs[:whole])
        for p in mine[:whole]:
            want_refs[p] += 1
        if lens[i] % page:
            if release and i not in seen:
                assert mine[-1] == theirs[-1]
                want_refs[mine[-1]] += 1
            else:
                assert mine[-1] == fresh  # the next free page
                fresh += 1
                want_refs[mine[-1]] = 1
                used = -(-(lens[i] % page) // 16)
                for w, x in zip(want, before):
                    w[mine[-1] * S: mine[-1] * S + used] = x[theirs[-1] * S: theirs[-1] * S + used]
        seen.add(i)
    assert at == len(out)
    if release:
        for p in ids:
            want_refs[p] -= 1
    assert refcounts(pool, total) == want_refs
    assert hkv.kv_pool_num_free(pool.handle) == sum(r == 0 for r in want_refs) and free - hkv.kv_pool_num_free(pool.handle) == sum(r > 0 for r in want_refs) - sum(count)
    for got, w in zip(after, want):
        np.testing.assert_array_equal(got, w)
    hkv.kv_pool_release(pool.handle, out)
    if not release:
        hkv.kv_pool_release(pool.handle, ids)
    assert hkv.kv_pool_num_free(pool.handle) == total
    pool.close()


@pytest.mark.parametrize("dtype", TYPES, ids=NAMES)
@pytest.mark.parametrize("page,n,live", [(16, 10, 4), (64, 9, 9), (16, 3000, 1700), (32, 7, 0), (128, 6, 1)])
def test_compact(dtype, page, n, live):
    rng = np.random.default_rng(n)
    order = rng.permutation(n).astype(np.int32)
    pool = make(n, 1, dtype, page, 6)
    hkv.kv_pool_destroy(pool.handle)
    pool.handle = hkv.kv_pool_create(n, 1, dtype, pool.k, pool.v, pool.k_scale, pool.v_scale, order, page_size=page)
    ids = hkv.kv_pool_alloc(pool.handle, live)
    hkv.kv_pool_retain(pool.handle, ids[: live // 2])
    before, refs, S = raw(pool), refcounts(pool, n), page // 16
    new = hkv.kv_pool_compact(pool.handle)
    torch.cuda.synchronize()
    assert sorted(new[ids]) == list(range(live)) and set(new) <= set(range(live)) | {-1} and (new >= 0).sum() == live
    stay = ids[ids < live]
    assert (new[stay] == stay).all()
    assert refcounts(pool, n) == [refs[list(new).index(i)] if i < live else 0 for i in range(n)]
    want = [x.copy() for x in before]
    for p in ids:
        for w, x in zip(want, before):
            w[new[p] * S: (new[p] + 1) * S] = x[p * S: (p + 1) * S]
    for got, w in zip(raw(pool), want):
        np.testing.assert_array_equal(got, w)
    if live < n:
        assert list(hkv.kv_pool_alloc(pool.handle, n - live)) == list(range(live, n))
    assert (hkv.kv_pool_num_free(pool.handle)) == 0
    pool.close()


def test_compact_with_a_cache():
    """A prefix cache goes on with its blocks under their new ids."""
    n = 12
    pool = make(n, 2, hkv.BF16, 16, 8)
    hkv.kv_pool_destroy(pool.handle)
    pool.handle = hkv.kv_pool_create(n, 2, hkv.BF16, pool.k, pool.v, free_order=np.arange(n, dtype=np.int32)[::-1])
    cache = hkv.kv_cache_create(pool.handle)
    prompt = np.arange(40, dtype=np.int32)
    first, _ = hkv.kv_cache_acquire(cache, prompt)
    other, _ = hkv.kv_cache_acquire(cache, prompt + 100)
    hkv.kv_cache_release(cache, other)
    content = pool.k.view(n, -1)[torch.from_numpy(first.astype(np.int64)).cuda()].clone()
    new = hkv.kv_pool_compact(pool.handle)
    assert (torch.equal(pool.k.view(n, -1)[torch.from_numpy(new[first].astype(np.int64)).cuda()], content))
    again, cached = hkv.kv_cache_acquire(cache, prompt)
    assert cached == 32 and list(again[:2]) == list(new[first[:2]])
    hkv.kv_cache_release(cache, again)
    hkv.kv_cache_release(cache, new[first])
    # memory runs short: the blocks that no one uses go, all pages come round
    long, cached = hkv.kv_cache_acquire(cache, np.arange(1000, 1000 + 16 * n, dtype=np.int32))
    assert cached == 0 and sorted(long) == list(range(n))
    hkv.kv_cache_release(cache, long)
    hkv.kv_cache_destroy(cache)
    assert hkv.kv_pool_num_free(pool.handle) == n
    pool.close()


def test_refused_under_capture():
    pool = make(4, 1, hkv.BF16, 16, 1)
    ids = hkv.kv_pool_alloc(pool.handle, 2)
    g, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    x = torch.zeros(4, device="cuda")
    with torch.cuda.graph(g, stream=s):
        x += 1
        for call in (lambda: hkv.kv_pool_copy_pages(pool.handle, [3], pool.handle, [0]), lambda: hkv.kv_pool_fork(pool.handle, ids[:1], [5], [0]),
                     lambda: hkv.kv_pool_compact(pool.handle)):
            with pytest.raises(hkv.HkvError):
                call()
        assert list(hkv.kv_pool_fork(pool.handle, ids[:1], [16], [0])) == [ids[0]]  # nothing to copy
    g.replay()
    torch.cuda.synchronize()
    assert hkv.kv_pool_num_free(pool.handle) == 2 and hkv.kv_pool_refcount(pool.handle, int(ids[0])) == 2
    pool.close()


def test_beams_in_use():
    """Beams of one prompt over a 4-bit pool, step by step: appended to, reordered by forks, attended; each equals its own history."""
    heads, hq, beams, page = 2, 8, 4, 16
    pool = four.Pool(80, heads, page, seed=3, poison=True)
    prompt = hkv.kv_pool_alloc(pool.handle, 3)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    kv = lambda n: [torch.randn(n, heads, 128, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]  # noqa: E731
    k0, v0 = kv(37)
    hkv.kv_pool_write(pool.handle, prompt, 0, 37, k0, v0)
    pages, n = [list(hkv.kv_pool_alloc(pool.handle, 1)) for _ in range(beams)], 0
    history = [[[], []] for _ in range(beams)]
    rng = np.random.default_rng(4)
    for step in range(36):
        k, v = kv(beams)
        if n and n % page == 0:
            for p in pages:
                p += list(hkv.kv_pool_alloc(pool.handle, 1))
        hkv.kv_pool_append(pool.handle, [p[-1] for p in pages], [n % page] * beams, k, v)
        n += 1
        for b in range(beams):
            history[b][0].append(k[b])
            history[b][1].append(v[b])
        if step in (0, 15, 16, 35):
            nodes = [(-1, 0, 3, 37)] + [(0, 3 + i * len(pages[0]), len(pages[0]), n) for i in range(beams)]
            plan = hkv.hkv_decode_plan_create(pool.handle, nodes, np.concatenate([prompt, *pages]), np.arange(1, beams + 1), hq)
            q = torch.randn(beams, hq, 128, device="cuda", generator=g).to(torch.bfloat16)
            out, lse = torch.empty_like(q), torch.empty(beams, hq, device="cuda")
            hkv.attn_decode_plan_run_static(plan, q, 0.09, out, lse)
            refs = []
            for b in range(beams):
                keys, vals = (four.quantised(torch.cat([x, torch.stack(h)]).double().cpu().numpy())[2] for x, h in zip((k0, v0), history[b]))
                refs.append(four.attention(q[b].double().cpu().numpy(), keys, vals, 0.09, np.ones(37 + n, dtype=bool)))
            four.check_rows(out.double().cpu().numpy(), lse.double().cpu().numpy(), tuple(np.stack([x[i] for x in refs]) for i in range(4)))
            hkv.hkv_decode_plan_destroy(plan)
        parent = rng.integers(0, beams, beams)
        out = hkv.kv_pool_fork(pool.handle, np.concatenate(pages), [n] * beams, parent, release=True)
        pages = [list(x) for x in np.split(out, beams)]
        history = [[list(history[p][0]), list(history[p][1])] for p in parent]
    hkv.kv_pool_release(pool.handle, np.concatenate([prompt, *pages]))
    assert hkv.kv_pool_num_free(pool.handle) == 80
    pool.close()


def test_the_readmes_lines():
    """What README.md has a program do with pages, run as it is written there."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        text = f.read()
    lines = textwrap.dedent(text[text.index("    # a prompt that no call waits for"): text.index("    hkv.kv_cache_release(cache, pages)")])
    warm, cold = make(40, 2, hkv.BF16, 16, 1), make(20, 2, hkv.FP4_E2M1, 16, 2)
    ids = hkv.kv_pool_alloc(warm.handle, 30)
    hkv.kv_pool_release(warm.handle, ids[3:9])
    pages, prompt, back, n = ids[20:25], ids[10:14], ids[14:18], 70
    at = lambda x: torch.from_numpy(np.asarray(x, dtype=np.int64)).cuda()
    content = warm.k.view(40, -1)[at(pages)].clone()
    names = dict(hkv=hkv, pool=warm.handle, four_bit_pool=cold.handle, cold_pages=np.arange(5, 9, dtype=np.int32), prompt_pages=prompt, warm_pages=back, pages=pages, n=n)
    exec(lines, names)
    new, branches = names["new_ids"], names["branches"]
    assert list(names["pages"]) == list(new[pages]) and branches.shape == (4, 5)
    for b in branches:  # four full pages of their own sequence's, and a copy of the fifth
        assert list(b[:4]) == list(pages[:4]) and torch.equal(warm.k.view(40, -1)[at(new[b])], content)
    assert len({int(b[4]) for b in branches} | {int(pages[4])}) == 5
    assert torch.equal(warm.k.view(40, -1)[at(names["pages"])], content)
    warm.close()
    cold.close()

"""The calls around a step's attention against plain 64-bit forms: stores of projection rows (norm, rotation, pool), weights of cached
keys, eviction; then all of them in a row, as a serving loop makes them."""
import numpy as np
import pytest
import torch

from paper_2603_16104_amd import binding as hkv

from operators_plain import ROW, Pool, blocks_of, check_rows, check_store, evicted, key_weights, normed, turned

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))


@pytest.fixture(scope="module", autouse=True)
def built():
    assert torch.cuda.is_available(), "these tests need an MI355X"
    hkv.lib()


class Rows:
    """Projection rows of a step, as one fused product leaves them or apart, and what they become."""

    def __init__(self, n, hq, heads, dtype, seed, *, norm=True, rotary=128, interleaved=False, axes=1, fused=True, in_place=False, big=1.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        act = torch.float32 if dtype == hkv.FP32 else torch.bfloat16
        self.dtype = hkv.FP32 if dtype == hkv.FP32 else hkv.BF16
        width = (hq + 2 * heads) * 128
        rand = lambda *s: torch.randn(*s, device="cuda", generator=g) * big  # noqa: E731
        if fused:
            self.all = rand(n, width + 64).to(act)
            self.q, self.k, self.v = (x.unflatten(1, (-1, 128)) for x in self.all[:, :width].split([hq * 128, heads * 128, heads * 128], dim=1))
        else:
            self.q, self.k, self.v = (rand(n, h, 128).to(act) for h in (hq, heads, heads))
        self.q_in = self.q.clone()
        self.q_out = self.q if in_place else torch.full((n, hq, 128), float("nan"), dtype=act, device="cuda")
        self.qw, self.kw = ((1 + 0.3 * torch.randn(128, device="cuda", generator=g)).to(act) if norm else None for _ in range(2))
        self.eps, self.rotary, self.interleaved = 1e-5, rotary, interleaved
        self.inv_freq = 5e5 ** (-torch.arange(0, max(rotary, 2), 2, dtype=torch.float64, device="cuda") / max(rotary, 2))
        self.axis = (np.arange(rotary // 2) * axes // max(1, rotary // 2)).astype(np.int32) if axes > 1 else None
        self.positions = torch.randint(-50, 100000, (axes, n), dtype=torch.int32, device="cuda", generator=g) if axes > 1 else None
        self.arg = hkv.qkv_rows(self.q, self.k, self.v, self.q_out, q_norm=self.qw, k_norm=self.kw, eps=self.eps, rotary_dim=rotary,
                                inv_freq=self.inv_freq if rotary else None, interleaved=interleaved, positions=self.positions, axis=self.axis)

    def exact(self, places):
        """q and k as they should come out, with the sizes their errors go by; places: a position for each row."""
        if self.rotary == 0:
            q, k = normed(self.q_in, self.qw, self.eps), normed(self.k, self.kw, self.eps)
            return q, np.abs(q), k, np.abs(k)
        pos = self.positions.cpu().double().numpy() if self.positions is not None else np.asarray(places, dtype=np.float64)[None]
        axis = self.axis if self.axis is not None else np.zeros(self.rotary // 2, dtype=np.int64)
        angle = np.longdouble(pos[axis].T) * np.longdouble(self.inv_freq.cpu().numpy()[None, : self.rotary // 2])
        angle = np.float64(np.fmod(angle, 2 * np.longdouble("3.14159265358979323846264338327950288")))
        q, qs = turned(normed(self.q_in, self.qw, self.eps), angle, self.interleaved)
        k, ks = turned(normed(self.k, self.kw, self.eps), angle, self.interleaved)
        return q, qs, k, ks

    def check(self, pool, before, rows, places, units, what=""):
        q, qs, k, ks = self.exact(places)
        got = self.q_out.float().cpu().double().numpy()
        check_rows(got[rows], q[rows], qs[rows], self.dtype, what + " q")
        if self.q_out is not self.q:
            others = np.setdiff1d(np.arange(len(got)), rows)
            assert np.isnan(got[others]).all(), what + ": rows that the plan does not name"
        check_store(pool, before, units, k, ks, self.v.float().cpu().double().numpy(), what)


def units_of(blocks, first, rows):
    """(block, low slot, rows) of tokens first .. of a sequence with these blocks."""
    out, i = [], 0
    while i < len(rows):
        low = (first + i) % 16
        n = min(16 - low, len(rows) - i)
        out.append((int(blocks[(first + i) // 16]), low, np.asarray(rows[i: i + n])))
        i += n
    return out


# ------------------------------------------------------------------------------------------------ store: prefill
STORE = [  # dtype, (q heads, kv heads), page size, (prefix, new) of the requests, rows
    (hkv.BF16, (8, 2), 16, [(0, 1), (32, 33), (16, 0), (48, 16)], dict()),
    (hkv.BF16, (5, 1), 32, [(7, 20), (0, 70)], dict(norm=False, rotary=64)),
    (hkv.BF16, (32, 2), 16, [(30, 5)], dict(rotary=96, interleaved=True, fused=False)),
    (hkv.BF16, (3, 3), 64, [(100, 100), (15, 2)], dict(axes=3, rotary=48)),
    (hkv.BF16, (4, 4), 16, [(0, 40)], dict(rotary=0, in_place=True, fused=False)),
    (hkv.BF16, (14, 7), 128, [(120, 17)], dict(norm=False, rotary=16)),
    (hkv.FP8_E4M3, (8, 2), 16, [(0, 1), (32, 33), (16, 0), (48, 16)], dict()),
    (hkv.FP8_E4M3, (10, 2), 32, [(7, 20), (9, 3)], dict(norm=False, interleaved=True)),
    (hkv.FP8_E4M3, (16, 1), 16, [(1, 50)], dict(norm=False, axes=4, big=0.01)),
    (hkv.FP8_E4M3, (3, 3), 64, [(21, 60)], dict(rotary=112, big=30.0)),
    (hkv.FP32, (8, 2), 16, [(0, 1), (32, 33), (16, 0), (48, 16)], dict(fused=False, in_place=True)),
    (hkv.FP32, (5, 1), 32, [(5, 40)], dict(norm=False, interleaved=True, rotary=32, axes=2)),
    # more blocks x heads than go with queries apart
    (hkv.BF16, (15, 5), 16, [(20, 2000), (0, 1700), (3, 1)], dict(fused=False, in_place=True)),
    (hkv.FP8_E4M3, (14, 7), 32, [(20, 2000), (0, 700), (3, 1)], dict(rotary=64)),
    (hkv.FP32, (6, 6), 16, [(20, 2000), (0, 1700), (3, 1)], dict(interleaved=True)),
]


@pytest.mark.parametrize("case", range(len(STORE)))
def test_store_of_a_prefill(case):
    dtype, (hq, heads), page, reqs, how = STORE[case]
    n_pages = [-(-(p + n) // page) for p, n in reqs]
    order = np.random.default_rng(case).permutation(sum(n_pages) + 3).astype(np.int32)
    pool = Pool(sum(n_pages) + 3, heads, dtype, page, seed=case)
    table = np.full((len(reqs), max(n_pages)), -1, dtype=np.int32)
    for r, e in enumerate(np.cumsum(n_pages)):
        table[r, : n_pages[r]] = order[e - n_pages[r]: e]
    cu = np.concatenate([[0], np.cumsum([n for _, n in reqs])])
    plan = hkv.hkv_prefill_plan_create(pool.handle, cu, table, [p + n for p, n in reqs], hq)
    x = Rows(int(cu[-1]), hq, heads, dtype, case, **how)
    before = pool.snapshot()
    hkv.hkv_prefill_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    places = np.concatenate([np.arange(p, p + n) for p, n in reqs])
    units = [u for r, (p, n) in enumerate(reqs) for u in units_of(blocks_of(table[r, : n_pages[r]], page), p, np.arange(cu[r], cu[r + 1]))]
    x.check(pool, before, np.arange(cu[-1]), places, units)
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3])
def test_store_of_more_requests_than_a_launch_takes_and_of_rows_of_their_own(dtype):
    n_req, hq, heads = 300, 4, 2
    rng = np.random.default_rng(1)
    new = rng.integers(0, 20, n_req)
    new[[0, 127, 128, 255, 299]] = [0, 0, 0, 17, 0]
    prefix = rng.integers(0, 20, n_req)
    table = np.arange(3 * n_req, dtype=np.int32).reshape(n_req, 3)
    begin = np.cumsum(np.concatenate([[5], new[:-1] + rng.integers(0, 3, n_req - 1)]))
    pool = Pool(3 * n_req, heads, dtype, seed=2)
    plan = hkv.hkv_prefill_plan_create_rows(pool.handle, begin, new, table, prefix + new, hq)
    x = Rows(int(begin[-1] + new[-1]) + 4, hq, heads, dtype, 3)
    before = pool.snapshot()
    hkv.hkv_prefill_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    places = np.zeros(len(x.q))
    rows, units = [], []
    for r in range(n_req):
        mine = np.arange(begin[r], begin[r] + new[r])
        places[mine] = np.arange(prefix[r], prefix[r] + new[r])
        rows.append(mine)
        units += units_of(table[r], int(prefix[r]), mine)
    x.check(pool, before, np.concatenate(rows), places, units)
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


def test_requests_of_a_prefill_that_write_to_one_block_are_refused():
    pool = Pool(8, 2, hkv.BF16)
    x = Rows(10, 4, 2, hkv.BF16, 0)
    for table, lens, ok in (([[0, 1], [0, 1]], [20, 20], False), ([[0, 1], [0, 2]], [21, 21], True), ([[0, 1], [0, 2]], [20, 17], False)):
        plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 5, 10], table, lens, 4)
        if ok:
            hkv.hkv_prefill_plan_store(plan, x.arg)
        else:
            with pytest.raises(hkv.HkvError) as e:
                hkv.hkv_prefill_plan_store(plan, x.arg)
            assert e.value.code == hkv.EINVAL
        hkv.hkv_prefill_plan_destroy(plan)
    torch.cuda.synchronize()
    pool.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP32])
@pytest.mark.parametrize("at", [-(1 << 31), -1, 0, 131071, 1 << 24, (1 << 31) - 1])
def test_far_positions_are_as_exact_as_near_ones(dtype, at):
    pool = Pool(2, 1, dtype)
    plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 7], [[0]], [7], 2)
    x = Rows(7, 2, 1, dtype, 5, norm=False)
    pos = torch.full((7,), at, dtype=torch.int32, device="cuda")
    x.positions = pos[None]
    x.arg = hkv.qkv_rows(x.q, x.k, x.v, x.q_out, rotary_dim=128, inv_freq=x.inv_freq, positions=pos)
    before = pool.snapshot()
    hkv.hkv_prefill_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    x.check(pool, before, np.arange(7), None, [(0, 0, np.arange(7))])
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3, hkv.FP32])
def test_a_row_that_is_no_number_spoils_nothing_but_itself(dtype):
    pool = Pool(4, 2, dtype)
    plan = hkv.hkv_prefill_plan_create(pool.handle, [0, 40], [[3, 1, 0]], [40], 8)
    x = Rows(40, 8, 2, dtype, 7, fused=False, rotary=64)
    x.q[20, 3, 100] = float("nan")                       # a dimension that is not turned: the norm spreads it over the head
    x.q[21, 0, 5] = float("inf")
    x.q[22] = 0
    x.k[35, 1, 0] = float("nan")
    x.q_in = x.q.clone()
    before = pool.snapshot()
    hkv.hkv_prefill_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    q, qs, k, ks = x.exact(np.arange(40))
    got = x.q_out.float().cpu().double().numpy()
    bad = np.zeros(got.shape[:2], dtype=bool)
    bad[20, 3] = bad[21, 0] = True
    check_rows(got[~bad], q[~bad], qs[~bad], x.dtype, "q")
    assert np.isnan(got[20, 3]).all() and not np.isfinite(got[21, 0, 5]) and (got[22] == 0).all()
    k[35, 1] = ks[35, 1] = 0
    gk = pool.values()[0]
    blk = np.asarray([3, 1, 0])
    for t in range(40):
        for h in range(2):
            if (t >= 32 and h == 1 and dtype == hkv.FP8_E4M3) or (t, h) == (35, 1):
                continue                                 # the block whose scale it enters
            step = {hkv.BF16: 2.0 ** -8, hkv.FP32: 2.0 ** -24, hkv.FP8_E4M3: 2.0 ** -3}[dtype]
            assert np.abs(gk[blk[t // 16], h, t % 16] - k[t, h]).max() <= step * np.abs(k[t, h]).max() + 2 * ROW * ks[t, h].max(), (t, h)
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


# ------------------------------------------------------------------------------------------------ store: decode
def forest(parent, tokens, page, seed=0, spare=0):
    """(nodes, page ids, blocks per node, pages in all) with shuffled pages."""
    counts = [-(-n // page) for n in tokens]
    order = np.random.default_rng(seed).permutation(sum(counts) + spare).astype(np.int32)
    nodes, begin = [], 0
    for p, n, c in zip(parent, tokens, counts):
        nodes.append((p, begin, c, n))
        begin += c
    blocks = [blocks_of(order[b: b + c], page)[: -(-n // 16)] for _, b, c, n in nodes]
    return np.asarray(nodes, dtype=np.int32), order[:begin], blocks, order[begin:]


def depth_start(parent, tokens):
    start = []
    for p in parent:
        start.append(0 if p < 0 else start[p] + tokens[p])
    return start


DECODE = [  # dtype, heads, page, parents, tokens, last nodes, tokens per request, rows
    (hkv.BF16, (8, 2), 16, [-1, 0, 0, -1], [32, 17, 1, 16], [1, 2, 3, 0], 1, dict()),
    (hkv.BF16, (16, 1), 32, [-1, 0, 0], [33, 17, 64], [1, 2], 1, dict(norm=False, interleaved=True)),
    (hkv.BF16, (15, 1), 16, [-1, 0], [33, 31], [1], 1, dict(rotary=32)),
    (hkv.BF16, (6, 2), 16, [-1, 0, 0], [33, 31, 5], [2, 1], 5, dict(axes=3)),
    (hkv.BF16, (8, 2), 64, [-1, 0, 0], [64, 100, 64], [1, 2], 64, dict(norm=False)),
    (hkv.FP8_E4M3, (8, 2), 16, [-1, 0, 0, -1], [32, 17, 1, 16], [1, 2, 3], 1, dict(big=3.0)),
    (hkv.FP8_E4M3, (16, 1), 16, [-1, 0, 0], [32, 20, 31], [1, 2], 1, dict(norm=False, axes=2, big=0.1)),
    (hkv.FP8_E4M3, (8, 2), 32, [-1, 0, 0], [33, 31, 18], [2, 1], 18, dict(big=4.0)),
    (hkv.FP32, (8, 2), 16, [-1, 0, 0], [32, 17, 3], [1, 2], 1, dict()),
    (hkv.FP32, (4, 1), 32, [-1, 0, 0], [32, 17, 40], [1, 2], 16, dict(interleaved=True, norm=False)),
    # around the numbers of tokens at which rows are dealt out another way; heads that do not fill the last sixteen of rows; more than one sixteen of K's rows
    (hkv.BF16, (5, 5), 16, [-1, 0, 0], [20, 2, 33], [1, 2], 2, dict(fused=False, in_place=True)),
    (hkv.BF16, (14, 7), 16, [-1, 0, 0], [20, 3, 33], [1, 2], 3, dict(fused=False, in_place=True, rotary=64)),
    (hkv.BF16, (20, 20), 32, [-1, 0, 0], [20, 17, 33], [1, 2], 1, dict(rotary=0)),
    (hkv.BF16, (8, 2), 16, [-1, 0], [20, 40], [1], 24, dict(interleaved=True, rotary=96)),
    (hkv.BF16, (8, 2), 16, [-1, 0], [20, 41], [1], 25, dict()),
    (hkv.FP8_E4M3, (20, 20), 16, [-1, 0, 0], [20, 31, 16], [1, 2], 1, dict(big=20.0)),
    (hkv.FP8_E4M3, (9, 3), 16, [-1, 0, 0], [20, 2, 33], [1, 2], 2, dict(fused=False, in_place=True, big=5.0)),
    (hkv.FP8_E4M3, (6, 2), 64, [-1, 0], [20, 50], [1], 24, dict(axes=4, norm=False)),
    (hkv.FP8_E4M3, (6, 2), 16, [-1, 0], [20, 70], [1], 64, dict(big=2.0)),
    (hkv.FP32, (20, 20), 16, [-1, 0, 0], [32, 17, 40], [1, 2], 1, dict(rotary=48)),
    (hkv.FP32, (6, 2), 16, [-1, 0, 0], [32, 17, 40], [1, 2], 2, dict(fused=False, in_place=True)),
    (hkv.FP32, (6, 2), 16, [-1, 0, 0], [32, 17, 40], [1, 2], 7, dict(axes=2)),
]


@pytest.mark.parametrize("case, mapped", [(i, m) for i, c in enumerate(DECODE) for m in (False, True) if not (m and c[0] == hkv.FP32)])  # (those have their rows in order)
def test_store_of_a_decode_plan(case, mapped):
    dtype, (hq, heads), page, parent, tokens, leaves, T, how = DECODE[case]
    nodes, pages, blocks, _ = forest(parent, tokens, page, case)
    pool = Pool(len(pages) + 2, heads, dtype, page, seed=case)
    n = len(leaves) * T
    row_of = np.random.default_rng(case).permutation(n + 3)[:n].astype(np.int32) if mapped else np.arange(n)
    visible = None if T <= 16 else np.tile(np.asarray([(1 << (t + 1)) - 1 for t in range(T)], dtype=np.uint64), len(leaves))
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, nodes, pages, leaves, hq, tokens_per_req=T, visible=visible, q_rows=row_of if mapped else None)
    x = Rows(n + 3, hq, heads, dtype, case, **how)
    before = pool.snapshot()
    hkv.hkv_decode_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    start, places, units = depth_start(parent, tokens), np.zeros(n + 3), []
    for r, v in enumerate(leaves):
        mine = row_of[r * T: (r + 1) * T]
        places[mine] = start[v] + tokens[v] - T + np.arange(T)
        units += units_of(blocks[v], tokens[v] - T, mine)
    x.check(pool, before, row_of, places, units)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


def test_decode_store_refuses_what_would_race():
    pool = Pool(8, 2, hkv.BF16)
    mine = hkv.kv_pool_alloc(pool.handle, 6)
    x = Rows(4, 8, 2, hkv.BF16, 0)
    nodes = np.asarray([(-1, 0, 1, 16), (0, 1, 1, 5), (0, 2, 1, 0)], dtype=np.int32)[:2]
    for leaves, pages, ok in (([1, 1], mine[:2], False), ([1], mine[:2], True)):
        plan = hkv.hkv_decode_plan_create(pool.handle, nodes, pages, leaves, 8)
        if ok:
            hkv.hkv_decode_plan_store(plan, x.arg)
            hkv.kv_pool_retain(pool.handle, mine[1:2])   # from now on somebody else's, too
        with pytest.raises(hkv.HkvError) as e:
            hkv.hkv_decode_plan_store(plan, x.arg)
        assert e.value.code == hkv.EINVAL
        hkv.hkv_decode_plan_destroy(plan)
    empty = hkv.hkv_decode_plan_create(pool.handle, [(-1, 0, 1, 16), (0, 1, 0, 0)], mine[:1], [1], 8)
    with pytest.raises(hkv.HkvError) as e:
        hkv.hkv_decode_plan_store(empty, x.arg)
    assert e.value.code == hkv.EINVAL
    hkv.hkv_decode_plan_destroy(empty)
    torch.cuda.synchronize()
    pool.close()


@pytest.mark.parametrize("n_req, large", [(3, 0), (3, 1), (256, 0), (257, 0)])
@pytest.mark.parametrize("dtype, page", [(hkv.BF16, 16), (hkv.FP8_E4M3, 32)])
def test_append_of_projections_through_a_generation(dtype, page, n_req, large):
    """A growing plan's steps with the store in the append: pool, queries and attention as from append, then store, on a twin; and the
    first and last step against the formula."""
    hq, heads, steps = 6, 2, 20
    rng = np.random.default_rng(n_req)
    own = rng.integers(1, 40, n_req)
    parent, tokens = [-1] + [0] * n_req, [48, *own.tolist()]
    nodes, pages, blocks, spare = forest(parent, tokens, page, 1, spare=2 * n_req + 2)
    twins = [Pool(len(pages) + len(spare), heads, dtype, page, seed=4) for _ in range(2)]
    plans = [hkv.hkv_decode_plan_create_ex(p.handle, nodes, pages, np.arange(1, n_req + 1), hq, reserve_tokens=steps, large_batch_updates=large) for p in twins]
    ws = [torch.empty(hkv.hkv_decode_plan_workspace_bytes(p) + 256, dtype=torch.uint8, device="cuda") for p in plans]
    length, at = own.copy(), [list(b) for b in blocks[1:]]
    opened, spare = 0, list(spare)
    for step in range(steps):
        ids = np.full(n_req, -1, dtype=np.int32)
        for r in np.flatnonzero(length % page == 0):
            ids[r] = spare[opened]
            opened += 1
            at[r] = at[r][: -(-int(length[r]) // 16)] + list(blocks_of([ids[r]], page))
        for r in np.flatnonzero((length % 16 == 0) & (length % page != 0)):
            if len(at[r]) <= length[r] // 16:
                at[r].append(at[r][-1] + 1)
        x = [Rows(n_req, hq, heads, dtype, 100 + step, rotary=64) for _ in range(2)]
        before = twins[0].snapshot() if step in (0, steps - 1) else None
        hkv.hkv_decode_plan_append_qkv(plans[0], ids, x[0].arg)
        hkv.hkv_decode_plan_append(plans[1], ids)
        hkv.hkv_decode_plan_store(plans[1], x[1].arg)
        out = [torch.zeros_like(y.q_out) for y in x]
        lse = [torch.zeros(n_req, hq, device="cuda") for _ in x]
        for i in range(2):
            hkv.attn_decode_plan_run(plans[i], x[i].q_out, SCALE, out[i], lse[i], ws[i], ws[i].numel())
        torch.cuda.synchronize()
        if before is not None:
            units = [(int(at[r][length[r] // 16]), int(length[r] % 16), np.asarray([r])) for r in range(n_req)]
            x[0].check(twins[0], before, np.arange(n_req), 48 + length, units, f"step {step}")
        length += 1
        assert torch.equal(x[0].q_out, x[1].q_out) and torch.equal(out[0], out[1]) and torch.equal(lse[0], lse[1]), step
        assert torch.isfinite(lse[0]).all()
    assert torch.equal(twins[0].k.view(torch.uint8), twins[1].k.view(torch.uint8)) and torch.equal(twins[0].v.view(torch.uint8), twins[1].v.view(torch.uint8))
    with pytest.raises(hkv.HkvError) as e:
        hkv.hkv_decode_plan_append_qkv(plans[0], np.zeros(n_req, dtype=np.int32) if not (length % page == 0).any() else np.arange(n_req, dtype=np.int32), x[0].arg)
    assert e.value.code in (hkv.ENOMEM, hkv.EINVAL)
    for p in plans:
        hkv.hkv_decode_plan_destroy(p)
    for p in twins:
        p.close()


def test_append_refuses_two_new_tokens_in_one_block():
    pool = Pool(8, 2, hkv.BF16)
    nodes = [(-1, 0, 1, 16), (0, 1, 1, 16), (0, 2, 1, 16)]
    plan = hkv.hkv_decode_plan_create_growing(pool.handle, nodes, [0, 1, 2], [1, 2], 8, 8)
    x = Rows(2, 8, 2, hkv.BF16, 0)
    for ids, want in (([3, 3], hkv.EINVAL), (None, hkv.EINVAL), ([3, 8], hkv.ERANGE)):
        with pytest.raises(hkv.HkvError) as e:
            hkv.hkv_decode_plan_append_qkv(plan, ids, x.arg)
        assert e.value.code == want
    hkv.hkv_decode_plan_append_qkv(plan, [3, 4], x.arg)
    torch.cuda.synchronize()
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


# ------------------------------------------------------------------------------------------------ weights of cached keys
def weight_nodes(parent, tokens, blocks, leaves, T, masks=None):
    """The nodes as operators_plain.key_weights takes them."""
    out = []
    for v, n in enumerate(tokens):
        rows, seen = [], []
        for r, leaf in enumerate(leaves):
            u = leaf
            while u >= 0 and u != v:
                u = parent[u]
            if u != v:
                continue
            for t in range(T):
                rows.append(r * T + t)
                s = np.ones(n, dtype=bool)
                if leaf == v:
                    m = (1 << (t + 1)) - 1 if masks is None else int(masks[r * T + t])
                    s[n - T:] = [(m >> j) & 1 for j in range(T)]
                seen.append(s)
        out.append((blocks[v], n, np.asarray(rows, dtype=np.int64), np.asarray(seen).reshape(len(rows), n), v in leaves))
    return out


def path_lse(k_values, parent, tokens, blocks, leaves, q, T, heads, masks=None):
    nodes = weight_nodes(parent, tokens, blocks, leaves, T, masks)
    lse = np.full(q.shape[:2], -np.inf)
    G = q.shape[1] // heads
    for b, n, rows, seen, _ in nodes:
        for h in range(heads):
            if n and len(rows):
                t = np.arange(n)
                x = np.einsum("rgd,td->rgt", q[rows][:, h * G: (h + 1) * G], k_values[b[t // 16], h, t % 16]) * SCALE
                x = np.where(seen[:, None], x, -np.inf)
                with np.errstate(divide="ignore"):
                    lse[rows, h * G: (h + 1) * G] = np.logaddexp(lse[rows, h * G: (h + 1) * G], np.log(np.exp(x).sum(-1)))
    return lse


# Scores below 40 in size are sums of 128 exact products of bf16 values in fp32, their exponents carry 40 * 2^-24 * (8 + 4 roundings and
# lse's own), the exponential 2^-22, the sum over rows (at most 2048 here) less than 2^-13 at worst, 2^-18 where errors do not line up;
# everything in the sum is positive.
WEIGHT_TOL = 2.0 ** -13

WEIGHTS = [  # dtype, heads, page, parents, tokens, last nodes, tokens per request, decay, n_new
    (hkv.BF16, (8, 2), 16, [-1, 0, 0, 0], [300, 17, 1, 129], [1, 2, 3], 1, 1.0, 1),
    (hkv.BF16, (5, 1), 32, [-1, 0, 1, 1, 0], [33, 70, 5, 0, 128], [2, 3, 4, 4, 1], 1, 0.5, 0),
    (hkv.BF16, (16, 1), 16, [-1, -1, 1], [16, 47, 31], [2, 0, 2], 1, 0.0, 1),
    (hkv.BF16, (1, 1), 16, [-1], [1], [0], 1, 1.0, 1),
    (hkv.BF16, (8, 2), 16, [-1, 0, 0], [130, 140, 9], [1, 2], 9, 1.0, 9),
    (hkv.BF16, (6, 2), 64, [-1, 0, 0], [40, 64, 130], [1, 2], 64, 0.25, 30),
    (hkv.BF16, (16, 1), 16, [-1] + [0] * 60, [500] + [3] * 60, list(range(1, 61)), 1, 1.0, 0),
    (hkv.FP8_E4M3, (8, 2), 16, [-1, 0, 0, 0], [300, 17, 1, 129], [1, 2, 3], 1, 1.0, 1),
    (hkv.FP8_E4M3, (10, 2), 32, [-1, 0, 0], [33, 31, 200], [1, 2], 21, 0.0, 21),
    (hkv.FP8_E4M3, (8, 1), 16, [-1] + [0] * 40, [260] + [20] * 40, list(range(1, 41)), 1, 0.9, 1),
    # a workgroup's keys are 64, 128, 256 and 512 of one long node, its rows less and more than it holds at a time; then wavefronts of 96 keys
    (hkv.BF16, (24, 8), 16, [-1], [4003], [0], 8, 1.0, 3),
    (hkv.FP8_E4M3, (24, 8), 32, [-1], [7001], [0], 8, 0.5, 0),
    (hkv.BF16, (24, 8), 64, [-1], [13001], [0], 6, 0.0, 6),
    (hkv.FP8_E4M3, (8, 2), 16, [-1] + [0] * 80, [40001] + [16] * 80, list(range(1, 81)), 1, 1.0, 1),
    (hkv.BF16, (8, 8), 16, [-1, 0], [35000, 12345], [1], 2, 0.9, 1),
    # fp32 pools: 4 partial sums of 32 products, each with a rounding, and 3 more: 35 * 2^-24 of the sum of |products| (below 40) in the exponent, the rest as above
    (hkv.FP32, (8, 2), 16, [-1, 0, 0, 0], [304, 17, 1, 129], [1, 2, 3], 1, 1.0, 1),
    (hkv.FP32, (16, 1), 32, [-1, 0, 1, 1, 0], [32, 64, 5, 0, 128], [2, 3, 4, 4, 1], 1, 0.5, 0),
    (hkv.FP32, (6, 2), 64, [-1, 0, 0], [64, 64, 270], [1, 2], 9, 0.0, 9),
    (hkv.FP32, (1, 1), 16, [-1], [1], [0], 1, 1.0, 1),
    (hkv.FP32, (8, 2), 16, [-1] + [0] * 40, [2000] + [20] * 40, list(range(1, 41)), 1, 0.9, 1),
]


# (plans over fp32 pools have no rows of their own)
@pytest.mark.parametrize("case, mapped", [(c, m) for c in range(len(WEIGHTS)) for m in (False, True) if not m or WEIGHTS[c][0] != hkv.FP32])
def test_weights_of_cached_keys(case, mapped):
    dtype, (hq, heads), page, parent, tokens, leaves, T, decay, n_new = WEIGHTS[case]
    nodes, pages, blocks, _ = forest(parent, tokens, page, case)
    pool = Pool(len(pages) + 2, heads, dtype, page, seed=case)
    rng = np.random.default_rng(case)
    n = len(leaves) * T
    masks = None
    if T > 16:  # a tree of drafts: every token under one of the earlier ones
        masks = np.zeros(n, dtype=np.uint64)
        for r in range(len(leaves)):
            for t in range(T):
                up = int(rng.integers(-1, t)) if t else -1
                masks[r * T + t] = (1 << t) | (int(masks[r * T + up]) if up >= 0 else 0)
    row_of = rng.permutation(n + 3)[:n].astype(np.int32) if mapped else np.arange(n)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, nodes, pages, leaves, hq, tokens_per_req=T, visible=masks, q_rows=row_of if mapped else None)
    g = torch.Generator(device="cuda")
    g.manual_seed(case)
    q = (2 * torch.randn(n + 3, hq, 128, device="cuda", generator=g)).to(torch.float32 if dtype == hkv.FP32 else torch.bfloat16)
    q64 = q.float().cpu().double().numpy()[row_of]
    kv = pool.values()[0]
    lse64 = path_lse(kv, parent, tokens, blocks, leaves, q64, T, heads, masks)
    lse = torch.full((n + 3, hq), float("nan"), device="cuda")
    lse[torch.from_numpy(np.asarray(row_of, dtype=np.int64)).cuda()] = torch.from_numpy(lse64).float().cuda()
    w = torch.rand(pool.blocks, heads, 16, device="cuda", generator=g)
    if decay == 0:
        w.fill_(float("nan"))                            # is not read
    for v in set(leaves):                                # nor are new tokens' slots
        for t in range(max(0, tokens[v] - n_new), tokens[v]):
            w[blocks[v][t // 16], :, t % 16] = float("nan")
    first = w.clone()
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, decay, n_new, w)
    torch.cuda.synchronize()
    use = lse.cpu().double().numpy()[row_of]
    listed = weight_nodes(parent, tokens, blocks, leaves, T, masks)
    want = key_weights(kv, listed, q64, use, SCALE, heads, first.cpu().numpy(), decay, n_new, T)
    got = w.cpu().double().numpy()
    live = np.zeros((pool.blocks, 16), dtype=bool)
    for b, m, rows, _, _ in listed:
        if len(rows):
            live[b[np.arange(m) // 16], np.arange(m) % 16] = True
    live = np.broadcast_to(live[:, None], got.shape)
    was = first.cpu().double().numpy()
    assert np.array_equal(got[~live], was[~live], equal_nan=True), "slots of no key"
    assert np.isfinite(got[live]).all() and (np.abs(got[live] - want[live]) <= WEIGHT_TOL * want[live]).all(), np.max(np.abs(got[live] - want[live]) / want[live])
    if decay == 0:                                       # every row gave away 1 in all
        assert abs(got[live].sum() - n * hq) <= 1e-4 * n * hq
    again = first.clone()
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, decay, n_new, again)
    torch.cuda.synchronize()
    assert np.array_equal(again.cpu().numpy(), w.cpu().numpy(), equal_nan=True)
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3])
def test_rows_without_a_finite_lse_add_nothing(dtype):
    parent, tokens, leaves, hq, heads = [-1, 0, 0, 0], [100, 20, 20, 20], [1, 2, 3], 8, 2
    nodes, pages, blocks, _ = forest(parent, tokens, 16)
    pool = Pool(len(pages), heads, dtype)
    plan = hkv.hkv_decode_plan_create(pool.handle, nodes, pages, leaves, hq)
    q = torch.randn(3, hq, 128, device="cuda").to(torch.bfloat16)
    q[0, 2] = float("nan")
    q[1, 7, 3] = float("inf")
    lse = torch.full((3, hq), 3.0, device="cuda")
    lse[0, 2], lse[1, 7], lse[2, 0] = float("nan"), float("inf"), -float("inf")
    w = torch.zeros(pool.blocks, heads, 16, device="cuda")
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, 1.0, 1, w)
    torch.cuda.synchronize()
    q64, l64 = q.float().cpu().double().numpy(), lse.cpu().double().numpy()
    want = key_weights(pool.values()[0], weight_nodes(parent, tokens, blocks, leaves, 1), q64, l64, SCALE, heads, np.zeros(w.shape), 1.0, 1, 1)
    got = w.cpu().double().numpy()
    assert np.isfinite(got).all() and (np.abs(got - want) <= WEIGHT_TOL * want).all()
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("n_req", [2, 12])
def test_a_key_that_is_no_number_gets_nothing(n_req):
    """Drafted tokens of a tree: a NaN or infinite key spoils the rows that see it and no other key's sum."""
    hq, heads, T, n = 4, 1, 3, 20
    pool = Pool(2 * n_req, heads, hkv.BF16)
    nodes = [(-1, 2 * r, 2, n) for r in range(n_req)]
    masks = np.tile(np.asarray([1, 3, 5], dtype=np.uint64), n_req)       # two tokens under the first
    plan = hkv.hkv_decode_plan_create_tree(pool.handle, nodes, np.arange(2 * n_req), np.arange(n_req), T, masks, hq)
    k = pool.k.view(2 * n_req, 4, 16, 32)
    k[1, 0, 2, 7] = float("nan")                                         # request 0's drafted token 1, seen by itself alone
    k[3, 0, 3, 0] = float("inf")                                         # request 1's drafted token 2
    q = torch.randn(n_req * T, hq, 128, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(n_req * T, hq, device="cuda")
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
    hkv.attn_decode_plan_run(plan, q, SCALE, out, lse, ws, ws.numel())
    lse[1] = float("nan")
    lse[T + 2] = float("inf")
    w = torch.zeros(2 * n_req, heads, 16, device="cuda")
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, 1.0, 3, w)
    torch.cuda.synchronize()
    got = w.cpu().double().numpy()[:, 0].reshape(n_req, 32)[:, :n]
    assert np.isfinite(got).all() and got[0, 18] == 0 and got[1, 19] == 0
    gave = np.full(n_req, float(T * hq))
    gave[:2] -= hq                                                       # the spoilt rows
    assert np.abs(got.sum(1) - gave).max() <= 1e-3 * T * hq
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


def test_slots_behind_a_node_may_hold_anything():
    pool = Pool(6, 1, hkv.BF16)
    nodes = [(-1, 0, 3, 35), (0, 3, 1, 3)]
    plan = hkv.hkv_decode_plan_create(pool.handle, nodes, [4, 2, 0, 5], [1], 4)
    k = pool.k.view(6, 4, 16, 32)
    k[0, :, 3:], k[5, :, 3:] = float("nan"), float("nan")
    q = torch.randn(1, 4, 128, device="cuda").to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(1, 4, device="cuda")
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan), dtype=torch.uint8, device="cuda")
    w = torch.full((6, 1, 16), float("nan"), device="cuda")
    hkv.attn_decode_plan_run(plan, q, SCALE, out, lse, ws, ws.numel())
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, 0.0, 0, w)
    torch.cuda.synchronize()
    got = w.cpu().double().numpy()[:, 0]
    live = np.concatenate([got[4], got[2], got[0, :3], got[5, :3]])
    assert abs(live.sum() - 4) <= 1e-3 and np.isnan(got[0, 3:]).all() and np.isnan(got[5, 3:]).all() and np.isnan(got[1]).all()
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("n_req, large", [(4, 0), (4, 1)])
def test_weights_through_a_generation(n_req, large):
    """A growing plan whose leaves pass from one chunk of keys to the next: after every step each key holds what all steps gave it."""
    hq, heads, steps, page = 8, 2, 140, 16
    own = np.asarray([1, 127, 16, 250])
    parent, tokens = [-1] + [0] * n_req, [30, *own.tolist()]
    nodes, pages, blocks, spare = forest(parent, tokens, page, 3, spare=n_req * 10)
    pool = Pool(len(pages) + len(spare), heads, hkv.BF16, page)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, nodes, pages, np.arange(1, n_req + 1), hq, reserve_tokens=steps, large_batch_updates=large)
    hkv.hkv_decode_plan_append(plan, np.where(own % page == 0, spare[:n_req], -1))
    at = [list(b) + ([int(spare[r])] if own[r] % page == 0 else []) for r, b in enumerate(blocks[1:])]
    own, taken = own + 1, n_req
    hkv.hkv_decode_plan_track_weights(plan)              # a plan that has grown already
    w = torch.zeros(pool.blocks, heads, 16, device="cuda")
    for r in range(n_req):
        w[int(at[r][(own[r] - 1) // 16]), :, int((own[r] - 1) % 16)] = float("nan")
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
    kv = pool.values()[0]
    want = np.zeros(w.shape)
    for step in range(steps):
        if step:
            ids = np.full(n_req, -1, dtype=np.int32)
            for r in np.flatnonzero(own % page == 0):
                ids[r] = spare[taken]
                at[r].append(int(spare[taken]))
                taken += 1
            for r in range(n_req):
                w[int(at[r][own[r] // 16]), :, int(own[r] % 16)] = float("nan")   # what a used page may hold
            hkv.hkv_decode_plan_append(plan, ids)
            own = own + 1
        q = torch.randn(n_req, hq, 128, device="cuda").to(torch.bfloat16)
        out, lse = torch.empty_like(q), torch.empty(n_req, hq, device="cuda")
        hkv.attn_decode_plan_run(plan, q, SCALE, out, lse, ws, ws.numel())
        hkv.attn_decode_plan_weights(plan, q, SCALE, lse, 0.75, 1, w)
        torch.cuda.synchronize()
        lens = [30, *own.tolist()]
        listed = weight_nodes(parent, lens, [blocks[0]] + [np.asarray(a) for a in at], list(range(1, n_req + 1)), 1)
        want = key_weights(kv, listed, q.float().cpu().double().numpy(), lse.cpu().double().numpy(), SCALE, heads, want, np.float64(0.75), 1, 1)
        if step % 20 == 0 or step == steps - 1:
            got = w.cpu().double().numpy()
            assert (np.abs(got - want) <= WEIGHT_TOL * np.abs(want)).all(), step
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


# ------------------------------------------------------------------------------------------------ eviction
EVICT = [  # dtype, kv heads, page, tokens, keep, first, recent, weights
    (hkv.BF16, 2, 16, [100, 17, 1], [37, 17, 1], 1, 0, "plain"),
    (hkv.BF16, 3, 32, [64, 33, 0, 5], [1, 20, 0, 0], 0, 0, "ties"),
    (hkv.BF16, 1, 16, [5000, 3000], [1111, 48], 4, 32, "plain"),
    (hkv.BF16, 2, 16, [40, 1025, 2049], [39, 1024, 17], 3, 14, "odd"),
    (hkv.BF16, 1, 128, [600], [129], 0, 128, "zeros"),
    (hkv.BF16, 1, 16, [20, 30], [20, 24], 12, 12, "plain"),
    (hkv.FP8_E4M3, 2, 16, [100, 17, 1], [37, 17, 1], 1, 0, "plain"),
    (hkv.FP8_E4M3, 2, 64, [1000, 200], [333, 65], 2, 16, "ties"),
    (hkv.FP32, 2, 16, [100, 17, 40], [37, 17, 20], 0, 5, "odd"),
    # around the lengths at which a thread holds another number of weights, or none
    (hkv.BF16, 1, 16, [2048, 4096, 8192, 8193], [1025, 4095, 4000, 8000], 1, 1024, "ties"),
    (hkv.FP8_E4M3, 1, 64, [16384, 16385, 40000], [16000, 3000, 2000], 5, 1500, "plain"),
    (hkv.BF16, 1, 16, [40000], [17000], 0, 0, "zeros"),
]


@pytest.mark.parametrize("case", range(len(EVICT)))
def test_eviction(case):
    dtype, heads, page, tokens, keep, first, recent, kind = EVICT[case]
    src_n, dst_n = ([-(-n // page) for n in x] for x in (tokens, keep))
    order = np.random.default_rng(case).permutation(sum(src_n) + sum(dst_n) + 2).astype(np.int32)
    src, dst = order[: sum(src_n)], order[sum(src_n): sum(src_n) + sum(dst_n)]
    pool = Pool(len(order), heads, dtype, page, seed=case)
    g = torch.Generator(device="cuda")
    g.manual_seed(case)
    w = torch.randn(pool.blocks, heads, 16, device="cuda", generator=g).exp()
    if kind == "ties":
        w = (w * 2).round() / 4
    elif kind == "zeros":
        w = torch.where(torch.rand(w.shape, device="cuda", generator=g) < 0.5, 0.0, -0.0)
    elif kind == "odd":
        pick = torch.randint(0, 8, w.shape, device="cuda", generator=g)
        for i, x in enumerate((float("nan"), float("inf"), -float("inf"), -1.0, 1e-42)):
            w[pick == i] = x
    was, before = w.cpu().numpy().copy(), pool.snapshot()
    kept = torch.full((heads, sum(keep)), -7, dtype=torch.int32, device="cuda")
    hkv.kv_pool_evict(pool.handle, src, tokens, dst, keep, first, recent, w, kept)
    torch.cuda.synchronize()
    got, now, after = kept.cpu().numpy(), w.cpu().numpy(), pool.snapshot()
    ks, vs = before[2], before[3]
    untouched = np.ones((pool.blocks, heads, 16), dtype=bool)
    col = sb = db = 0
    for n, m, a, b in zip(tokens, keep, src_n, dst_n):
        sblocks, dblocks = blocks_of(src[sb: sb + a], page), blocks_of(dst[db: db + b], page)
        j = np.arange(m)
        for h in range(heads):
            t = evicted(was[:, h], sblocks, n, m, first, recent)
            assert np.array_equal(got[h, col: col + m], t), (n, m, h)
            to, fr = dblocks[j // 16], sblocks[t // 16]
            untouched[to, h, j % 16] = False
            assert np.array_equal(now[to, h, j % 16], was[fr, h, t % 16], equal_nan=True)
            if dtype != hkv.FP8_E4M3:
                for i in range(2):
                    assert np.array_equal(after[i][to, h, j % 16], before[i][fr, h, t % 16])
                continue
            for i, s in ((0, ks), (1, vs)):
                x = before[i][fr, h, t % 16] * s[fr, h][:, None]
                for b0 in range(0, m, 16):
                    z, block = x[b0: b0 + 16], dblocks[b0 // 16]
                    want = np.abs(z).max() / 448 if np.abs(z).max() else 1.0
                    sc = after[2 + i][block, h]
                    assert abs(sc - want) <= 2.0 ** -22 * want
                    # a product, a division and a half step, in normal and subnormal codes
                    assert (np.abs(after[i][block, h, : len(z)] * sc - z) <= 2.0 ** -4 * (1 + 2.0 ** -20) * np.abs(z) + 2.0 ** -10 * sc).all()
        col, sb, db = col + m, sb + a, db + b
    for i in range(2):
        assert np.array_equal(after[i][untouched], before[i][untouched]), "slots that no kept token goes to"
    assert np.array_equal(now[untouched], was[untouched], equal_nan=True)
    pool.close()


def test_eviction_is_refused_while_a_graph_is_captured():
    """... and the capture goes on."""
    pool = Pool(8, 1, hkv.BF16)
    w, kept = torch.rand(8, 1, 16, device="cuda"), torch.full((1, 10), -1, dtype=torch.int32, device="cuda")
    x = torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(hkv.HkvError) as e:
            hkv.kv_pool_evict(pool.handle, [0, 1], [20], [2], [10], 0, 0, w, kept)
        x += 1
    assert e.value.code == hkv.EINVAL
    for i in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert (x == 3).all() and (kept == -1).all()
    hkv.kv_pool_evict(pool.handle, [0, 1], [20], [2], [10], 0, 0, w, kept)
    assert np.array_equal(kept.cpu().numpy()[0], evicted(w.cpu().numpy()[:, 0], np.arange(2), 20, 10, 0, 0))
    pool.close()


def test_eviction_of_more_than_a_staging_slot_describes():
    """Nine long sequences, whose page lists need two slots of the ring; then many short ones."""
    for tokens, keep in (([16 * 7500 - 3] * 9, [100] * 9), ([33] * 700, [17] * 700)):
        src_n, dst_n = -(-tokens[0] // 16), -(-keep[0] // 16)
        n = len(tokens)
        pool = Pool(n * (src_n + dst_n), 1, hkv.FP8_E4M3, seed=1)
        order = np.random.default_rng(0).permutation(n * (src_n + dst_n)).astype(np.int32)
        src, dst = order[: n * src_n], order[n * src_n:]
        w = torch.rand(pool.blocks, 1, 16, device="cuda")
        was = w.cpu().numpy().copy()
        kept = torch.full((1, sum(keep)), -7, dtype=torch.int32, device="cuda")
        hkv.kv_pool_evict(pool.handle, src, tokens, dst, keep, 2, 10, w, kept)
        torch.cuda.synchronize()
        got, now = kept.cpu().numpy()[0], w.cpu().numpy()
        for i in range(n):
            sb, db, j = src[i * src_n: (i + 1) * src_n], dst[i * dst_n: (i + 1) * dst_n], np.arange(keep[0])
            t = evicted(was[:, 0], sb, tokens[0], keep[0], 2, 10)
            assert np.array_equal(got[i * keep[0]: (i + 1) * keep[0]], t), i
            assert np.array_equal(now[db[j // 16], 0, j % 16], was[sb[t // 16], 0, t % 16])
        pool.close()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3])
def test_a_prompt_is_stored_judged_and_shrunk(dtype):
    """Prefill of a prompt through the store, its 16 newest queries judge the keys, a third stays, and the next token attends to what stayed:
    every step against 64 bits on what the pool holds."""
    hq, heads, n, keep, T = 8, 2, 200, 70, 16
    pool = Pool(40, heads, dtype, seed=9)
    pages = hkv.kv_pool_alloc(pool.handle, 13)
    plan = hkv.hkv_prefill_plan_create(pool.handle, [0, n], pages[None], [n], hq)
    x = Rows(n, hq, heads, dtype, 11, rotary=128)
    before = pool.snapshot()
    hkv.hkv_prefill_plan_store(plan, x.arg)
    torch.cuda.synchronize()
    x.check(pool, before, np.arange(n), np.arange(n), units_of(pages, 0, np.arange(n)))
    # the window's queries: a decode plan over the prompt, its newest tokens queried together
    window = hkv.hkv_decode_plan_create_multi(pool.handle, [(-1, 0, 13, n)], pages, [0], T, hq)
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(window), dtype=torch.uint8, device="cuda")
    q = x.q_out[n - T:]
    out, lse = torch.empty_like(q), torch.empty(T, hq, device="cuda")
    hkv.attn_decode_plan_run(window, q, SCALE, out, lse, ws, ws.numel())
    w = torch.full((pool.blocks, heads, 16), float("nan"), device="cuda")
    hkv.hkv_decode_plan_track_weights(window)
    hkv.attn_decode_plan_weights(window, q, SCALE, lse, 0.0, 0, w)
    fresh = hkv.kv_pool_alloc(pool.handle, 5)
    kept = torch.empty(heads, keep, dtype=torch.int32, device="cuda")
    hkv.kv_pool_evict(pool.handle, pages, [n], fresh, [keep], 4, 8, w, kept)
    hkv.kv_pool_release(pool.handle, pages)
    torch.cuda.synchronize()
    kv, vv = pool.values()
    nodes = weight_nodes([-1], [n], [np.asarray(pages, dtype=np.int64)], [0], T)
    want = key_weights(kv, nodes, q.float().cpu().double().numpy(), lse.cpu().double().numpy(), SCALE, heads, np.zeros(w.shape), 0.0, 0, T)
    got, t = w.cpu().double().numpy(), np.arange(n)
    assert (np.abs(got[pages[t // 16], :, t % 16] - want[pages[t // 16], :, t % 16]) <= WEIGHT_TOL * want[pages[t // 16], :, t % 16]).all()
    for h in range(heads):
        assert np.array_equal(kept.cpu().numpy()[h], evicted(w.cpu().numpy()[:, h], np.asarray(pages), n, keep, 4, 8))
    # the next token: one more slot, its position the prompt's length
    grown = hkv.hkv_decode_plan_create_growing(pool.handle, [(-1, 0, 5, keep)], fresh, [0], hq, 8)
    y = Rows(1, hq, heads, dtype, 12, rotary=128)
    pos = torch.full((1, 1), n, dtype=torch.int32, device="cuda")
    y.positions, y.arg = pos, hkv.qkv_rows(y.q, y.k, y.v, y.q_out, q_norm=y.qw, k_norm=y.kw, eps=y.eps, rotary_dim=128, inv_freq=y.inv_freq, positions=pos)
    before = pool.snapshot()
    hkv.hkv_decode_plan_append_qkv(grown, None, y.arg)
    out, lse = torch.empty_like(y.q_out), torch.empty(1, hq, device="cuda")
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(grown) + 256, dtype=torch.uint8, device="cuda")
    hkv.attn_decode_plan_run(grown, y.q_out, SCALE, out, lse, ws, ws.numel())
    torch.cuda.synchronize()
    y.check(pool, before, np.arange(1), None, [(int(fresh[keep // 16]), keep % 16, np.arange(1))])
    kv, vv = pool.values()
    t, q64 = np.arange(keep + 1), y.q_out.float().cpu().double().numpy()
    for h in range(hq):
        s = kv[fresh[t // 16], h // 4, t % 16] @ q64[0, h] * SCALE
        p = np.exp(s - s.max())
        o = p @ vv[fresh[t // 16], h // 4, t % 16] / p.sum()
        assert abs(lse[0, h].item() - (s.max() + np.log(p.sum()))) <= 2e-3
        assert np.abs(out[0, h].float().cpu().double().numpy() - o).max() <= 2e-2     # the library's bound for a decode step
    for p in (window, grown):
        hkv.hkv_decode_plan_destroy(p)
    hkv.hkv_prefill_plan_destroy(plan)
    pool.close()


@pytest.mark.parametrize("dtype", [hkv.BF16, hkv.FP8_E4M3, hkv.FP32])
def test_the_attentions_own_lse_and_then_eviction(dtype):
    """Every row of a step gives away 1 in all, whatever the pool's type; what is kept weighs at least what is dropped."""
    hq, heads, T = 8, 2, 2
    nodes, pages, blocks, _ = forest([-1, 0, 0, 0], [160, 70, 33, 2], 16, 4)
    pool = Pool(len(pages) + 8, heads, dtype, seed=9)
    plan = hkv.hkv_decode_plan_create_ex(pool.handle, nodes, pages, [1, 2, 3], hq, tokens_per_req=T)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    q = (2 * torch.randn(3 * T, hq, 128, device="cuda", generator=g)).to(torch.float32 if dtype == hkv.FP32 else torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(3 * T, hq, device="cuda")
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
    w = torch.full((pool.blocks, heads, 16), float("nan"), device="cuda")
    hkv.attn_decode_plan_run(plan, q, SCALE, out, lse, ws, ws.numel())
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.attn_decode_plan_weights(plan, q, SCALE, lse, 0.0, T, w)
    got = w.cpu().double().numpy()
    live = ~np.isnan(got)
    assert live.sum() == (160 + 70 + 33 + 2) * heads
    assert abs(got[live].sum() - 3 * T * hq) <= 1e-3 * 3 * T * hq    # (lse as the attention rounds it)
    kept = torch.empty(heads, 40, dtype=torch.int32, device="cuda")
    free = np.setdiff1d(np.arange(len(pages) + 8), pages)[:3]
    hkv.kv_pool_evict(pool.handle, pages[:10], [160], free, [40], 2, 5, w, kept)
    k = kept.cpu().numpy()
    for h in range(heads):
        assert np.array_equal(k[h], evicted(got[:, h].astype(np.float32), blocks[0], 160, 40, 2, 5))
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()


def test_an_8_bit_pool_holds_what_is_no_number_as_its_writer_does():
    pools = [Pool(3, 2, hkv.FP8_E4M3, seed=5) for _ in range(2)]
    x = Rows(40, 2, 2, hkv.FP8_E4M3, 6, norm=False, rotary=0, fused=False)
    bad = (float("nan"), float("inf"), -float("inf"))
    for i, b in enumerate(bad):
        x.k[16 * i + 3, 0, 7 * i], x.v[16 * i + 4, 1, 9 * i] = b, b
    plan = hkv.hkv_prefill_plan_create(pools[0].handle, [0, 40], [[2, 0, 1]], [40], 2)
    hkv.hkv_prefill_plan_store(plan, x.arg)
    hkv.kv_pool_write(pools[1].handle, [2, 0, 1], 0, 40, x.k, x.v)
    torch.cuda.synchronize()
    for a, b in zip(*((p.k.view(torch.uint8), p.v.view(torch.uint8), p.k_scale.view(torch.int32), p.v_scale.view(torch.int32)) for p in pools)):
        assert torch.equal(a, b)
    hkv.hkv_prefill_plan_destroy(plan)
    for p in pools:
        p.close()


def test_captured_and_on_other_streams():
    """Stores and weights in a captured graph, replayed between eager runs of other plans, and eviction on a stream of its own."""
    hq, heads = 8, 2
    pool = Pool(64, heads, hkv.FP8_E4M3, seed=3)
    nodes, pages, blocks, _ = forest([-1, 0, 0], [100, 40, 33], 16, 2, spare=20)
    plan = hkv.hkv_decode_plan_create(pool.handle, nodes, pages, [1, 2], hq)
    hkv.hkv_decode_plan_track_weights(plan)
    x = Rows(2, hq, heads, hkv.FP8_E4M3, 1)
    ws = torch.empty(hkv.hkv_decode_plan_workspace_bytes(plan) + 256, dtype=torch.uint8, device="cuda")
    out, lse = torch.zeros_like(x.q_out), torch.zeros(2, hq, device="cuda")
    w = torch.zeros(pool.blocks, heads, 16, device="cuda")

    def step(stream):
        hkv.hkv_decode_plan_store(plan, x.arg, stream)
        hkv.attn_decode_plan_run(plan, x.q_out, SCALE, out, lse, ws, ws.numel(), stream)
        hkv.attn_decode_plan_weights(plan, x.q_out, SCALE, lse, 0.0, 1, w, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    mine = torch.from_numpy(np.concatenate(blocks)).cuda()   # (the evictions below write to others)
    held = lambda: (pool.k.view(torch.uint8).view(64, -1)[mine], pool.k_scale.view(64, -1)[mine])  # noqa: E731
    eager = [t.clone() for t in (x.q_out, out, lse, w, *held())]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step(torch.cuda.current_stream())
    other = torch.cuda.Stream()
    for i in range(3):
        for t in (x.q_out, out):
            t.fill_(float("nan"))
        lse.fill_(float("nan"))
        w.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        live = ~torch.isnan(w)
        for got, want in zip((x.q_out, out, lse, w[live], *held()), (eager[0], eager[1], eager[2], eager[3][live], *eager[4:])):
            assert torch.equal(got, want), i
        assert int(live.sum()) == (100 + 40 + 33) * heads
        kept = torch.empty(heads, 20, dtype=torch.int32, device="cuda")
        v = torch.rand(pool.blocks, heads, 16, device="cuda")
        other.wait_stream(torch.cuda.current_stream())
        free = np.setdiff1d(np.arange(64), pages)[:2]
        hkv.kv_pool_evict(pool.handle, pages[:7], [100], free, [20], 0, 0, v, kept, other)
        other.synchronize()
        vn = v.cpu().numpy()
        for h in range(heads):
            assert np.array_equal(kept.cpu().numpy()[h], evicted(vn[:, h], blocks[0], 100, 20, 0, 0))
    hkv.hkv_decode_plan_destroy(plan)
    pool.close()

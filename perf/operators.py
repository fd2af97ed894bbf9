"""What goes into a KV pool besides attention's reading of it, and what comes out: the calls around a step's attention whose speed counts.

A case is one of three operators over a paged pool (16-token blocks; K block [4 or 2 chunks of 64 bytes][16 tokens][chunk], V block
[128 dims][16 tokens], per KV head) with a head shape and a pool type:
  store    rows of a step's fused q / k / v projection: per-head RMS norm and rotation by position of q and k, queries out, K and V into
           the pool.  "new" tokens of each of `n` requests behind `prefix` shared ones (a prefill), or the newest `draft` tokens of
           requests that have `own` tokens behind them (a generation or verification step)
  weights  what every cached key got from the queries of a step, summed over rows and the query heads of its KV head, added to a
           running sum per key: `roots` prompts of `prefix` tokens, `fan` requests with up to `own` tokens under each
  evict    the `keep` heaviest tokens per KV head of `n` sequences of up to `tokens` tokens, moved in order to other pages
Token counts of the last level are drawn between `ragged` times the figure and the figure.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / np.sqrt(np.float32(D))))


def _store(name, dtype, heads, n, new, *, prefix=0, ragged=1.0, norm=True, rotary=128, interleaved=False, axes=1, page=16):
    c = {"op": "store", "dtype": dtype, "q_heads": heads[0], "kv_heads": heads[1], "n": n, "new": new, "prefix": prefix, "ragged": float(ragged),
         "norm": norm, "rotary": rotary, "interleaved": interleaved, "axes": axes, "page": page, "draft": 0, "own": 0}
    return {"name": name, **c} if name else c


def _step(name, dtype, heads, n, own_tokens, *, draft=1, **kw):
    return {**_store(name, dtype, heads, n, 0, **kw), "draft": draft, "own": own_tokens}


def _weights(name, dtype, heads, roots, fan, prefix, own_tokens, *, ragged=1.0, draft=1, decay=1.0, page=16):
    c = {"op": "weights", "dtype": dtype, "q_heads": heads[0], "kv_heads": heads[1], "roots": roots, "fan": fan, "prefix": prefix, "own": own_tokens,
         "ragged": float(ragged), "draft": draft, "decay": float(decay), "page": page}
    return {"name": name, **c} if name else c


def _evict(name, dtype, kv_heads, n, tokens, keep, *, first=4, recent=32, ragged=1.0, page=16):
    c = {"op": "evict", "dtype": dtype, "kv_heads": kv_heads, "n": n, "tokens": tokens, "keep": keep, "first": first, "recent": recent,
         "ragged": float(ragged), "page": page}
    return {"name": name, **c} if name else c


def listed():
    return [
        # the smallest generation step: four calls of one small workflow (a launch and its latency)
        _step("store_tiny_bf16", "bf16", (8, 2), 4, 17, prefix=256, norm=False),
        # the ordinary generation step of a chat-like batch: 64 calls under one system prompt (Llama-8B-shaped layer: rotation only)
        _step("store_chat_bf16", "bf16", (32, 8), 64, 512, prefix=2048, ragged=0.5, norm=False),
        # the large batch on a 70B-shaped layer, fp8 pool: each token continues a block, whose running scale may grow
        _step("store_forest_fp8", "fp8", (64, 8), 512, 512, prefix=8192, ragged=0.5, norm=False),
        # one call at a time behind a cached prefix, as a worker that follows a schedule runs them
        _store("store_one_call_bf16", "bf16", (32, 8), 1, 700, prefix=4096, norm=False),
        # a batch of prompts that hit a long cached prefix (a layer with normed heads): the largest store
        _store("store_prefix_hit_bf16", "bf16", (32, 8), 32, 1024, prefix=8192, ragged=0.75),
        # a few prompts with video among them over an fp8 pool (Qwen3-14B heads): positions in time, height and width
        _store("store_video_fp8", "fp8", (40, 8), 6, 512, prefix=2048, ragged=0.5, axes=3, page=64),
        # a generation step that keeps score of the keys: 64 calls under one system prompt
        _weights("weights_chat_bf16", "bf16", (32, 8), 1, 64, 2048, 512, ragged=0.7),
        # the large batch: 512 calls under 16 long prompts on a 70B-shaped layer, 1.2 GB of fp8 keys
        _weights("weights_forest_fp8", "fp8", (64, 8), 16, 32, 8192, 2048),
        # the 32 newest queries of a long prompt look back once, before what they pass over is dropped
        _weights("weights_window_bf16", "bf16", (32, 8), 1, 4, 1024, 8000, ragged=0.6, draft=32, decay=0.0),
        # a small workflow's calls over short contexts
        _weights("weights_tiny_bf16", "bf16", (8, 2), 1, 4, 256, 49, ragged=0.5),
        # one long call shrinks to a quarter
        _evict("evict_one_call_bf16", "bf16", 8, 1, 8190, 2048),
        # a batch of calls shrinks over an fp8 pool: blocks of mixed origin are scaled anew
        _evict("evict_batch_fp8", "fp8", 8, 32, 4096, 1000, ragged=0.6),
    ]


HEADS = [(32, 8), (32, 8), (40, 8), (64, 8), (8, 2)]  # Llama-8B / Qwen3-8B, Qwen3-14B, Qwen3-32B or 70B, a small layer


def draw(rng: random.Random):
    """A case of the same ranges: sizes spread over their logarithm, odd ones among them."""

    def size(lo, hi, multiple=1):
        return max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple))) * multiple

    while True:
        op = rng.choice(["store", "store", "step", "weights", "weights", "evict"])
        heads = rng.choice(HEADS)
        page = rng.choice([16, 16, 16, 32, 64])
        ragged = rng.choice([1.0, 0.75, 0.5, 0.3])
        dtype = rng.choice(["bf16", "bf16", "fp8", "fp8", "fp32"])
        how = {"norm": rng.random() < 0.5, "rotary": rng.choice([128, 128, 128, 64, 32, 96]), "interleaved": rng.random() < 0.3, "axes": rng.choice([1, 1, 1, 3])}
        if op == "store":
            c = _store("", dtype, heads, size(1, 32), size(1, 1024), prefix=size(16, 8192, page), ragged=ragged, page=page, **how)
        elif op == "step":
            draft = rng.choice([1, 1, 1, 2, 5, 21])
            c = _step("", dtype, heads, size(1, 512), size(32, 512), prefix=size(16, 8192, page), draft=min(draft, 16) if dtype == "fp32" else draft,
                      ragged=max(ragged, 0.75), page=page, **how)
        elif op == "weights":
            draft = rng.choice([1, 1, 1, 4, 16, 32])
            c = _weights("", "bf16" if dtype == "fp32" else dtype, heads, rng.choice([1, 1, 2, 4, 16]), size(1, 64), size(64, 8192), size(64, 2048), ragged=max(ragged, 0.5),
                         draft=draft, decay=rng.choice([1.0, 0.9, 0.0]), page=page)
        else:
            tokens = size(64, 8192)
            keep = max(1, int(tokens * 0.5 * rng.uniform(0.05, 1.0)))
            c = _evict("", dtype, heads[1], size(1, 64), tokens, keep, first=min(rng.choice([0, 1, 4]), keep // 4), recent=min(rng.choice([0, 16, 33]), keep // 4),
                       ragged=max(ragged, 0.5), page=page)
        w = work(c)
        most = {"store": (8.2e8, math.inf), "weights": (1.25e9, 7e10), "evict": (5.2e8, math.inf)}[c["op"]]
        if w["bytes"] <= most[0] and w["flops"] <= most[1]:
            return c


# ------------------------------------------------------------------------------------------------- shapes
TORCH = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "fp32": torch.float32}
ELEM = {"bf16": 2, "fp8": 1, "fp32": 4}


def _ragged(case, count, most, least=1):
    """Token counts of the last level, fixed by the case alone."""
    rng = np.random.default_rng([count, most, int(1000 * case["ragged"])])
    return rng.integers(max(least, int(case["ragged"] * most)), max(least, most) + 1, size=count).astype(np.int64)


def _lengths(case):
    if case["op"] == "store":
        return _ragged(case, case["n"], case["new"]) if not case["draft"] else _ragged(case, case["n"], case["own"], case["draft"])
    if case["op"] == "weights":
        return _ragged(case, case["roots"] * case["fan"], case["own"], case["draft"])
    return _ragged(case, case["n"], case["tokens"], case["keep"])


def work(case):
    """store: the projections' rows, the queries and what goes into the pages.  weights: every key of the forest, queries, their lse, the
    running sums in and out; 2 * 128 operations per visible pair.  evict: the sums of all tokens, K and V of the kept ones in and out."""
    hk, e = case["kv_heads"], ELEM[case["dtype"]]
    lens, per_scale = _lengths(case), 4 / 16 if case["dtype"] == "fp8" else 0
    if case["op"] == "store":
        rows = int(lens.sum()) if not case["draft"] else case["n"] * case["draft"]
        src = 4 if case["dtype"] == "fp32" else 2
        return {"bytes": rows * (2 * case["q_heads"] * D * src + 2 * hk * (D * (src + e) + per_scale) + (12 if case["axes"] > 1 else 0)), "flops": 0}
    if case["op"] == "weights":
        T, hq = case["draft"], case["q_heads"]
        tokens, rows = int(lens.sum()) + case["roots"] * case["prefix"], len(lens) * T
        pairs = case["prefix"] * rows + sum(T * (int(n) - T) + T * (T + 1) // 2 for n in lens)
        return {"bytes": tokens * hk * (D * e + per_scale + (8 if case["decay"] else 4)) + rows * hq * (2 * D + 4), "flops": 2 * D * hq * pairs}
    kept = case["n"] * case["keep"] * hk
    return {"bytes": int(lens.sum()) * hk * 4 + kept * (4 * D * e + 4 * per_scale + 8), "flops": 0}


def _layout(case, seed):
    """Block ids of everything the case keeps in the pool: (16-token blocks in all, page ids of the shared prompts [roots][pages], of the
    sequences (one array each), of their new places)."""
    page, lens = case["page"], _lengths(case)
    roots = case.get("roots", 1) if case["op"] != "evict" else 0
    n_root = -(-case["prefix"] // page) if roots else 0
    n_own = [-(-int(n) // page) for n in lens]
    n_dst = -(-case["keep"] // page) if case["op"] == "evict" else 0
    used = roots * n_root + sum(n_own) + n_dst * len(lens)
    total = used + used // 4 + 1
    order = np.random.default_rng([int(seed), 5]).permutation(total).astype(np.int32)
    ends = np.cumsum([roots * n_root, *n_own, *([n_dst] * (len(lens) if n_dst else 0))])
    parts = np.split(order[: ends[-1]], ends[:-1])
    return total, parts[0].reshape(roots, n_root), parts[1: 1 + len(lens)], parts[1 + len(lens):]


def _blocks(pages, page):
    """16-token blocks of a page list: block j of page p is p * (page / 16) + j."""
    s = page // 16
    return (np.asarray(pages, dtype=np.int64)[..., None] * s + np.arange(s)).reshape(*np.shape(pages)[:-1], -1)


# ------------------------------------------------------------------------------------------------- inputs
class _State:
    """What a program keeps between calls: page buffers, rows, indices of its tokens, and the library's pool and plan."""

    hkv = pool = plan = rows = None

    def __del__(self):
        try:
            if self.plan is not None:
                (self.hkv.hkv_prefill_plan_destroy if self.prefill else self.hkv.hkv_decode_plan_destroy)(self.plan)
            if self.pool is not None:
                self.hkv.kv_pool_destroy(self.pool)
        except Exception:
            pass


def _cuda(a, dtype=torch.int64):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


def _inputs(case, seed):
    """Everything an operator reads, on the GPU, from the seed alone, and where the tokens lie."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 29)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen)

    s = _State()
    s.case, hk, page = case, case["kv_heads"], case["page"]
    lens = s.lens = _lengths(case)
    total, root_pages, own_pages, dst_pages = s.pages = _layout(case, seed)
    nb = s.nb = total * (page // 16)
    s.k_scale = s.v_scale = None
    if case["dtype"] == "fp8":  # codes as a writer leaves them: block maxima near 448
        s.k, s.v = (torch.empty(nb * hk * 2048, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        for t in (s.k, s.v):
            for a in range(0, t.numel(), 1 << 27):
                t[a: a + (1 << 27)] = (normal(min(t.numel() - a, 1 << 27)) * 120).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s.k_scale, s.v_scale = (torch.empty(nb * hk, device="cuda").uniform_(0.006, 0.011, generator=gen) for _ in range(2))
    else:
        s.k, s.v = (normal(nb * hk * 2048, dtype=TORCH[case["dtype"]]) for _ in range(2))
    act = torch.float32 if case["dtype"] == "fp32" else torch.bfloat16
    if case["op"] == "store":
        hq, T = case["q_heads"], case["draft"]
        new = lens if not T else np.full(len(lens), T)
        rows = s.n_rows = int(new.sum())
        qkv = normal(rows, (hq + 2 * hk) * D, dtype=act)  # as one product of the projections leaves them
        s.q, s.k_new, s.v_new = (x.unflatten(1, (-1, D)) for x in qkv.split([hq * D, hk * D, hk * D], dim=1))
        s.q_out = torch.empty(rows, hq, D, dtype=act, device="cuda")
        s.q_norm, s.k_norm = ((1 + 0.2 * normal(D)).to(act) if case["norm"] else None for _ in range(2))
        R = case["rotary"]
        s.inv_freq = 1e6 ** (-torch.arange(0, R, 2, dtype=torch.float64, device="cuda") / R)
        # the new tokens' places: request by request, `first` tokens of the sequence's own page list before them
        first = np.zeros(len(lens), dtype=np.int64) if not T else lens - T
        at = np.concatenate([f + np.arange(n) for f, n in zip(first, new)])
        blocks = [_blocks(p, page) for p in own_pages]
        block = np.concatenate([b[(f + np.arange(n)) // 16] for b, f, n in zip(blocks, first, new)])
        starts = np.flatnonzero(np.concatenate([[True], block[1:] != block[:-1]]))  # a run of one block's tokens each
        unit = np.cumsum(np.concatenate([[False], block[1:] != block[:-1]]))
        low = at[starts] % 16
        s.block, s.slot, s.unit, s.unit_block, s.unit_low = _cuda(block), _cuda(at % 16), _cuda(unit), _cuda(block[starts]), _cuda(low)
        s.continued = _cuda(np.flatnonzero(low > 0))
        s.position = _cuda(case["prefix"] + at, torch.float64)[None, :]
        s.positions = s.axis = None
        if case["axes"] > 1:  # frames of 12 x 20 patches: each axis has its own share of the pairs
            p = case["prefix"] + at
            s.positions = _cuda(np.stack([p // 240, p // 20 % 12, p % 20]), torch.int32)
            s.position = s.positions.double()
            pairs = R // 2
            s.axis = np.repeat(np.arange(3), [pairs - 2 * (3 * pairs // 8), 3 * pairs // 8, 3 * pairs // 8]).astype(np.int32)
        s.axis_of = _cuda(s.axis if s.axis is not None else np.zeros(R // 2))
    elif case["op"] == "weights":
        T, hq, n = case["draft"], case["q_heads"], len(lens)
        s.q = normal(n * T, hq, D, dtype=act) * 2
        nb0, nb1 = -(-case["prefix"] // 16), -(-int(lens.max()) // 16)
        own_blocks = np.zeros((n, nb1), dtype=np.int64)
        for i, p in enumerate(own_pages):
            b = _blocks(p, page)[: -(-int(lens[i]) // 16)]
            own_blocks[i, : len(b)] = b
        s.root_blocks, s.own_blocks = _cuda(_blocks(root_pages, page)[:, :nb0]), _cuda(own_blocks)
        s.lens_gpu = _cuda(lens)
        s.weights = torch.empty(nb, hk, 16, device="cuda").uniform_(0, 0.02, generator=gen)  # some steps' worth
        lse = [torch.logsumexp(x, dim=2) for x in (_root_scores(s), _own_scores(s))]  # [roots][hk][rows], [n][hk][rows]
        lse = [_rows(s, lse[0], case["roots"], case["fan"] * T), _rows(s, lse[1], n, T)]
        s.lse = torch.logaddexp(*lse).contiguous()
    else:
        w = torch.exp(2 * normal(nb, hk, 16))
        s.weights = torch.where(torch.rand(w.shape, device="cuda", generator=gen) < 0.1, torch.zeros_like(w), w)  # a tenth was never looked at
        L, keep = int(lens.max()), case["keep"]
        src = np.zeros((len(lens), -(-L // 16)), dtype=np.int64)
        for i, p in enumerate(own_pages):
            b = _blocks(p, page)[: -(-int(lens[i]) // 16)]
            src[i, : len(b)] = b
        dst = np.stack([_blocks(p, page)[: -(-keep // 16)] for p in dst_pages])
        s.src_blocks, s.dst_blocks, s.lens_gpu = _cuda(src), _cuda(dst), _cuda(lens)
        s.src_pages, s.dst_pages = np.concatenate(own_pages), np.concatenate(dst_pages)
        s.kept = torch.empty(hk, len(lens) * keep, dtype=torch.int32, device="cuda")
    return s


def _forest(s):
    """The requests as the library takes them: shared prompts, then a node for each request."""
    case, page = s.case, s.case["page"]
    _, root_pages, own_pages, _ = s.pages
    roots, fan = case.get("roots", 1), len(s.lens) // case.get("roots", 1)
    nodes, begin = [], 0
    for p in root_pages:
        nodes.append((-1, begin, len(p), case["prefix"]))
        begin += len(p)
    for i, (p, n) in enumerate(zip(own_pages, s.lens)):
        nodes.append((i // fan, begin, len(p), int(n)))
        begin += len(p)
    return np.asarray(nodes, dtype=np.int32), np.concatenate([root_pages.ravel(), *own_pages]), np.arange(roots, roots + len(s.lens), dtype=np.int32)


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2603_16104_amd import binding as hkv
        s.hkv, hk, page = hkv, case["kv_heads"], case["page"]
        dtype = {"bf16": hkv.BF16, "fp8": hkv.FP8_E4M3, "fp32": hkv.FP32}[case["dtype"]]
        s.stream = torch.cuda.current_stream().cuda_stream
        s.pool = hkv.kv_pool_create(s.nb * 16 // page, hk, dtype, s.k, s.v, s.k_scale, s.v_scale, page_size=page)
        s.prefill = case["op"] == "store" and not case["draft"]
        if s.prefill:
            _, root_pages, own_pages, _ = s.pages
            cu = np.concatenate([[0], np.cumsum(s.lens)]).astype(np.int32)
            table = np.full((len(s.lens), root_pages.shape[1] + max(len(p) for p in own_pages)), -1, dtype=np.int32)
            table[:, : root_pages.shape[1]] = root_pages
            for i, p in enumerate(own_pages):
                table[i, root_pages.shape[1]: root_pages.shape[1] + len(p)] = p
            s.plan = hkv.hkv_prefill_plan_create(s.pool, cu, table, case["prefix"] + s.lens, case["q_heads"])
        elif case["op"] != "evict":
            T, (nodes, node_pages, leaves) = case["draft"], _forest(s)
            if T <= 16:
                s.plan = hkv.hkv_decode_plan_create_multi(s.pool, nodes, node_pages, leaves, T, case["q_heads"])
            else:  # more query tokens than a run may have: the same by masks
                masks = np.tile(np.asarray([(1 << (t + 1)) - 1 for t in range(T)], dtype=np.uint64), len(leaves))
                s.plan = hkv.hkv_decode_plan_create_tree(s.pool, nodes, node_pages, leaves, T, masks, case["q_heads"])
        if case["op"] == "store":
            s.rows = hkv.qkv_rows(s.q, s.k_new, s.v_new, s.q_out, q_norm=s.q_norm, k_norm=s.k_norm, eps=1e-6, rotary_dim=case["rotary"],
                                  inv_freq=s.inv_freq, interleaved=case["interleaved"], positions=s.positions, axis=s.axis)
        elif case["op"] == "weights":
            hkv.hkv_decode_plan_track_weights(s.plan)
    return s


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    case = s.case
    if own:
        if case["op"] == "store":
            (s.hkv.hkv_prefill_plan_store if s.prefill else s.hkv.hkv_decode_plan_store)(s.plan, s.rows, s.stream)
        elif case["op"] == "weights":
            s.hkv.attn_decode_plan_weights(s.plan, s.q, SCALE, s.lse, case["decay"], case["draft"], s.weights, s.stream)
        else:
            n = len(s.lens)
            s.hkv.kv_pool_evict(s.pool, s.src_pages, s.lens, s.dst_pages, np.full(n, case["keep"]), case["first"], case["recent"], s.weights, s.kept,
                                s.stream)
    elif case["op"] == "store":
        _plain_store(s)
    elif case["op"] == "weights":
        _plain_weights(s)
    else:
        _plain_evict(s)
    if case["op"] == "weights":
        return {"weights": s.weights}
    out = {"k": s.k, "v": s.v}
    if case["dtype"] == "fp8":
        out |= {"k_scale": s.k_scale, "v_scale": s.v_scale}
    return out | ({"q": s.q_out} if case["op"] == "store" else {"kept": s.kept, "weights": s.weights})


def _k_blocks(s):
    """The K buffer as [block][head][chunk][token][dim of the chunk]."""
    c = 64 // s.k.element_size()
    return s.k.view(s.nb, -1, D // c, 16, c)


def _v_blocks(s):
    return s.v.view(s.nb, -1, D, 16)


def _values(x, scale=None):
    """What codes or elements stand for, in 32 bits; `scale` has the shape of x's leading axes."""
    return x.float() if scale is None else x.float() * scale


def _normed(x, w):
    x = x.float()
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w.float()


def _rotated(x, cos, sin, interleaved):
    R = 2 * cos.shape[-1]
    rot, rest = x[..., :R], x[..., R:]
    a, b = (rot[..., 0::2], rot[..., 1::2]) if interleaved else (rot[..., : R // 2], rot[..., R // 2:])
    a, b = a * cos - b * sin, b * cos + a * sin
    return torch.cat([torch.stack([a, b], dim=-1).flatten(-2) if interleaved else torch.cat([a, b], dim=-1), rest], dim=-1)


def _codes(x, scale):
    return (x / scale).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _put(s, buf, scales, x, view, slots_last):
    """Rows x [n][head][128] into one of the page buffers, given as blocks; fp8: with the blocks' scales."""
    if scales is not None:
        scales = scales.view(s.nb, -1)
        amax = torch.zeros(len(s.unit_block), x.shape[1], device="cuda")
        amax.scatter_reduce_(0, s.unit[:, None].expand(-1, x.shape[1]), x.abs().amax(-1), "amax")
        full = torch.full_like(amax, 448.0)  # (a tensor divisor: a division by a number multiplies with its reciprocal)
        cand, old = amax / full, scales[s.unit_block]
        new = torch.where(s.unit_low[:, None] > 0, torch.maximum(old, cand), torch.where(amax > 0, cand, torch.ones_like(cand)))
        scales[s.unit_block] = new
        if len(s.continued):  # the earlier codes of a block whose scale grew are rounded again
            c, low = s.continued, s.unit_low[s.continued]
            b = view[s.unit_block[c]]
            r = _codes(b.float() * old[c][:, :, None, None, None], new[c][:, :, None, None, None]) if not slots_last else \
                _codes(b.float() * old[c][:, :, None, None], new[c][:, :, None, None])
            t = torch.arange(16, device="cuda")
            earlier = t[None] < low[:, None]
            earlier = earlier[:, None, None, :] & (new > old)[c][:, :, None, None] if slots_last else earlier[:, None, None, :, None] & (new > old)[c][:, :, None, None, None]
            view[s.unit_block[c]] = torch.where(earlier, r.float(), b.float()).to(torch.float8_e4m3fn)
        x = _codes(x, new[s.unit][:, :, None])
    x = x.to(buf.dtype)
    if slots_last:
        view[s.block, :, :, s.slot] = x
    else:
        view[s.block, :, :, s.slot] = x.unflatten(2, (view.shape[2], -1))


def _plain_store(s):
    angle = s.position[s.axis_of].T * s.inv_freq[None, :]  # in 64 bits: places are far from 0
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]
    turned = s.case["interleaved"]
    s.q_out.copy_(_rotated(_normed(s.q, s.q_norm), cos, sin, turned))
    _put(s, s.k, s.k_scale, _rotated(_normed(s.k_new, s.k_norm), cos, sin, turned), _k_blocks(s), False)
    _put(s, s.v, s.v_scale, s.v_new.float(), _v_blocks(s), True)


def _scores(s, blocks, q):
    """scale * K q of the listed blocks [nodes][blocks] and rows q [nodes][head][rows][128]: [nodes][head][tokens][rows]."""
    k = _k_blocks(s)[blocks]
    k = _values(k, None if s.k_scale is None else s.k_scale.view(s.nb, -1)[blocks][..., None, None, None])
    k = k.permute(0, 2, 1, 4, 3, 5).reshape(blocks.shape[0], k.shape[2], -1, D)
    return torch.matmul(k, q.transpose(2, 3).contiguous()) * SCALE


def _grouped(s, x, nodes):
    """[rows][q head][...] as [nodes][KV head][rows of the node x heads of the group][...]."""
    hk = s.case["kv_heads"]
    x = x.unflatten(1, (hk, -1)).unflatten(0, (nodes, -1))
    return x.transpose(1, 2).flatten(2, 3)


def _rows(s, x, nodes, rows):
    """The way back for one value per row: [nodes][KV head][rows x group] as [rows][q head]."""
    return x.unflatten(2, (rows, -1)).transpose(1, 2).flatten(2, 3).flatten(0, 1)


def _root_scores(s):
    c = s.case
    x = _scores(s, s.root_blocks, _grouped(s, s.q.float(), c["roots"]))
    return x.masked_fill_((torch.arange(x.shape[2], device="cuda") >= c["prefix"])[:, None], -math.inf)


def _own_scores(s):
    T = s.case["draft"]
    x = _scores(s, s.own_blocks, _grouped(s, s.q.float(), len(s.lens)))
    t, row = torch.arange(x.shape[2], device="cuda"), torch.arange(x.shape[3], device="cuda") // (x.shape[3] // T)
    last = (s.lens_gpu - T)[:, None] + row  # [nodes][rows]: the newest key that a row sees
    return x.masked_fill_((t[:, None] > last[:, None, :])[:, None], -math.inf)


def _add(s, blocks, got, alive, fresh):
    """The running sums of the listed blocks, where `alive` says that there is a token; `fresh` ones start from 0."""
    old = s.weights[blocks]                                       # [nodes][blocks][head][16]
    got = got.unflatten(2, (-1, 16)).transpose(1, 2)
    alive, fresh = (m.unflatten(1, (-1, 16))[:, :, None, :] for m in (alive, fresh))
    decay = s.case["decay"]
    new = got if decay == 0 else got + torch.where(fresh, torch.zeros_like(old), decay * old)
    keep = alive.expand_as(old)
    at = blocks[:, :, None, None].expand_as(old)[keep]
    head, slot = (torch.arange(n, device="cuda").view(v).expand_as(old)[keep] for n, v in ((old.shape[2], (1, 1, -1, 1)), (16, (1, 1, 1, -1))))
    s.weights[at, head, slot] = new[keep]


def _plain_weights(s):
    c, T = s.case, s.case["draft"]
    roots, n = c["roots"], len(s.lens)
    x = _root_scores(s)
    got = torch.exp(x - _grouped(s, s.lse, roots)[:, :, None, :]).sum(-1)
    t = torch.arange(x.shape[2], device="cuda")[None]
    alive = (t < c["prefix"]).expand(roots, -1)
    _add(s, s.root_blocks, got, alive, torch.zeros_like(alive))
    x = _own_scores(s)
    got = torch.exp(x - _grouped(s, s.lse, n)[:, :, None, :]).sum(-1)
    t = torch.arange(x.shape[2], device="cuda")[None]
    _add(s, s.own_blocks, got, t < s.lens_gpu[:, None], t >= s.lens_gpu[:, None] - T)


def _plain_evict(s):
    c, hk, n, keep = s.case, s.case["kv_heads"], len(s.lens), s.case["keep"]
    w = s.weights[s.src_blocks].permute(0, 2, 1, 3).flatten(2)    # [n][head][tokens]
    t, end = torch.arange(w.shape[2], device="cuda")[None], s.lens_gpu[:, None]
    must, dead = ((t < c["first"]) | (t >= end - c["recent"])) & (t < end), t >= end
    key = torch.where(must[:, None], torch.full_like(w, math.inf), torch.where(dead[:, None], torch.full_like(w, -math.inf), w))
    order = torch.sort(key, dim=2, descending=True, stable=True).indices[:, :, :keep]
    kept = torch.sort(order, dim=2).values                        # [n][head][keep]
    s.kept.copy_(kept.transpose(0, 1).flatten(1))
    j = torch.arange(keep, device="cuda")
    head = torch.arange(hk, device="cuda")[None, :, None]
    src, slot = s.src_blocks[torch.arange(n, device="cuda")[:, None, None], kept // 16], kept % 16
    dst = s.dst_blocks[:, None, j // 16].expand_as(src)
    s.weights[dst, head, j % 16] = s.weights[src, head, slot]
    kv, vv = _k_blocks(s), _v_blocks(s)
    k, v = kv[src, head, :, slot], vv[src, head, :, slot]         # [n][head][keep][chunk][dim], [n][head][keep][128]
    if s.k_scale is not None:
        k, v = _anew(s, s.k_scale, k.flatten(3), src, head).view(k.shape), _anew(s, s.v_scale, v, src, head)
    kv[dst, head, :, j % 16] = k
    vv[dst, head, :, j % 16] = v


def _anew(s, scales, codes, src, head):
    """Codes of mixed origin [n][head][keep][128] under one scale for each new block."""
    n, keep = len(s.lens), s.case["keep"]
    scales = scales.view(s.nb, -1)
    x = codes.float() * scales[src, head][..., None]
    pad = -keep % 16
    amax = torch.nn.functional.pad(x.abs().amax(-1), (0, pad)).unflatten(2, (-1, 16)).amax(-1)
    new = torch.where(amax > 0, amax / torch.full_like(amax, 448.0), torch.ones_like(amax))
    scales[s.dst_blocks[:, None, :].expand(n, x.shape[1], -1), head] = new
    return _codes(x, new.repeat_interleave(16, dim=2)[:, :, :keep, None])


# ------------------------------------------------------------------------------------------------- the same in 64 bits
def _flat(block, head, slot, dim, hk, elem, is_k):
    """Element of the page buffers that holds (slot, dim) of a block and head."""
    c = 64 // elem
    return (block * hk + head) * 2048 + ((dim // c) * 16 * c + slot * c + dim % c if is_k else dim * 16 + slot)


def exact(case, seed):
    s = _inputs(case, seed)
    return {"store": _exact_store, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](s, case)


def _exact_scale(amax):
    return torch.where(amax > 0, amax / 448.0, torch.ones_like(amax))


def _exact_store(s, case):
    hk, e = case["kv_heads"], ELEM[case["dtype"]]
    ids = torch.arange(D, device="cuda")
    pairs = case["rotary"] // 2
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s.position[s.axis_of].T * s.inv_freq)[:, None, :]

    def z(x, w):
        x = x.double()
        if w is not None:
            x = x / ((x * x).sum(-1, keepdim=True) / D + 1e-6).sqrt() * w.double()
        a, b = (2 * ids[:pairs], 2 * ids[:pairs] + 1) if case["interleaved"] else (ids[:pairs], ids[:pairs] + pairs)
        y = torch.complex(x[..., a], x[..., b]) * turn
        x = x.clone()
        x[..., a], x[..., b] = y.real, y.imag
        return x

    out = {"q": z(s.q, s.q_norm)}
    for name, x, buf, scales in (("k", z(s.k_new, s.k_norm), s.k, s.k_scale), ("v", s.v_new.double(), s.v, s.v_scale)):
        got = buf.double()
        head = torch.arange(hk, device="cuda")
        if scales is not None:
            scales = scales.double().view(-1, hk)
            amax = torch.zeros((s.nb, hk), dtype=torch.float64, device="cuda")
            amax.index_reduce_(0, s.block, x.abs().amax(-1), "amax")
            amax, old = amax[s.unit_block], scales[s.unit_block].clone()
            new = torch.where(s.unit_low[:, None] > 0, torch.maximum(old, amax / 448.0), _exact_scale(amax))
            scales[s.unit_block] = new
            t = torch.arange(16, device="cuda")
            at = _flat(s.unit_block[:, None, None, None], head[:, None, None], t[:, None], ids, hk, e, name == "k")
            earlier = (t[None] < s.unit_low[:, None])[:, None, :, None].expand(at.shape)
            got[at[earlier]] = (got[at] * (old / new)[:, :, None, None])[earlier]
            x = x / scales[s.block][..., None]
            out[name + "_scale"] = scales.flatten()
        at = _flat(s.block[:, None, None], head[:, None], s.slot[:, None, None], ids, hk, e, name == "k")
        got[at] = x
        out[name] = got
    return out


def _exact_weights(s, case):
    hk, e, T, roots = case["kv_heads"], ELEM[case["dtype"]], case["draft"], case["roots"]
    G, fan = case["q_heads"] // hk, case["fan"]
    out = s.weights.double()
    ids, head = torch.arange(D, device="cuda"), torch.arange(hk, device="cuda")

    def node(blocks, n, rows, limit, n_new):
        """Adds to the first n tokens of the blocks what the rows give; row i sees the tokens before limit[i], the last n_new start from 0."""
        t = torch.arange(n, device="cuda")
        b = blocks[t // 16]
        at = _flat(b[:, None, None], head[:, None], (t % 16)[:, None, None], ids, hk, e, True)
        keys = s.k[at].double()
        if s.k_scale is not None:
            keys = keys * s.k_scale.double().view(-1, hk)[b][..., None]
        q = s.q[rows].double().view(len(rows), hk, G, D)
        x = torch.einsum("thd,rhgd->hrgt", keys, q) * SCALE - s.lse[rows].double().view(-1, hk, G).transpose(0, 1)[..., None]
        got = (torch.exp(x) * (t[None] < limit[:, None])[None, :, None, :]).sum((1, 2)).T  # [t][head]
        old = out[b, :, t % 16] if case["decay"] else torch.zeros_like(got)
        out[b, :, t % 16] = got + case["decay"] * old * (t < n - n_new)[:, None]

    for r in range(roots):
        rows = torch.arange(r * fan * T, (r + 1) * fan * T, device="cuda")
        node(s.root_blocks[r], case["prefix"], rows, torch.full((len(rows),), case["prefix"], device="cuda"), 0)
    for i, n in enumerate(s.lens.tolist()):
        node(s.own_blocks[i], n, torch.arange(i * T, (i + 1) * T, device="cuda"), n - T + 1 + torch.arange(T, device="cuda"), T)
    return {"weights": out}


def _exact_evict(s, case):
    hk, e, keep, n = case["kv_heads"], ELEM[case["dtype"]], case["keep"], len(s.lens)
    ids, head = torch.arange(D, device="cuda"), torch.arange(hk, device="cuda")
    w = s.weights.double().cpu().numpy()
    kept = np.empty((n, hk, keep), dtype=np.int64)
    for i, m in enumerate(s.lens.tolist()):
        rows = w[s.src_blocks[i].cpu().numpy()].transpose(1, 0, 2).reshape(hk, -1)[:, :m].copy()
        rows[:, : case["first"]] = np.inf
        rows[:, m - case["recent"]:] = np.inf
        kept[i] = np.sort(np.argsort(-rows, axis=1, kind="stable")[:, :keep], axis=1)
    at = _cuda(kept)
    j = torch.arange(keep, device="cuda")
    src = torch.gather(s.src_blocks[:, None, :].expand(-1, hk, -1), 2, at // 16)
    dst = s.dst_blocks[:, j // 16][:, None, :].expand_as(src)
    out = {"kept": _cuda(kept.transpose(1, 0, 2).reshape(hk, -1), torch.int32)}
    weights = s.weights.double()
    weights[dst, head[None, :, None], j % 16] = weights[src, head[None, :, None], at % 16]
    out["weights"] = weights
    for name, buf, scales in (("k", s.k, s.k_scale), ("v", s.v, s.v_scale)):
        got, h = buf.double(), head[None, :, None, None]
        x = got[_flat(src[..., None], h, (at % 16)[..., None], ids, hk, e, name == "k")]
        if scales is not None:
            scales = scales.double().view(-1, hk).clone()
            x = x * scales[src, head[None, :, None]][..., None]
            amax = torch.zeros(s.nb * hk, dtype=torch.float64, device="cuda")
            amax.index_reduce_(0, (dst * hk + head[None, :, None]).flatten(), x.abs().amax(-1).flatten(), "amax")
            there = dst * hk + head[None, :, None]
            scales.view(-1)[there.flatten()] = _exact_scale(amax)[there.flatten()]
            x = x / scales.view(-1)[there][..., None]
            out[name + "_scale"] = scales.flatten()
        got[_flat(dst[..., None], h, (j % 16)[:, None], ids, hk, e, name == "k")] = x
        out[name] = got
    return out

"""A KV pool in 4 bits, with the attention that reads it, and the calls that move pages: into it and back, to new sequences, together.

A 4-bit pool holds e2m1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) and an 8-bit power of two for each 32 dims of a token.  Of
a 16-token block and KV head, K is [t % 4][t / 4][64 bytes], V [t / 4][d / 8][t % 4][4 bytes], the even dim in the low half of a byte;
scales are [d / 32][t], byte b standing for 2^(b - 127).  A case is one of
  write    `n` prompts' K and V of up to `new` tokens go in, or (`new` 0) one token each behind up to `own` ones; what the blocks then
           hold is read back as bf16
  decode   attention of the newest `draft` tokens of each of `fan` requests under `roots` prompts of `prefix` tokens, up to `own` tokens each
  prefill  attention of `n` requests' up to `new` tokens behind `prefix` cached ones
  cold     the pages of `n` sequences of up to `tokens` tokens go from a pool of `dtype` to 4 bits, and come back to other pages
  fork     `n` sequences of up to `tokens` tokens, their last pages not full, become `fan` * n ones that share the full pages
  compact  the pages in use, a share `live` of a pool, move to its front
Token counts are drawn between `ragged` times the figure and the figure.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / np.sqrt(np.float32(D))))


def _case(name, op, **kw):
    return {"name": name, "op": op, **kw} if name else {"op": op, **kw}


def _write(name, kv_heads, n, new, own_tokens=0, *, ragged=1.0, page=16):
    return _case(name, "write", kv_heads=kv_heads, n=n, new=new, own=own_tokens, ragged=float(ragged), page=page)


def _decode(name, heads, roots, fan, prefix, own_tokens, *, ragged=1.0, draft=1, page=16):
    return _case(name, "decode", q_heads=heads[0], kv_heads=heads[1], roots=roots, fan=fan, prefix=prefix, own=own_tokens, ragged=float(ragged),
                 draft=draft, page=page)


def _prefill(name, heads, n, new, prefix, *, ragged=1.0, page=16):
    return _case(name, "prefill", q_heads=heads[0], kv_heads=heads[1], n=n, new=new, prefix=prefix, ragged=float(ragged), page=page)


def _cold(name, dtype, kv_heads, n, tokens, *, ragged=1.0, page=16):
    return _case(name, "cold", dtype=dtype, kv_heads=kv_heads, n=n, tokens=tokens, ragged=float(ragged), page=page)


def _fork(name, dtype, kv_heads, n, tokens, fan, *, ragged=1.0, page=16):
    return _case(name, "fork", dtype=dtype, kv_heads=kv_heads, n=n, tokens=tokens, fan=fan, ragged=float(ragged), page=page)


def _compact(name, dtype, kv_heads, pages, live, *, page=16):
    return _case(name, "compact", dtype=dtype, kv_heads=kv_heads, pages=pages, live=float(live), page=page)


def listed():
    return [
        # a generation step's new tokens: 64 calls, one token each (a launch and its latency)
        _write("write_step", 8, 64, 0, 512, ragged=0.5),
        # one long prompt is stored
        _write("write_prompt", 8, 1, 8190),
        # the smallest step: four calls of one small workflow
        _decode("decode_tiny", (8, 2), 1, 4, 256, 49, ragged=0.5),
        # the ordinary generation step: 64 calls under one system prompt (Llama-8B-shaped layer)
        _decode("decode_chat", (32, 8), 1, 64, 2048, 512, ragged=0.7),
        # the large batch: 512 calls under 16 long prompts on a 70B-shaped layer, 1.1 GB of 4-bit keys and values
        _decode("decode_forest", (64, 8), 16, 32, 8192, 2048, ragged=0.5),
        # drafted tokens are verified, 8 at a time, behind a cached context (Qwen3-14B heads)
        _decode("decode_drafts", (40, 8), 4, 4, 4096, 1000, ragged=0.6, draft=8),
        # one call at a time behind a cached prefix, as a worker that follows a schedule runs them
        _prefill("prefill_one_call", (32, 8), 1, 700, 4096),
        # a batch of prompts that hit a long cached prefix
        _prefill("prefill_prefix_hit", (32, 8), 8, 1024, 8192, ragged=0.75),
        # prompts that no call waits for go to 4 bits, and come back when one hits them
        _cold("cold_prompts", "bf16", 8, 8, 4096, ragged=0.7),
        # the branches of 16 calls go on from where those are, four each: only their last pages are copied
        _fork("fork_branches", "bf16", 8, 16, 500, 4, ragged=0.6),
        # a long call's fork in a pool of large pages
        _fork("fork_one_call", "fp8", 8, 1, 8000, 2, page=64),
        # a pool half in use after calls of all lengths have come and gone
        _compact("compact_half", "bf16", 8, 8192, 0.5),
    ]


HEADS = [(32, 8), (32, 8), (40, 8), (64, 8), (8, 2)]  # Llama-8B / Qwen3-8B, Qwen3-14B, Qwen3-32B or 70B, a small layer


def draw(rng: random.Random):
    """A case of the same ranges: sizes spread over their logarithm, odd ones among them."""

    def size(lo, hi, multiple=1):
        return max(1, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple))) * multiple

    while True:
        op = rng.choice(["write", "decode", "decode", "decode", "prefill", "prefill", "cold", "fork", "compact"])
        heads = rng.choice(HEADS)
        hk = heads[1]
        page = rng.choice([16, 16, 16, 32, 64])
        ragged = rng.choice([1.0, 0.75, 0.5])
        dtype = rng.choice(["bf16", "bf16", "fp8", "fp32"])
        if op == "write":
            c = _write("", hk, size(1, 512), 0, size(16, 512), ragged=ragged, page=page) if rng.random() < 0.5 else _write("", hk, size(1, 8), size(1, 8190), ragged=ragged, page=page)
        elif op == "decode":
            draft = rng.choice([1, 1, 1, 2, 5, 8, 16])
            c = _decode("", heads, rng.choice([1, 1, 2, 4, 16]), size(1, 64), size(16, 8192, page), size(32, 2048), ragged=ragged, draft=draft, page=page)
        elif op == "prefill":
            c = _prefill("", heads, size(1, 16), size(1, 1024), size(16, 8192, page), ragged=ragged, page=page)
        elif op == "cold":
            c = _cold("", dtype, hk, size(1, 16), size(16, 8192), ragged=ragged, page=page)
        elif op == "fork":
            c = _fork("", dtype, hk, size(1, 64), size(16, 8192), rng.choice([1, 2, 4, 8]), ragged=ragged, page=page)
        else:
            c = _compact("", dtype, hk, size(64, 8192), rng.uniform(0.1, 0.95), page=page)
        w = work(c)
        most = {"write": (1.1e8, math.inf), "decode": (1.2e9, 1.3e11), "prefill": (math.inf, 1.05e12), "cold": (2.8e8, math.inf), "fork": (1.2e8, math.inf), "compact": (3e8, math.inf)}[op]
        in_pool = _in_pool(c) * hk * D * 2 * {"bf16": 2, "fp8": 1, "fp32": 4}.get(c.get("dtype"), 0.5)
        if w["bytes"] <= most[0] and w["flops"] <= most[1] and in_pool <= 4e9:
            return c


# ------------------------------------------------------------------------------------------------- shapes
TORCH = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn, "fp32": torch.float32}
ELEM = {"bf16": 2, "fp8": 1, "fp32": 4}
FP4_TOKEN = 2 * (D // 2 + D // 32)  # bytes of a token's K and V of one head in 4 bits


def _ragged(case, count, most, least=1):
    """Token counts, fixed by the case alone."""
    rng = np.random.default_rng([count, most, int(1000 * case["ragged"])])
    return rng.integers(max(least, int(case["ragged"] * most)), max(least, most) + 1, size=count).astype(np.int64)


def _lengths(case):
    op = case["op"]
    if op == "write":
        return _ragged(case, case["n"], case["new"] or case["own"])
    if op == "decode":
        return _ragged(case, case["roots"] * case["fan"], case["own"], case["draft"])
    if op == "prefill":
        return _ragged(case, case["n"], case["new"])
    lens = _ragged(case, case["n"], case["tokens"])
    return lens + (lens % 16 == 0) if op == "fork" else lens  # (a last page that is full is shared like the others)


def _in_pool(case):
    """Tokens of room in the case's pages, about."""
    if case["op"] == "compact":
        return case["pages"] * case["page"]
    lens = _lengths(case)
    return int(lens.sum()) + case["page"] * len(lens) * case.get("fan", 1) + case.get("roots", 1) * case.get("prefix", 0)


def _moves(case):
    """compact: the pages in use, and those of them that move where."""
    n = case["pages"]
    n_live = min(n, max(1, int(case["live"] * n)))
    live = np.random.default_rng([n, n_live]).permutation(n)[:n_live].astype(np.int32)
    used = np.zeros(n, dtype=bool)
    used[live] = True
    return live, np.flatnonzero(used[n_live:]) + n_live, np.flatnonzero(~used[:n_live])


def _token_bytes(case):
    """K and V of one token and head in the case's own type."""
    e = ELEM[case["dtype"]]
    return 2 * D * e + (2 * 4 / 16 if e == 1 else 0)


def work(case):
    """write, cold: rows in, 4 bits out and in again, values out.  decode, prefill: every key and value of the forest, the rows in and out; 4 * 128
    operations per visible pair.  fork, compact: the blocks that have to be copied, in and out."""
    hk, op = case["kv_heads"], case["op"]
    if op == "compact":
        return {"bytes": 2 * len(_moves(case)[1]) * case["page"] * hk * _token_bytes(case), "flops": 0}
    lens = _lengths(case)
    if op == "write":
        new = int(lens.sum()) if case["new"] else len(lens)
        seen = int((-(-lens // 16)).sum()) * 16 if case["new"] else len(lens) * 16
        return {"bytes": hk * (new * (2 * D * 2 + FP4_TOKEN) + seen * (FP4_TOKEN + 2 * D * 2)), "flops": 0}
    if op == "cold":
        return {"bytes": int(lens.sum()) * hk * 2 * (_token_bytes(case) + FP4_TOKEN), "flops": 0}
    if op == "fork":
        return {"bytes": 2 * int((-(-(lens % case["page"]) // 16)).sum()) * 16 * case["fan"] * hk * _token_bytes(case), "flops": 0}
    hq = case["q_heads"]
    if op == "decode":
        T = case["draft"]
        tokens, rows = int(lens.sum()) + case["roots"] * case["prefix"], len(lens) * T
        pairs = case["prefix"] * rows + sum(T * (int(n) - T) + T * (T + 1) // 2 for n in lens)
    else:
        tokens, rows = int(lens.sum()) + case["prefix"], int(lens.sum())
        pairs = case["prefix"] * rows + sum(int(n) * (int(n) + 1) // 2 for n in lens)
    return {"bytes": tokens * hk * FP4_TOKEN + rows * hq * (2 * 2 * D + 4), "flops": 4 * D * hq * pairs}


def _layout(case, seed):
    """Pages in all, then page ids: of the shared prompts [roots][pages], of the sequences (one array each), of their places when they come back."""
    page, lens = case["page"], _lengths(case)
    roots = {"decode": case.get("roots"), "prefill": 1}.get(case["op"], 0)
    n_root = case["prefix"] // page if roots else 0
    n_own = [-(-int(n) // page) for n in lens]
    n_back = n_own if case["op"] == "cold" else []
    n_new = int((lens % page > 0).sum()) * case["fan"] if case["op"] == "fork" else 0
    used = roots * n_root + sum(n_own) + sum(n_back)
    total = used + (n_new if case["op"] == "fork" else used // 4 + 1)
    order = np.random.default_rng([int(seed), 5]).permutation(total).astype(np.int32)
    ends = np.cumsum([roots * n_root, *n_own, *n_back])
    parts = np.split(order, ends)
    return total, parts[0].reshape(roots, n_root), parts[1: 1 + len(lens)], parts[1 + len(lens): -1], parts[-1]


def _blocks(pages, page):
    """16-token blocks of a page list: block j of page p is p * (page / 16) + j."""
    s = page // 16
    return (np.asarray(pages, dtype=np.int64)[..., None] * s + np.arange(s)).reshape(*np.shape(pages)[:-1], -1)


def _table(lists, page, lens):
    """Blocks of the sequences, [n][blocks of the longest], those behind a sequence's end repeating its first."""
    out = np.zeros((len(lists), -(-int(lens.max()) // 16)), dtype=np.int64)
    for i, p in enumerate(lists):
        b = _blocks(p, page)[: -(-int(lens[i]) // 16)]
        out[i] = b[0]
        out[i, : len(b)] = b
    return out


# ------------------------------------------------------------------------------------------------- inputs
class _State:
    """What a program keeps between calls: page buffers, rows, indices of its tokens, and the library's pools and plan."""

    hkv = pool = other = plan = None

    def __del__(self):
        try:
            if self.plan is not None:
                (self.hkv.hkv_prefill_plan_destroy if self.case["op"] == "prefill" else self.hkv.hkv_decode_plan_destroy)(self.plan)
            for p in (self.pool, self.other):
                if p is not None:
                    self.hkv.kv_pool_destroy(p)
        except Exception:
            pass


def _cuda(a, dtype=torch.int64):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()


class _Pool:
    """Page buffers of one type."""

    def __init__(self, dtype, nb, hk):
        self.dtype, self.nb, self.hk, self.k_scale, self.v_scale = dtype, nb, hk, None, None
        n = nb * hk * 2048
        if dtype == "fp4":
            self.k, self.v = (torch.zeros(n // 2, dtype=torch.uint8, device="cuda") for _ in range(2))
            self.k_scale, self.v_scale = (torch.full((nb * hk * 64,), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        else:
            self.k, self.v = (torch.zeros(n, dtype=TORCH[dtype], device="cuda") for _ in range(2))
            if dtype == "fp8":
                self.k_scale, self.v_scale = (torch.ones(nb * hk, device="cuda") for _ in range(2))

    def outputs(self):
        out = {"k": self.k, "v": self.v}
        return out if self.dtype != "fp8" else out | {"k_scale": self.k_scale, "v_scale": self.v_scale}

    def open(self, hkv, page, free_order=None):
        dtype = {"bf16": hkv.BF16, "fp8": hkv.FP8_E4M3, "fp32": hkv.FP32, "fp4": hkv.FP4_E2M1}[self.dtype]
        return hkv.kv_pool_create(self.nb * 16 // page, self.hk, dtype, self.k, self.v, self.k_scale, self.v_scale, free_order, page_size=page)


def _inputs(case, seed):
    """Everything an operator reads, on the GPU, from the seed alone, and where the tokens lie."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 1000003 + 31)

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, dtype=dtype, device="cuda", generator=gen)

    s = _State()
    s.case, op, hk, page = case, case["op"], case["kv_heads"], case["page"]
    if op == "compact":
        nb = case["pages"] * page // 16
    else:
        lens = s.lens = _lengths(case)
        total, root_pages, own_pages, back_pages, s.fresh = s.pages = _layout(case, seed)
        nb = total * page // 16
        s.lens_gpu = _cuda(lens)
        s.own_blocks = _cuda(_table(own_pages, page, lens))
    s.a = _Pool(case.get("dtype", "fp4"), nb, hk)
    if s.a.dtype == "fp8":  # codes as a writer leaves them: block maxima near 448
        for t in (s.a.k, s.a.v):
            for i in range(0, t.numel(), 1 << 27):
                t[i: i + (1 << 27)] = (normal(min(t.numel() - i, 1 << 27)) * 120).clamp_(-448, 448).to(torch.float8_e4m3fn)
        s.a.k_scale.uniform_(0.006, 0.011, generator=gen)
        s.a.v_scale.uniform_(0.006, 0.011, generator=gen)
    elif s.a.dtype == "fp4":  # normal numbers that went through the store
        for i in range(0, nb, 1 << 13):
            at = torch.arange(i, min(nb, i + (1 << 13)), device="cuda")
            for is_k in (True, False):
                _put4(s.a, is_k, at, normal(len(at), hk, 16, D))
    else:
        s.a.k.normal_(generator=gen)
        s.a.v.normal_(generator=gen)
    if op == "write":
        new = lens if case["new"] else np.ones(len(lens), dtype=np.int64)
        s.k_new, s.v_new = (normal(int(new.sum()), hk, D, dtype=torch.bfloat16) for _ in range(2))
        # the new tokens' places, request by request, and the blocks that they are in
        at = np.concatenate([np.arange(n) if case["new"] else [n - 1] for n in lens])
        seq = np.repeat(np.arange(len(lens)), new)
        table = s.own_blocks.cpu().numpy()
        s.block, s.slot = _cuda(table[seq, at // 16]), _cuda(at % 16)
        s.ends = np.concatenate([[0], np.cumsum(new)])
        s.last = (np.stack([p[(n - 1) // page] for p, n in zip(own_pages, lens)]), ((lens - 1) % page).astype(np.int32))
        s.seen = np.concatenate(own_pages) if case["new"] else s.last[0]  # pages that are read back: whole prompts, or the last page of each call
        s.seen_tokens = np.concatenate([np.minimum(page, -(-n // 16) * 16 - page * np.arange(len(p))) for p, n in zip(own_pages, lens)]) if case["new"] else s.last[1] // 16 * 16 + 16
        s.b = _Pool("bf16", nb, hk)
        b = _blocks(s.seen[:, None], page)
        s.seen_blocks = _cuda(b[np.arange(b.shape[1]) < s.seen_tokens[:, None] // 16])
    elif op == "decode":
        s.q = normal(len(lens) * case["draft"], case["q_heads"], D, dtype=torch.bfloat16) * 2
        s.root_blocks = _cuda(_blocks(root_pages, page))
    elif op == "prefill":
        n, rows = len(lens), int(lens.sum())
        s.q = normal(rows, case["q_heads"], D, dtype=torch.bfloat16) * 2
        s.root_blocks = _cuda(_blocks(root_pages, page))
        s.row_at = _cuda(np.concatenate([i * int(lens.max()) + np.arange(m) for i, m in enumerate(lens)]))  # a row's place in [n][longest]
    elif op == "cold":
        s.b = _Pool("fp4", int(sum(len(p) for p in own_pages)) * page // 16, hk)
        s.src, s.dst = np.concatenate(own_pages), np.concatenate(back_pages)
        s.mid = np.random.default_rng([int(seed), 6]).permutation(len(s.src)).astype(np.int32)
        s.tokens = np.concatenate([np.minimum(page, n - page * np.arange(len(p))) for p, n in zip(own_pages, lens)]).astype(np.int32)
        at = np.concatenate([np.arange(n) for n in lens])
        seq = np.repeat(np.arange(len(lens)), lens)
        first = np.concatenate([[0], np.cumsum([len(p) for p in own_pages])])[:-1]  # of a sequence's pages in the lists
        in_list, block = first[seq] + at // page, at % page // 16
        s.block, s.back, s.mid_block = (_cuda(p[in_list].astype(np.int64) * (page // 16) + block) for p in (s.src, s.dst, s.mid))
        s.slot = _cuda(at % 16)
        unit = np.concatenate([[True], (block[1:] != block[:-1]) | (in_list[1:] != in_list[:-1])])
        s.unit, s.unit_block = _cuda(np.cumsum(unit) - 1), s.back[_cuda(np.flatnonzero(unit))]
    elif op == "fork":
        s.parent = np.random.default_rng([int(seed), 7]).permutation(np.repeat(np.arange(len(lens)), case["fan"])).astype(np.int32)
        s.own_pages = np.concatenate(own_pages)
    else:
        s.live, s.moved, s.gaps = _moves(case)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op in ("decode", "prefill"):
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty(s.q.shape[:2], device="cuda")
    if own:
        from paper_2603_16104_amd import binding as hkv
        s.hkv, page = hkv, case["page"]
        s.stream = torch.cuda.current_stream().cuda_stream
        order = None
        if op == "fork":
            order = np.concatenate([s.own_pages, s.fresh])
        elif op == "compact":
            order = np.concatenate([s.live, np.setdiff1d(np.arange(case["pages"], dtype=np.int32), s.live)])
        s.pool = s.a.open(hkv, page, order)
        if op in ("write", "cold"):
            s.other = s.b.open(hkv, page)
        elif op == "fork":
            hkv.kv_pool_alloc(s.pool, len(s.own_pages))
        elif op == "compact":
            hkv.kv_pool_alloc(s.pool, len(s.live))
            s.rest, s.gone = case["pages"] - len(s.live), np.concatenate([s.gaps, np.setdiff1d(np.arange(len(s.live), case["pages"]), s.moved)]).astype(np.int32)
        elif op == "prefill":
            _, root_pages, own_pages, _, _ = s.pages
            cu = np.concatenate([[0], np.cumsum(s.lens)]).astype(np.int32)
            table = np.full((len(s.lens), root_pages.shape[1] + max(len(p) for p in own_pages)), -1, dtype=np.int32)
            table[:, : root_pages.shape[1]] = root_pages
            for i, p in enumerate(own_pages):
                table[i, root_pages.shape[1]: root_pages.shape[1] + len(p)] = p
            s.plan = hkv.hkv_prefill_plan_create(s.pool, cu, table, case["prefix"] + s.lens, case["q_heads"])
            s.ws_bytes = hkv.hkv_prefill_plan_workspace_bytes(s.plan)
        else:
            s.plan = hkv.hkv_decode_plan_create_multi(s.pool, *_forest(s), case["draft"], case["q_heads"])
            s.ws_bytes = hkv.hkv_decode_plan_workspace_bytes(s.plan)
        if op in ("decode", "prefill"):
            s.ws = torch.empty(max(256, s.ws_bytes), dtype=torch.uint8, device="cuda")
    return s


def _forest(s):
    """The requests as the library takes them: shared prompts, then a node for each request."""
    case = s.case
    _, root_pages, own_pages, _, _ = s.pages
    nodes, begin = [], 0
    for p in root_pages:
        nodes.append((-1, begin, len(p), case["prefix"]))
        begin += len(p)
    for i, (p, n) in enumerate(zip(own_pages, s.lens)):
        nodes.append((i // case["fan"], begin, len(p), int(n)))
        begin += len(p)
    return np.asarray(nodes, dtype=np.int32), np.concatenate([root_pages.ravel(), *own_pages]), np.arange(case["roots"], case["roots"] + len(s.lens), dtype=np.int32)


# ------------------------------------------------------------------------------------------------- one pass
def run(s):
    op = s.case["op"]
    if own:
        return _own(s, op)
    if op == "write":
        for is_k, x in ((True, s.k_new), (False, s.v_new)):
            _put4_tokens(s.a, is_k, s.block, s.slot, x.float())
            _put(s.b, is_k, s.seen_blocks, _values4(s.a, is_k, s.seen_blocks))
        return s.b.outputs()
    if op in ("decode", "prefill"):
        (_plain_decode if op == "decode" else _plain_prefill)(s)
        return {"out": s.out, "lse": s.lse}
    if op == "cold":
        for is_k in (True, False):
            _put4_tokens(s.b, is_k, s.mid_block, s.slot, _tokens(s.a, is_k, s.block, s.slot))
            _put_tokens(s, is_k, _tokens4(s.b, is_k, s.mid_block, s.slot))
        return s.a.outputs()
    if op == "fork":
        return s.a.outputs() | {"pages": _plain_fork(s)}
    new = np.full(s.case["pages"], -1, dtype=np.int32)
    new[s.live] = s.live
    new[s.moved] = s.gaps
    _copy_pages(s.a, s.case["page"], s.moved, s.gaps)
    return s.a.outputs() | {"pages": new}


def _own(s, op):
    hkv, case = s.hkv, s.case
    if op == "write":
        if case["new"]:
            for i, pages in enumerate(s.pages[2]):
                a, b = int(s.ends[i]), int(s.ends[i + 1])
                hkv.kv_pool_write(s.pool, pages, 0, b - a, s.k_new[a:b], s.v_new[a:b], s.stream)
        else:
            hkv.kv_pool_append(s.pool, *s.last, s.k_new, s.v_new, s.stream)
        hkv.kv_pool_copy_pages(s.other, s.seen, s.pool, s.seen, s.seen_tokens, s.stream)
        return s.b.outputs()
    if op == "decode":
        hkv.attn_decode_plan_run(s.plan, s.q, SCALE, s.out, s.lse, s.ws, s.ws_bytes, s.stream)
        return {"out": s.out, "lse": s.lse}
    if op == "prefill":
        hkv.attn_prefill_plan_run(s.plan, s.q, SCALE, s.out, s.lse, s.stream, s.ws, s.ws_bytes)
        return {"out": s.out, "lse": s.lse}
    if op == "cold":
        hkv.kv_pool_copy_pages(s.other, s.mid, s.pool, s.src, s.tokens, s.stream)
        hkv.kv_pool_copy_pages(s.pool, s.dst, s.other, s.mid, s.tokens, s.stream)
        return s.a.outputs()
    if op == "fork":  # the branches are dropped again
        pages = hkv.kv_pool_fork(s.pool, s.own_pages, s.lens, s.parent, stream=s.stream)
        hkv.kv_pool_release(s.pool, pages)
        return s.a.outputs() | {"pages": pages}
    pages = hkv.kv_pool_compact(s.pool, s.stream)
    hkv.kv_pool_alloc(s.pool, s.rest)  # calls come and go until the same pages are in use again
    hkv.kv_pool_release(s.pool, s.gone)
    return s.a.outputs() | {"pages": pages}


# ------------------------------------------------------------------------------------------------- plain forms
def _codes4(x):
    """Codes 0 .. 15 and scale bytes of rows [..., 128]: the scale is 2^(floor(log2 of the largest) - 2), codes round to nearest, ties to the even one."""
    x = x.unflatten(-1, (4, 32))
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, torch.full_like(top, -126, dtype=torch.int32)).clamp(-126, 125)
    y = x * ((127 - e) << 23).view(torch.float32)[..., None]
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0) + 8 * torch.signbit(y)
    return code.flatten(-2).to(torch.uint8), (e + 127).to(torch.uint8)


def _bytes(codes):
    return codes[..., 0::2] | codes[..., 1::2] << 4


def _view4(p, is_k):
    """The codes' bytes as [block][head][...] and the scales as [block][head][group][token]."""
    if is_k:
        return p.k.view(p.nb, p.hk, 4, 4, 64), p.k_scale.view(p.nb, p.hk, 4, 16)
    return p.v.view(p.nb, p.hk, 4, 16, 4, 4), p.v_scale.view(p.nb, p.hk, 4, 16)


def _put4(p, is_k, blocks, x):
    """Whole blocks [n][head][16][128]."""
    codes, scale = _codes4(x)
    view, scales = _view4(p, is_k)
    b = _bytes(codes).unflatten(2, (4, 4))  # [n][head][t / 4][t % 4][64]
    view[blocks] = b.transpose(2, 3) if is_k else b.unflatten(4, (16, 4)).permute(0, 1, 2, 4, 3, 5)
    scales[blocks] = scale.transpose(2, 3)


def _put4_tokens(p, is_k, block, slot, x):
    """Rows [n][head][128] at a slot of a block each."""
    codes, scale = _codes4(x)
    view, scales = _view4(p, is_k)
    b = _bytes(codes)
    if is_k:
        view[block, :, slot % 4, slot // 4] = b
    else:
        view[block, :, slot // 4, :, slot % 4] = b.unflatten(2, (16, 4))
    scales[block, :, :, slot] = scale


def _pairs(device="cuda"):
    v = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=device)
    i = torch.arange(256, device=device)
    return torch.stack([v[i & 15], v[i >> 4]], dim=1)


def _scales(b):
    return (b.int() << 23).view(torch.float32)


def _values4(p, is_k, blocks):
    """What the listed blocks hold: [...][head][16][128]."""
    view, scales = _view4(p, is_k)
    b = view[blocks]
    lead = blocks.dim()
    b = b.transpose(lead + 1, lead + 2) if is_k else b.transpose(lead + 2, lead + 3)  # [...][head][t / 4][t % 4][64 bytes]
    x = _pairs()[b.reshape(*blocks.shape, p.hk, 16, 64).int()].flatten(-2)
    return (x.unflatten(-1, (4, 32)) * _scales(scales[blocks]).transpose(-1, -2)[..., None]).flatten(-2)


def _tokens4(p, is_k, block, slot):
    view, scales = _view4(p, is_k)
    b = view[block, :, slot % 4, slot // 4] if is_k else view[block, :, slot // 4, :, slot % 4].flatten(2)
    x = _pairs()[b.int()].flatten(-2)
    return (x.unflatten(-1, (4, 32)) * _scales(scales[block, :, :, slot])[..., None]).flatten(-2)


def _view(p, is_k):
    """The elements as [block][head][chunk][token][dim of the chunk] (K) or [block][head][dim][token] (V)."""
    c = 64 // p.k.element_size()
    return p.k.view(p.nb, p.hk, D // c, 16, c) if is_k else p.v.view(p.nb, p.hk, D, 16)


def _put(p, is_k, blocks, x):
    view = _view(p, is_k)
    view[blocks] = (x.unflatten(3, (view.shape[2], -1)).transpose(2, 3) if is_k else x.transpose(2, 3)).to(view.dtype)


def _tokens(p, is_k, block, slot):
    view = _view(p, is_k)
    x = (view[block, :, :, slot].flatten(2) if is_k else view[block, :, :, slot]).float()
    scale = p.k_scale if is_k else p.v_scale
    return x if scale is None else x * scale.view(p.nb, p.hk)[block][..., None]


def _put_tokens(s, is_k, x):
    """Rows [n][head][128] to where they come back, fp8 with a scale of each block's largest."""
    p, view = s.a, _view(s.a, is_k)
    if p.dtype == "fp8":
        top = torch.zeros(len(s.unit_block), p.hk, device="cuda")
        top.scatter_reduce_(0, s.unit[:, None].expand(-1, p.hk), x.abs().amax(-1), "amax")
        scale = torch.where(top > 0, top / torch.full_like(top, 448.0), torch.ones_like(top))
        (p.k_scale if is_k else p.v_scale).view(p.nb, p.hk)[s.unit_block] = scale
        x = (x / scale[s.unit][..., None]).clamp(-448.0, 448.0)
    x = x.to(view.dtype)
    view[s.back, :, :, s.slot] = x.unflatten(2, (view.shape[2], -1)) if is_k else x


def _grouped(x, hk, nodes):
    """[rows][q head][...] as [nodes][KV head][rows of the node x heads of the group][...]."""
    return x.unflatten(1, (hk, -1)).unflatten(0, (nodes, -1)).transpose(1, 2).flatten(2, 3)


def _rows(x, nodes, rows):
    """The way back: [nodes][KV head][rows x group][...] as [rows][q head][...]."""
    return x.unflatten(2, (rows, -1)).transpose(1, 2).flatten(2, 3).flatten(0, 1)


def _keys(p, is_k, blocks):
    """[nodes][KV head][tokens][128]."""
    return _values4(p, is_k, blocks).transpose(1, 2).flatten(2, 3)


def _products(q, k):
    return torch.matmul(q, k.transpose(2, 3).contiguous()) * SCALE


def _plain_decode(s):
    c, T, hk, n = s.case, s.case["draft"], s.case["kv_heads"], len(s.lens)
    q = s.q.float()
    root = _products(_grouped(q, hk, c["roots"]), _keys(s.a, True, s.root_blocks))
    mine = _products(_grouped(q, hk, n), _keys(s.a, True, s.own_blocks))
    t, row = torch.arange(mine.shape[3], device="cuda"), torch.arange(mine.shape[2], device="cuda") // (mine.shape[2] // T)
    last = (s.lens_gpu - T)[:, None] + row  # the newest key that a row sees
    mine.masked_fill_((t > last[:, :, None])[:, None], -math.inf)
    rows = c["fan"] * T
    top = torch.maximum(_rows(root.amax(3), c["roots"], rows), _rows(mine.amax(3), n, T))
    root = torch.exp(root - _grouped(top, hk, c["roots"])[..., None])
    mine = torch.exp(mine - _grouped(top, hk, n)[..., None])
    total = _rows(root.sum(3), c["roots"], rows) + _rows(mine.sum(3), n, T)
    o = _rows(torch.matmul(root, _keys(s.a, False, s.root_blocks)), c["roots"], rows) + _rows(torch.matmul(mine, _keys(s.a, False, s.own_blocks)), n, T)
    s.out.copy_(o / total[..., None])
    s.lse.copy_(top + torch.log(total))


def _plain_prefill(s):
    c, hk, n, longest = s.case, s.case["kv_heads"], len(s.lens), int(s.lens.max())
    q = torch.zeros(n * longest, *s.q.shape[1:], device="cuda")
    q[s.row_at] = s.q.float()
    q = _grouped(q, hk, n)
    x = torch.cat([_products(q, _keys(s.a, True, s.root_blocks).expand(n, -1, -1, -1)), _products(q, _keys(s.a, True, s.own_blocks))], dim=3)
    t, row = torch.arange(x.shape[3], device="cuda"), torch.arange(x.shape[2], device="cuda") // (x.shape[2] // longest)
    x.masked_fill_(t > c["prefix"] + row[:, None], -math.inf)
    top = x.amax(3, keepdim=True)
    x = x.sub_(top).exp_()
    total = x.sum(3)
    o = torch.matmul(x[..., : c["prefix"]], _keys(s.a, False, s.root_blocks).expand(n, -1, -1, -1)) + torch.matmul(x[..., c["prefix"]:], _keys(s.a, False, s.own_blocks))
    s.out.copy_(_rows(o / total[..., None], n, longest)[s.row_at])
    s.lse.copy_(_rows(top[..., 0] + torch.log(total), n, longest)[s.row_at])


def _copy_pages(p, page, src, dst, tokens=None):
    """Pages of one pool, or of each the 16-token blocks that hold its first tokens."""
    a, b = _blocks(src[:, None], page), _blocks(dst[:, None], page)
    used = slice(None) if tokens is None else np.arange(page // 16) < -(-tokens // 16)[:, None]
    a, b = _cuda(a[used].ravel()), _cuda(b[used].ravel())
    for x in (p.k, p.v, p.k_scale, p.v_scale):
        if x is not None:
            x = x.view(p.nb, -1)
            x = x.view(torch.uint8) if x.element_size() == 1 else x
            x[b] = x[a]


def _plain_fork(s):
    page, lens, parent = s.case["page"], s.lens, s.parent
    n_pages = -(-lens // page)
    ends = np.cumsum(n_pages)
    count = n_pages[parent]
    at = np.arange(count.sum()) - np.repeat(np.cumsum(count) - count, count) + np.repeat((ends - n_pages)[parent], count)
    pages = s.own_pages[at]
    cut = lens[parent] % page > 0
    last = (np.cumsum(count) - 1)[cut]
    fresh = s.fresh[: len(last)]
    _copy_pages(s.a, page, pages[last], fresh, lens[parent][cut] % page)
    pages[last] = fresh
    return pages


# ------------------------------------------------------------------------------------------------- the same in 64 bits
def exact(case, seed):
    if case["op"] in ("fork", "compact"):
        return None  # (nothing is computed)
    s = _inputs(case, seed)
    return {"write": _exact_write, "decode": _exact_decode, "prefill": _exact_prefill, "cold": _exact_cold}[case["op"]](s, case)


def _read64(p, is_k, block, head, slot, dim):
    """Single values of a 4-bit pool, by the formulas of its format."""
    at = slot % 4 * 256 + slot // 4 * 64 + dim // 2 if is_k else slot // 4 * 256 + dim // 8 * 16 + slot % 4 * 4 + dim % 8 // 2
    base = block * p.hk + head
    code = (p.k if is_k else p.v)[base * 1024 + at].long() >> 4 * (dim % 2) & 15
    e, m = code >> 1 & 3, code & 1
    size = torch.where(e > 0, (1 + 0.5 * m.double()) * 2.0 ** (e - 1).double(), 0.5 * m.double())
    exponent = (p.k_scale if is_k else p.v_scale)[base * 64 + dim // 32 * 16 + slot].double() - 127
    return torch.where(code > 7, -size, size) * 2.0 ** exponent


def _nearest64(x):
    """Rows [..., 128] as 4 bits hold them: of the eight sizes the nearest, of two equally near ones that of even number."""
    x = x.double().unflatten(-1, (4, 32))
    sizes = torch.tensor([0, 1, 2, 4, 0.5, 1.5, 3, 6], dtype=torch.float64, device="cuda")  # numbers 0, 2, 4, 6, 1, 3, 5, 7: argmin takes the first of equals
    top = x.abs().amax(-1, keepdim=True)
    unit = 2.0 ** (torch.floor(torch.log2(top.clamp_min(2.0 ** -124))) - 2).clamp(-126, 125)
    near = (x.abs() / unit)[..., None] - sizes
    return (torch.sign(x) * sizes[near.abs_().argmin(-1)] * unit).flatten(-2)


def _flat(block, hk, head, slot, dim, elem, is_k):
    """Element of the other pools' buffers that holds (slot, dim) of a block and head."""
    c = 64 // elem
    return (block * hk + head) * 2048 + ((dim // c) * 16 * c + slot * c + dim % c if is_k else dim * 16 + slot)


def _exact_write(s, case):
    hk, out = case["kv_heads"], {}
    dim, head, slot = torch.arange(D, device="cuda"), torch.arange(hk, device="cuda")[:, None], torch.arange(16, device="cuda")[:, None, None]
    for name, is_k, x in (("k", True, s.k_new), ("v", False, s.v_new)):
        got = torch.zeros_like(s.b.k, dtype=torch.float64)
        b = s.seen_blocks[:, None, None, None]
        got[_flat(b, hk, head, slot, dim, 2, is_k)] = _read64(s.a, is_k, b, head, slot, dim)
        got[_flat(s.block[:, None, None], hk, head, s.slot[:, None, None], dim, 2, is_k)] = _nearest64(x)
        out[name] = got
    return out


def _sequence64(p, is_k, blocks, n):
    """[head][n][128] of a list of blocks."""
    t, head, dim = torch.arange(n, device="cuda"), torch.arange(p.hk, device="cuda")[:, None, None], torch.arange(D, device="cuda")
    return _read64(p, is_k, blocks[t // 16][:, None], head, (t % 16)[:, None], dim)


def _attend64(q, k, v, seen):
    """Rows q [rows][q head][128], of which row i sees the first seen[i] of the keys [head][n][128]."""
    hk, n = k.shape[:2]
    q = q.double().view(q.shape[0], hk, -1, D).permute(1, 0, 2, 3).flatten(1, 2)     # [head][rows x group][128]
    x = torch.bmm(q, k.transpose(1, 2).contiguous()) * SCALE
    x.view(hk, len(seen), -1, n).masked_fill_(torch.arange(n, device="cuda") >= seen[:, None, None], -math.inf)
    lse = torch.logsumexp(x, dim=2)
    o = torch.bmm(torch.exp(x - lse[..., None]), v)
    back = lambda y: y.unflatten(1, (len(seen), -1)).transpose(0, 1).flatten(1, 2)  # noqa: E731
    return back(o), back(lse)


def _exact_decode(s, case):
    T, P, fan = case["draft"], case["prefix"], case["fan"]
    out, lse = [], []
    root = None
    for i, n in enumerate(s.lens.tolist()):
        if i % fan == 0:
            root = [_sequence64(s.a, is_k, s.root_blocks[i // fan], P) for is_k in (True, False)]
        k, v = (torch.cat([r, _sequence64(s.a, is_k, s.own_blocks[i], n)], dim=1) for r, is_k in zip(root, (True, False)))
        o, x = _attend64(s.q[i * T: (i + 1) * T], k, v, P + n - T + 1 + torch.arange(T, device="cuda"))
        out.append(o)
        lse.append(x)
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_prefill(s, case):
    P, out, lse, first = case["prefix"], [], [], 0
    root = [_sequence64(s.a, is_k, s.root_blocks[0], P) for is_k in (True, False)]
    for i, n in enumerate(s.lens.tolist()):
        k, v = (torch.cat([r, _sequence64(s.a, is_k, s.own_blocks[i], n)], dim=1) for r, is_k in zip(root, (True, False)))
        for a in range(0, n, 256):
            b = min(n, a + 256)
            o, x = _attend64(s.q[first + a: first + b], k, v, P + 1 + torch.arange(a, b, device="cuda"))
            out.append(o)
            lse.append(x)
        first += n
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_cold(s, case):
    hk, e, out = case["kv_heads"], ELEM[case["dtype"]], {}
    dim, head = torch.arange(D, device="cuda"), torch.arange(hk, device="cuda")
    for name, is_k in (("k", True), ("v", False)):
        buf, scales = (s.a.k, s.a.k_scale) if is_k else (s.a.v, s.a.v_scale)
        x = buf.double()[_flat(s.block[:, None, None], hk, head[:, None], s.slot[:, None, None], dim, e, is_k)]
        if scales is not None:
            x = x * scales.double().view(-1, hk)[s.block][..., None]
        x = _nearest64(x)
        if scales is not None:
            scales = scales.double().view(-1, hk).clone()
            top = torch.zeros_like(scales).index_reduce_(0, s.back, x.abs().amax(-1), "amax")[s.unit_block]
            scales[s.unit_block] = torch.where(top > 0, top / 448.0, torch.ones_like(top))
            x = x / scales[s.back][..., None]
            out[name + "_scale"] = scales.flatten()
        got = buf.double()
        got[_flat(s.back[:, None, None], hk, head[:, None], s.slot[:, None, None], dim, e, is_k)] = x
        out[name] = got
    return out

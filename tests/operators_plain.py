"""Plain 64-bit forms of the calls around a step's attention, on the host, for the tests: rows into a pool, weights of cached keys,
eviction.  A pool is here a pair of arrays [16-token blocks][kv heads][16 tokens][128]."""
import numpy as np
import torch

from paper_2603_16104_amd import binding as hkv

TORCH = {hkv.BF16: torch.bfloat16, hkv.FP8_E4M3: torch.float8_e4m3fn, hkv.FP32: torch.float32}
HALF_STEP = {hkv.BF16: 2.0 ** -8, hkv.FP8_E4M3: 2.0 ** -4, hkv.FP32: 2.0 ** -24}


class Pool:
    """Device buffers of a pool full of random values, and its handle."""

    def __init__(self, pages, heads, dtype, page_size=16, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        n = pages * page_size * heads * 128
        self.heads, self.dtype, self.page_size, self.blocks = heads, dtype, page_size, pages * page_size // 16

        def fill():
            x = torch.randn(n, device="cuda", generator=g)
            return (x * 100).clamp_(-448, 448).to(torch.float8_e4m3fn) if dtype == hkv.FP8_E4M3 else x.to(TORCH[dtype])

        self.k, self.v = fill(), fill()
        self.k_scale = self.v_scale = None
        if dtype == hkv.FP8_E4M3:
            self.k_scale, self.v_scale = (torch.empty(self.blocks * heads, device="cuda").uniform_(0.004, 0.009, generator=g) for _ in range(2))
        self.handle = hkv.kv_pool_create(pages, heads, dtype, self.k, self.v, self.k_scale, self.v_scale, page_size=page_size)

    def close(self):
        hkv.kv_pool_destroy(self.handle)

    def codes(self, t, is_k):
        """One buffer as [blocks][heads][16][128] float64, without scales."""
        x = t.cpu().float().double()
        if is_k:
            c = 64 // t.element_size()
            return x.view(self.blocks, self.heads, 128 // c, 16, c).transpose(2, 3).reshape(self.blocks, self.heads, 16, 128).numpy()
        return x.view(self.blocks, self.heads, 128, 16).transpose(2, 3).contiguous().numpy()

    def scales(self):
        if self.k_scale is None:
            one = np.ones((self.blocks, self.heads))
            return one, one
        return tuple(s.cpu().double().view(self.blocks, self.heads).numpy() for s in (self.k_scale, self.v_scale))

    def snapshot(self):
        (ks, vs) = self.scales()
        return self.codes(self.k, True), self.codes(self.v, False), ks.copy(), vs.copy()

    def values(self):
        k, v, ks, vs = self.snapshot()
        return k * ks[:, :, None, None], v * vs[:, :, None, None]


def blocks_of(pages, page_size):
    s = page_size // 16
    return np.asarray([p * s + j for p in pages for j in range(s)], dtype=np.int64)


def normed(x, w, eps):
    x = x.cpu().double().numpy()
    with np.errstate(invalid="ignore"):
        return x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + np.float64(np.float32(eps))) * w.cpu().double().numpy()


def turned(y, angle, interleaved):
    """y [rows][heads][128], angle [rows][pairs] -> (z, size of what each element was made of)."""
    n = angle.shape[1]
    a, b = (np.arange(n) * 2, np.arange(n) * 2 + 1) if interleaved else (np.arange(n), np.arange(n) + n)
    z, size = y.copy(), np.abs(y)
    co, si = np.cos(angle)[:, None], np.sin(angle)[:, None]
    z[..., a], z[..., b] = y[..., a] * co - y[..., b] * si, y[..., b] * co + y[..., a] * si
    size[..., a] = size[..., b] = np.abs(y[..., a]) + np.abs(y[..., b])
    return z, size


# What a row's element may be off before it is rounded, relative to the values it is made of.  The sum of 128 squares is 8 + 4
# additions and its root halves that, scaling takes three roundings, the rotation three, the sine and cosine 1.25e-7 (2.1 * 2^-24) and the
# part of a turn is narrowed to 2^-26 of a turn (1.6 * 2^-24 in the angle): below 20 * 2^-24.
ROW = 2.0 ** -19


def check_rows(got, z, size, dtype, what):
    """Rows that were rounded once, to bf16 or fp32."""
    err = np.abs(got - z)
    tol = HALF_STEP[dtype] * np.abs(z) + (1 + HALF_STEP[dtype]) * ROW * size + 1e-38
    worst = np.max(err / tol) if err.size else 0.0
    assert np.isfinite(got).all() and worst <= 1, f"{what}: {worst:.3g} of what it may be off"


def check_store(pool, before, places, k, k_size, v, what=""):
    """The pool after a store: places: per unit (block, low slot, rows of k / v in slot order); everything else as `before`."""
    bk, bv, bks, bvs = before
    gk, gv, gks, gvs = pool.snapshot()
    touched = np.zeros((pool.blocks, 16), dtype=bool)
    fp8 = pool.dtype == hkv.FP8_E4M3
    for block, low, rows in places:
        n = len(rows)
        touched[block, low: low + n] = True
        for name, got, gs, old_codes, old_s, x, size in (("K", gk, gks, bk, bks, k, k_size), ("V", gv, gvs, bv, bvs, v, np.abs(v))):
            z, sz = x[rows].transpose(1, 0, 2), size[rows].transpose(1, 0, 2)       # [heads][n][128]
            new = got[block, :, low: low + n]
            where = f"{what} {name} of block {block}"
            if not fp8:
                step = HALF_STEP[pool.dtype] if name == "K" else 0.0
                assert (np.abs(new - z) <= step * np.abs(z) + (0 if name == "V" else 2 * ROW * sz) + 1e-38).all(), where
                continue
            want = np.abs(z).max((1, 2)) / 448
            slack = 2.0 ** -22 * want + (0 if name == "V" else ROW * sz.max((1, 2)) / 448)  # a division and what the keys are off
            want = np.where(want == 0, 0 if low else 1, want)
            if low:
                want = np.maximum(want, old_s[block])
            s = gs[block]
            assert (np.abs(s - want) <= slack).all(), f"{where}: scales {s} for {want}"
            tol = 2.0 ** -4 * np.abs(z) + 2.0 ** -10 * s[:, None, None] + 2 * ROW * sz
            assert (np.abs(new * s[:, None, None] - z) <= tol).all(), where
            if low:                                                                 # the earlier tokens, rounded again where the scale grew
                old = old_codes[block, :, :low] * old_s[block][:, None, None]
                now = got[block, :, :low] * s[:, None, None]
                grew = s > old_s[block]
                tol = (2.0 ** -4 * np.abs(old) + 2.0 ** -10 * s[:, None, None]) * grew[:, None, None]
                assert (np.abs(now - old) <= tol + 1e-6 * np.abs(old)).all(), where + ", earlier tokens"
                assert (got[block, ~grew, :low] == old_codes[block, ~grew, :low]).all(), where + ", earlier tokens under an old scale"
                touched[block, :low] = True
    rest = ~touched[:, None, :, None] & np.ones_like(bk, dtype=bool)
    assert (gk[rest] == bk[rest]).all() and (gv[rest] == bv[rest]).all(), what + ": slots that no token goes to"
    if fp8:
        others = np.setdiff1d(np.arange(pool.blocks), [b for b, *_ in places])
        assert (gks[others] == bks[others]).all() and (gvs[others] == bvs[others]).all(), what + ": other blocks' scales"


def key_weights(k_values, nodes, q, lse, scale, heads, old, decay, n_new, T):
    """nodes: per node (blocks, tokens, rows, per row the visible tokens as a mask [rows][tokens], is it a last node)."""
    out = old.astype(np.float64).copy()
    G = q.shape[1] // heads
    for blocks, n, rows, seen, last in nodes:
        if len(rows) == 0 or n == 0:
            continue
        t = np.arange(n)
        b = blocks[t // 16]
        for h in range(heads):
            keys = k_values[b, h, t % 16]
            qs = q[rows][:, h * G: (h + 1) * G]                                     # [rows][G][128]
            l = lse[rows][:, h * G: (h + 1) * G]
            counts = np.isfinite(l)[..., None]
            x = np.einsum("rgd,td->rgt", np.where(counts, qs, 0), keys) * scale - np.where(counts, l[..., None], 0)
            w = np.exp(np.where(counts & seen[:, None, :], x, -np.inf)).sum((0, 1))
            fresh = last & (t >= n - n_new)
            was = np.where(fresh | (decay == 0), 0.0, out[b, h, t % 16])
            out[b, h, t % 16] = w + decay * was
    return out


def evicted(weights, blocks, n, keep, first, recent):
    """Kept tokens of one sequence and head's weights [tokens]."""
    w = weights[blocks[np.arange(n) // 16], np.arange(n) % 16].astype(np.float64) if n else np.zeros(0)
    key = np.where(np.isnan(w), -np.inf, w)
    rank = np.lexsort((np.arange(n), -key, np.isnan(w)))                            # numbers first, heavy ones first, then the earlier
    must = (np.arange(n) < first) | (np.arange(n) >= n - recent)
    rest = [t for t in rank if not must[t]][: max(0, keep - int(must.sum()))]
    return np.sort(np.concatenate([np.flatnonzero(must), np.asarray(rest, dtype=np.int64)])).astype(np.int64)

"""4-bit pools in plain 64-bit form, on the host, for the tests: the format, the stores, attention."""
import math

import numpy as np
import torch

from paper_2603_16104_amd import binding as hkv

SIZES = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
STEP = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}  # a rounding's largest error, relative


def quantised(x):
    """Rows [..., 128]: (codes, scale bytes [..., 4], values), from the definition: scale 2^(floor(log2 of the largest) - 2), the nearest size, of two
    equally near ones the even code."""
    x = np.asarray(x, dtype=np.float64).reshape(*np.shape(x)[:-1], 4, 32)
    top = np.abs(x).max(-1)
    e = np.where(top > 0, np.frexp(top)[1] - 1 - 2, -126).clip(-126, 125)
    y = x / np.exp2(e)[..., None]
    far = np.abs(np.abs(y)[..., None] - SIZES)
    order = [0, 2, 4, 6, 1, 3, 5, 7]
    code = np.array(order)[far[..., order].argmin(-1)]
    code = code + 8 * np.signbit(y)
    value = np.where(code > 7, -1, 1) * SIZES[code & 7] * np.exp2(e)[..., None]
    flat = (*x.shape[:-2], 128)
    return code.reshape(flat), (e + 127).astype(np.uint8), value.reshape(flat)


def code_at(is_k, t, d):
    """Byte of a block's 1024 that holds dims d, d + 1 (d even) of slot t."""
    return t % 4 * 256 + t // 4 * 64 + d // 2 if is_k else t // 4 * 256 + d // 8 * 16 + t % 4 * 4 + d % 8 // 2


class Pool:
    """Device buffers of a 4-bit pool that holds random codes under scales near 1 (`poison`: bytes that stand for no number), and its handle."""

    dtype = hkv.FP4_E2M1

    def __init__(self, pages, heads, page_size=16, seed=0, poison=False, free_order=None):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.heads, self.page_size, self.blocks = heads, page_size, pages * page_size // 16
        n = self.blocks * heads
        self.k, self.v = (torch.randint(0, 256, (n * 1024,), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2))
        self.k_scale, self.v_scale = (torch.randint(123, 127, (n * 64,), dtype=torch.uint8, device="cuda", generator=g) for _ in range(2))
        if poison:
            self.k_scale.fill_(255)
            self.v_scale.fill_(255)
        self.handle = hkv.kv_pool_create(pages, heads, self.dtype, self.k, self.v, self.k_scale, self.v_scale, free_order, page_size=page_size)

    def close(self):
        hkv.kv_pool_destroy(self.handle)

    def read(self):
        """(codes, scale bytes) of K, then of V: [blocks][heads][16][128] and [blocks][heads][16][4]."""
        out = []
        for is_k, buf, sc in ((True, self.k, self.k_scale), (False, self.v, self.v_scale)):
            b = buf.cpu().numpy().reshape(self.blocks, self.heads, 1024)
            t, d = np.arange(16)[:, None], np.arange(128)
            byte = b[:, :, code_at(is_k, t, d - d % 2)]
            out += [byte >> (4 * (d % 2)) & 15, sc.cpu().numpy().reshape(self.blocks, self.heads, 4, 16).transpose(0, 1, 3, 2)]
        return out

    def values(self):
        """K and V as they stand, [blocks][heads][16][128]."""
        kc, ks, vc, vs = self.read()
        return tuple(np.where(c > 7, -1, 1) * SIZES[c & 7] * np.repeat(np.exp2(s.astype(np.float64) - 127), 32, axis=-1) for c, s in ((kc, ks), (vc, vs)))


def blocks_of(pages, page_size):
    s = page_size // 16
    return np.asarray([p * s + j for p in pages for j in range(s)], dtype=np.int64)


def of_sequence(values, pages, page_size, n):
    """[n][heads][128] of a page list."""
    b = blocks_of(pages, page_size)
    t = np.arange(n)
    return values[b[t // 16], :, t % 16]


def attention(q, k, v, scale, seen):
    """q [heads of q][128], k and v [n][kv heads][128], seen [n] of truth values: out, lse, and what tolerances are made of: sum of p |v| per dim, and how far a
    score may be off: 130 roundings of 2^-24 of the largest sum of |q k| scale, and 2^-17 of the row's largest element for those below 2^-9 of it (decode
    splits a row of q into two terms of 4 bits each above the smallest step of 2^-9, the row's largest brought into [128, 256))."""
    hq, hk = q.shape[0], k.shape[1]
    out, weight, lse, size = np.zeros((hq, 128)), np.zeros((hq, 128)), np.full(hq, -math.inf), np.zeros(hq)
    if not seen.any():
        return out, lse, weight, size
    for h in range(hq):
        kk, vv = k[seen][:, h // (hq // hk)], v[seen][:, h // (hq // hk)]
        x = kk @ q[h] * scale
        far = np.where(np.abs(q[h]) < 2.0 ** -9 * np.abs(q[h]).max(), 2.0 ** -17 * np.abs(q[h]).max(), 0)
        size[h] = ((np.abs(kk) @ np.abs(q[h])) * 130 * STEP["fp32"] + np.abs(kk) @ far).max() * abs(scale)
        lse[h] = x.max() + math.log(np.exp(x - x.max()).sum())
        p = np.exp(x - lse[h])
        out[h], weight[h] = p @ vv, p @ np.abs(vv)
    return out, lse, weight, size


def check_rows(out, lse, ref, tile=False):
    """Rows of a kernel against attention()'s.  out: a probability is rounded to bf16 (half a step of 2^-8, into the sum of p |v|), the partial to 11 bits of the
    row's largest, the result to bf16; what a score is off by, p and lse carry, and some 160 roundings of sums and exponentials (1e-5)."""
    o, x, w, size = ref
    off = size + 1e-5
    tol = (2.0 ** -8 + 2 * off[..., None]) * w + 2.0 ** -11 * w.max(-1, keepdims=True)
    tol = tol + 2.0 ** -8 * (np.abs(o) + tol) + 1e-30
    assert (np.abs(out - o) <= tol).all(), float((np.abs(out - o) / tol).max())
    if lse is not None:
        empty = np.isneginf(x)
        assert (np.isneginf(lse) == empty).all()
        assert (np.abs(np.where(empty, 0, lse) - np.where(empty, 0, x)) <= off + 2.0 ** -22 * np.abs(np.where(empty, 0, x))).all()
